// dmr_attn_paged for few rows to a key head (decode, a few drafted tokens): bound by reading the keys and values once.
//
// A workgroup has all rows of a request to one key head, 16 or 32, and a part of its keys (share_of_item), dealt to its four waves in
// units of 32, or of 64 e4m3 ones.  Operands go from the cache straight into registers, 16 bytes a lane and whole lines a wave; the keys of the next unit
// are requested once the scores have used this one's, the values once the outputs have, 4 .. 16 KB each, and no barrier holds a wave.  Between
// the scores and the next keys lie the next unit's entries of the block table: vector loads, which return in order, so there, once a
// unit, a wave waits for its values and then for the table with nothing else in flight, and the other waves of the CU have the memory.  The rows are the columns of 16 x 16 x 32 MFMAs (S^T = K Q^T, O^T += V^T P^T): maximum
// and sum are per-lane numbers, and a lane's scores are the keys that its value pieces hold.  As the matrix cores have time to
// spare, the weights enter as two bf16 each, 16 bits.  The waves' results are joined in LDS, the workgroups' by a second kernel.
#include "attn.hpp"

namespace dmr {

namespace {

__device__ __forceinline__ float group_max(float v) {      // over lanes l, l ^ 16, l ^ 32, l ^ 48
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float group_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// By value: a choice between two elements of an array would keep the array in memory.
__device__ __forceinline__ int64_t either(bool second, int64_t a, int64_t b) { return second ? b : a; }

template <int D, bool E4M3, int NQ>
__global__ __launch_bounds__(256, E4M3 && D == 128 && NQ == 2 ? 1 : 2) void attn_few_kernel(AttnArgs a) {
    constexpr int ROWS = 16 * NQ, BLOCK = 16 * D * (E4M3 ? 1 : 2);
    constexpr int UNIT = few_unit(E4M3), TILES = UNIT / 16, STEPS = UNIT / 32;      // score tiles, steps of the second product
    constexpr int KL = E4M3 ? D / 64 : D / 32;       // loads of a score tile
    constexpr float kSlack = 8.f;                    // the reference of the exponents may lag the largest score by 2^8
    __shared__ float so[4][ROWS][D + 4];
    __shared__ float2 sml[4][ROWS];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
    const int head = (int)blockIdx.x % a.kv_heads, item = (int)blockIdx.x / a.kv_heads;
    Share sh;
    if (a.parts == 0) {
        sh = Share{item, 0, 0, 1, item, request_at(a, item)};
    } else {
        sh = share_of_item<UNIT>(a, item, lane);
        if (sh.b >= 0 && sh.part == 0 && head == 0 && tid == 0) a.split[sh.b] = make_int2(sh.first_item, sh.parts);
    }
    const Request rq = sh.rq;
    const int rows = min(rq.n * a.G, ROWS);
    if (sh.b < 0 || rows == 0) return;
    const int32_t *pages = a.table + (int64_t)sh.b * a.width;
    const int units = units_in<UNIT>(rq.keys);
    const int u0 = (int)((int64_t)units * sh.part / sh.parts), u1 = (int)((int64_t)units * (sh.part + 1) / sh.parts);
    const int last_block = max(rq.keys - 1, 0) >> 4;
    const int first_seen = rq.keys - rq.n + 1;       // keys that the first row sees; later ones see more

    // queries: lane (col, g) holds 8 elements of row col along each step of 32
    Frag q[NQ][D / 32];
    int seen[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = min(16 * n + col, rows - 1), token = row / a.G;
        seen[n] = first_seen + token;
        const uint16_t *src = a.q + ((int64_t)(rq.first + token) * a.q_heads + head * a.G + (row - token * a.G)) * D;
#pragma unroll
        for (int s = 0; s < D / 32; ++s)
            q[n][s].u = *reinterpret_cast<const uint4 *>(src + (E4M3 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g));
    }

    u32x4_t kf[TILES][KL], vf[D / 16];
    int64_t base[TILES];
    auto find = [&](int u) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) base[i] = uniform_block_offset<BLOCK>(a, pages, min(TILES * u + i, last_block), head);
    };
    auto pick = [&](int i) {                         // base[i] for a lane's own i
        if constexpr (TILES == 2) return either(i & 1, base[0], base[1]);
        else return either(i & 2, either(i & 1, base[0], base[1]), either(i & 1, base[2], base[3]));
    };
    auto load = [&](const uint8_t *p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p)); };
    // Row r of score tile T is key 8 (r / 4) + 4 T + r % 4 of the unit, with e4m3 key 16 (r / 4) + 4 T + r % 4: register i of lane group
    // g is then key 8 g + 4 T + i, or 16 g + 4 T + i, and two tiles are a run of 8.
    auto load_keys = [&] {
        const uint8_t *p = a.k + g * 256 + (col & 3) * 16 + (E4M3 ? pick(col >> 2) : pick(col >> 3) + (col & 4) * 32);
#pragma unroll
        for (int T = 0; T < TILES; ++T)
#pragma unroll
            for (int s = 0; s < KL; ++s) kf[T][s] = load(p + T * 64 + s * 1024);
    };
    auto load_values = [&] {
        const uint8_t *p = a.v + col * 16 + (E4M3 ? pick(g) : pick(g >> 1) + (g & 1) * (D * 16));
#pragma unroll
        for (int t = 0; t < D / 16; ++t) vf[t] = load(p + t * 256);
    };

    f32x4 o[NQ][D / 16];
    float m[NQ], l[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = kNoKey;
        l[n] = 0.f;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) o[n][t] = f32x4{};
    }
    auto frag = [](const u32x4_t &v) {
        Frag f;
        f.u = make_uint4(v[0], v[1], v[2], v[3]);
        return f;
    };

    auto unit = [&](int u, auto more) {
        constexpr bool MORE = decltype(more)::value;
        if constexpr (MORE) find(u + 4);
        f32x4 s[NQ][TILES];
#pragma unroll
        for (int T = 0; T < TILES; ++T) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) s[n][T] = f32x4{};
#pragma unroll
            for (int st = 0; st < D / 32; ++st) {
                Frag k;
                if constexpr (E4M3) {
                    const u32x4_t &r = kf[T][st >> 1];
                    k.u = st & 1 ? bf16_of_e4m3(r[2], r[3]) : bf16_of_e4m3(r[0], r[1]);
                } else {
                    k = frag(kf[T][st]);
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[n][T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.v, q[n][st].v, s[n][T], 0, 0, 0);
            }
        }
        if constexpr (MORE) load_keys();
        const int first = u * UNIT;
        const bool masked = first > first_seen - UNIT;
        Frag ph[NQ][STEPS], pl[NQ][STEPS];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float x[4 * TILES], top = kNoKey;
#pragma unroll
            for (int i = 0; i < 4 * TILES; ++i) x[i] = s[n][i >> 2][i & 3] * a.scale_log2;
            if (masked) {
                const int left = seen[n] - first;
#pragma unroll
                for (int i = 0; i < 4 * TILES; ++i) {
                    const int T = i >> 2, key = (E4M3 ? 16 : 8) * g + 4 * T + (i & 3);
                    x[i] = key < left ? x[i] : -INFINITY;
                }
            }
#pragma unroll
            for (int i = 0; i < 4 * TILES; ++i) top = fmaxf(top, x[i]);
            // only then is the reference moved, and with it what was summed so far
            if (__any(top > m[n] + kSlack)) {
                const float to = fmaxf(m[n], group_max(top)), fade = exp2_fast(m[n] - to);
                m[n] = to;
                l[n] *= fade;
#pragma unroll
                for (int t = 0; t < D / 16; ++t) o[n][t] *= fade;
            }
#pragma unroll
            for (int i = 0; i < 4 * TILES; i += 2) {
                const float e0 = exp2_fast(x[i] - m[n]), e1 = exp2_fast(x[i + 1] - m[n]);
                l[n] += e0 + e1;
                const uint32_t hi = pack_bf16x2(e0, e1);
                ph[n][i >> 3].w[(i & 7) >> 1] = hi;
                pl[n][i >> 3].w[(i & 7) >> 1] = pack_bf16x2(e0 - __uint_as_float(hi << 16), e1 - __uint_as_float(hi & 0xFFFF0000u));
            }
        }
        // values of slots behind the last key may hold anything, and 0 x NaN is NaN
        uint32_t keep[STEPS][4];
        const bool ragged = first > rq.keys - UNIT;
        if (ragged) {
#pragma unroll
            for (int st = 0; st < STEPS; ++st)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int left = rq.keys - first - (E4M3 ? 16 * g + 8 * st : 8 * g) - 2 * w;
                    keep[st][w] = (left > 0 ? 0xFFFFu : 0u) | (left > 1 ? 0xFFFF0000u : 0u);
                }
        }
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
#pragma unroll
            for (int t = 0; t < D / 16; ++t) {
                Frag v;
                if constexpr (E4M3) {
                    const u32x4_t &r = vf[t];
                    v.u = st ? bf16_of_e4m3(r[2], r[3]) : bf16_of_e4m3(r[0], r[1]);
                } else {
                    v = frag(vf[t]);
                }
                if (ragged)
#pragma unroll
                    for (int w = 0; w < 4; ++w) v.w[w] &= keep[st][w];
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, ph[n][st].v, o[n][t], 0, 0, 0);
                    o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, pl[n][st].v, o[n][t], 0, 0, 0);
                }
            }
        if constexpr (MORE) load_values();
    };

    int u = u0 + wave;
    if (u < u1) {
        find(u);
        load_keys();
        load_values();
        for (; u + 4 < u1; u += 4) unit(u, std::true_type{});
        unit(u, std::false_type{});
    }

    // the four waves' results: register i of tile t is element 16 t + 4 g + i of row col
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float sum = group_sum(l[n]);
        if (g == 0) sml[wave][16 * n + col] = make_float2(m[n], sum);
#pragma unroll
        for (int t = 0; t < D / 16; ++t) *reinterpret_cast<f32x4 *>(&so[wave][16 * n + col][16 * t + 4 * g]) = o[n][t];
    }
    __syncthreads();
    constexpr int PER_ROW = D / 8;
    for (int i = tid; i < rows * PER_ROW; i += 256) {
        const int row = i / PER_ROW, d = (i - row * PER_ROW) * 8;
        float M = kNoKey, L = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, sml[w][row].x);
        float acc[8] = {};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 ml = sml[w][row];
            const float f = exp2_fast(ml.x - M);
            L = fmaf(f, ml.y, L);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf(f, so[w][row][d + e], acc[e]);
        }
        if (sh.parts == 1) {
            const float r = L > 0.f ? a.v_scale / L : 0.f;
            const int token = row / a.G;
            const int64_t at = ((int64_t)(rq.first + token) * a.q_heads + head * a.G + (row - token * a.G)) * D + d;
            *reinterpret_cast<uint4 *>(a.out + at) =
                make_uint4(pack_bf16x2(acc[0] * r, acc[1] * r), pack_bf16x2(acc[2] * r, acc[3] * r), pack_bf16x2(acc[4] * r, acc[5] * r),
                           pack_bf16x2(acc[6] * r, acc[7] * r));
        } else {
            const int64_t slot = ((int64_t)item * a.kv_heads + head) * ROWS + row;
            if (d == 0) a.ml[slot] = make_float2(M, L);
            f32x4 *dst = reinterpret_cast<f32x4 *>(a.part + slot * D + d);
            dst[0] = f32x4{acc[0], acc[1], acc[2], acc[3]};
            dst[1] = f32x4{acc[4], acc[5], acc[6], acc[7]};
        }
    }
}

}  // namespace

hipError_t launch_attn_few(const AttnArgs &a, const AttnPlan &p, int D, bool e4m3, hipStream_t stream) {
    const dim3 grid((unsigned)(p.items * a.kv_heads));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
    auto rows = [&](auto d, auto e) {
        constexpr int DIM = decltype(d)::value;
        constexpr bool E = decltype(e)::value;
        if (p.tile_rows == 16) go(attn_few_kernel<DIM, E, 1>); else go(attn_few_kernel<DIM, E, 2>);
    };
    auto type = [&](auto d) {
        if (e4m3) rows(d, std::true_type{}); else rows(d, std::false_type{});
    };
    if (D == 64) type(std::integral_constant<int, 64>{}); else type(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace dmr
