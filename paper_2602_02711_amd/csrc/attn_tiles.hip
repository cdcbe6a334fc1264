// dmr_attn_paged for many rows to a key head: a workgroup of four waves has 128 (token, query head) rows of one request and one key
// head, 32 to a wave, and walks along the keys up to its last row's, 64 at a time, staged in LDS for all four waves.
//
// S^T = K Q^T on 32 x 32 x 16 MFMAs leaves lane l with the scores of query l % 32 for 16 keys of each 32, so the exponents' reference and
// the running sum are per-lane numbers, and the weights, rounded to bf16 in place (as many bits as the values have: 16 would take
// a second product), are the B operand of O^T += V^T P^T, whose columns are the queries again.  Row r of a score tile is key
// 8 (r / 4 % 2) + 4 (r / 8 % 2) + r % 4 of block r / 16: the order in which lane half l / 32 then holds 8 consecutive keys of each 16,
// as the pieces of the value pool do.
//
// The keys and values of the next 64 arrive while these are worked on: bf16 ones by loads into the other half of the buffer, e4m3
// ones through registers, where a thread makes them bf16 once for all four waves, before the last products (at the unit's end 4 %
// slower).  One barrier for each 64 keys; a second workgroup on the CU works through it.
//
// Bound by power: 2048 rows over 32768 keys run at 1.7 GHz with the matrix pipes busy 64 % of the cycles, as long bf16 products do;
// 910 .. 960 us, 1.11 .. 1.17 PFLOP/s, where one of 8192^3 reaches 1.14 .. 1.28.  What brought it there, from 1840 us: loads ahead and masks at
// the edges alone, 1072; a loop of its own for units without an edge (the branch inside kept copies of all accumulators) and the
// maximum looked for only when a sum says so, 9 % less; every operand read from LDS eight MFMAs before its own, 6 %; the tiles with
// the most keys first, 8 .. 12 % of a causal prompt; priority for the wave that is at its products, 2 %.  Eight waves on the same
// keys, 64 rows to a wave, 32 keys at a time, and the weights of one half among the other's products were level or slower.
#include "attn.hpp"
#include "lds_loads.hpp"

namespace dmr {

namespace {

constexpr int kRows = 128;         // of a tile
constexpr int kUnit = 64;          // keys staged at a time
// A lane's 32 weights of a unit may sum to this before the reference of its row's exponents is moved to the largest score so far.
constexpr float kMost = 4096.f;

typedef __attribute__((ext_vector_type(2))) __bf16 pair_bf16;

// N times an MFMA and a read from LDS, in turn: what the reads bring is used a group later.
template <int N, int GROUP>
__device__ __forceinline__ void read_among_products() {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, GROUP);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, GROUP);
    }
    __builtin_amdgcn_sched_barrier(0);
}

template <int D, bool E4M3>
__global__ __launch_bounds__(256, 2) void attn_tiles_kernel(AttnArgs a) {
    constexpr int BLOCK = 16 * D * 2;                         // bytes of a block as bf16
    constexpr int SRC = E4M3 ? 16 * D : 16 * D * 2;           // and in the cache
    constexpr int STAGE = 4 * BLOCK;                          // keys of a unit, and values
    constexpr int KS = D / 16, VT = D / 32;                   // steps of the first product, tiles of the second
    __shared__ __align__(16) uint8_t lds[4 * STAGE];          // [2][keys, values]
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    // the last tiles of a request have the most keys: they start first
    const int head = (int)blockIdx.x % a.kv_heads, item = a.items - 1 - (int)blockIdx.x / a.kv_heads;
    const int part = item % a.parts;
    const Share sh = share_of_tile(a, item / a.parts, kRows, lane);
    if (sh.b < 0) return;
    const Request rq = sh.rq;
    const int rows = rq.n * a.G, row0 = sh.tile * kRows;
    const int32_t *pages = a.table + (int64_t)sh.b * a.width;
    // this lane's query; rows past the last repeat it
    const int row = min(row0 + 32 * wave + col, rows - 1), token = row / a.G, qh = head * a.G + row % a.G;
    const int64_t q_at = ((int64_t)(rq.first + token) * a.q_heads + qh) * D;
    const int seen = rq.keys - rq.n + token + 1;              // keys this lane's query sees
    auto seen_by = [&](int r) { return rq.keys - rq.n + min(r, rows - 1) / a.G + 1; };
    const int most = seen_by(row0 + kRows - 1);               // the tile's last row
    // and the first and the last of the wave's; a wave without rows stages what the others read
    const bool any = row0 + 32 * wave < rows;
    const int wave_least = any ? seen_by(row0 + 32 * wave) : 0, wave_most = any ? seen_by(row0 + 32 * wave + 31) : 0;
    const int units = most > 0 ? units_in<kUnit>(most) : 0;
    const int u0 = (int)((int64_t)units * part / a.parts), u1 = (int)((int64_t)units * (part + 1) / a.parts);

    Frag q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s].u = *reinterpret_cast<const uint4 *>(a.q + q_at + 16 * s + 8 * h);
    f32x16 o[VT];
#pragma unroll
    for (int t = 0; t < VT; ++t) o[t] = f32x16{};
    float m = kNoKey, l = 0.f;
    const int last_block = (rq.keys - 1) >> 4;
    const int key_row = 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3), key_block = col >> 4;

    // staging: pieces of 16 bytes, a block at a time to each wave or pair of waves
    constexpr int CHUNKS = E4M3 ? 4 * SRC / 4096 : 1;
    u32x4_t hk[CHUNKS], hv[CHUNKS];
    auto request = [&](int u, int buf) {
        if constexpr (E4M3) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int blk = (i * 256 + wave * 64) / (SRC / 16), p = (i * 256 + tid) % (SRC / 16);
                const int64_t src = uniform_block_offset<SRC>(a, pages, min(4 * u + blk, last_block), head) + 16 * p;
                hk[i] = *reinterpret_cast<const u32x4_t *>(a.k + src);
                hv[i] = *reinterpret_cast<const u32x4_t *>(a.v + src);
            }
        } else {
            uint8_t *dst = lds + buf * (2 * STAGE);
#pragma unroll
            for (int blk = 0; blk < 4; ++blk) {
                const int64_t src = uniform_block_offset<SRC>(a, pages, min(4 * u + blk, last_block), head);
                if constexpr (D == 128) {
                    load16_to_lds(a.k + src, BLOCK, dst + blk * BLOCK + wave * 1024, (uint32_t)(tid * 16), 0);
                    load16_to_lds(a.v + src, BLOCK, dst + STAGE + blk * BLOCK + wave * 1024, (uint32_t)(tid * 16), 0);
                } else {      // keys to two waves, values to the others
                    load16_to_lds((wave & 2 ? a.v : a.k) + src, BLOCK, dst + (wave & 2 ? STAGE : 0) + blk * BLOCK + (wave & 1) * 1024,
                                  (uint32_t)((tid & 127) * 16), 0);
                }
            }
        }
    };
    // e4m3 pieces that have come, as bf16 into LDS (after the last unit nothing has, and nothing reads what this leaves)
    auto deposit = [&](int buf) {
        if constexpr (E4M3) {
            uint8_t *dst = lds + buf * (2 * STAGE);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int blk = (i * 256 + wave * 64) / (SRC / 16), p = (i * 256 + tid) % (SRC / 16);
                uint8_t *dk = dst + blk * BLOCK + (p >> 4) * 512 + (p & 15) * 16;      // pieces 2 p' and 2 p' + 1 of a token
                *reinterpret_cast<uint4 *>(dk) = bf16_of_e4m3(hk[i][0], hk[i][1]);
                *reinterpret_cast<uint4 *>(dk + 256) = bf16_of_e4m3(hk[i][2], hk[i][3]);
                uint8_t *dv = dst + STAGE + blk * BLOCK + p * 16;                      // tokens 0 .. 7 and 8 .. 15 of an element
                *reinterpret_cast<uint4 *>(dv) = bf16_of_e4m3(hv[i][0], hv[i][1]);
                *reinterpret_cast<uint4 *>(dv + D * 16) = bf16_of_e4m3(hv[i][2], hv[i][3]);
            }
        }
    };
    // what was requested or deposited lies in LDS, and every wave is done with the buffer before
    auto settle = [&] {
        if constexpr (E4M3) wait_lds(); else wait_loads<0>();
        bare_barrier();
    };

    // EDGE: some key of the unit is not seen by some row of the wave, or lies behind the request's last
    auto unit = [&](int first, int buf, auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
        const uint8_t *sk = lds + buf * (2 * STAGE) + key_block * BLOCK + h * 256 + key_row * 16;
        const uint8_t *sv = lds + buf * (2 * STAGE) + STAGE + h * (D * 16) + col * 16;
        Frag k[2][KS], v[2][2 * VT], p[2][2];
        auto read_values = [&](int half) {
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                Frag w[VT];
                read_frags<VT, 512>(sv + (2 * half + st) * BLOCK, sv + (2 * half + st) * BLOCK, w);
#pragma unroll
                for (int t = 0; t < VT; ++t) v[half][st * VT + t] = w[t];
            }
        };
        f32x16 s[2];
        auto scores = [&](int half) {
            s[half] = f32x16{};
#pragma unroll
            for (int st = 0; st < KS; ++st) s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[half][st].v, q[st].v, s[half], 0, 0, 0);
        };
        // 2^(score - m) in bf16; returns their sum
        auto weigh = [&] {
            float sum = 0.f;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float e0 = exp2_fast(fmaf(s[half][i], a.scale_log2, -m)), e1 = exp2_fast(fmaf(s[half][i + 1], a.scale_log2, -m));
                    const uint32_t w = pack_bf16x2(e0, e1);
                    p[half][i >> 3].w[(i & 7) >> 1] = w;
                    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair_bf16, w), __builtin_bit_cast(pair_bf16, 0x3F803F80u), sum, false);
                }
            return sum;
        };
        auto outputs = [&](int half) {
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                if constexpr (EDGE) {      // values of slots behind the last key may hold anything, and 0 x NaN is NaN
                    const int left = rq.keys - (first + 32 * half + 16 * st + 8 * h);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t keep = (2 * w < left ? 0xFFFFu : 0u) | (2 * w + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int t = 0; t < VT; ++t) v[half][st * VT + t].w[w] &= keep;
                    }
                }
#pragma unroll
                for (int t = 0; t < VT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[half][st * VT + t].v, p[half][st].v, o[t], 0, 0, 0);
            }
        };

        __builtin_amdgcn_s_setprio(1);
        read_frags<KS, 512>(sk, sk, k[0]);
        __builtin_amdgcn_sched_barrier(0);
        read_frags<KS, 512>(sk + 2 * BLOCK, sk + 2 * BLOCK, k[1]);
        scores(0);
        read_among_products<KS, 0>();
        read_values(0);
        scores(1);
        read_among_products<KS, 1>();
        if constexpr (EDGE) {      // register i of a half is key first + 32 half + 16 (i / 8) + 8 h + i % 8
            const int left = seen - first - 8 * h;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[half][i] = 32 * half + 16 * (i >> 3) + (i & 7) < left ? s[half][i] : -INFINITY;
        }
        __builtin_amdgcn_s_setprio(0);
        float sum = weigh();
        // the first unit comes here (its reference is still kNoKey), and then few: what was summed so far fades to the new reference
        if (__builtin_expect(__any(!(sum <= kMost)), 0)) {
            float top = kNoKey;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 16; i += 2) top = fmaxf(top, fmaxf(s[half][i], s[half][i + 1]));
            top *= a.scale_log2;
            const float to = fmaxf(m, fmaxf(top, __shfl_xor(top, 32))), fade = exp2_fast(m - to);
            m = to;
            l *= fade;
#pragma unroll
            for (int t = 0; t < VT; ++t) o[t] *= fade;
            sum = weigh();
        }
        l += sum;
        __builtin_amdgcn_s_setprio(1);
        read_values(1);
        outputs(0);
        read_among_products<2 * VT, 2>();
        deposit(buf ^ 1);
        outputs(1);
    };

    if (u0 < u1) {
        request(u0, 0);
        deposit(0);
        settle();
    }
    const int whole = min(u1, max(u0, wave_least / kUnit));
    int u = u0;
    for (; u < whole; ++u) {
        const int buf = (u - u0) & 1;
        if (u + 1 < u1) request(u + 1, buf ^ 1);
        unit(u * kUnit, buf, std::false_type{});
        if (u + 1 < u1) settle();
    }
    for (; u < u1; ++u) {
        const int buf = (u - u0) & 1;
        if (u + 1 < u1) request(u + 1, buf ^ 1);
        if (u * kUnit < wave_most) unit(u * kUnit, buf, std::true_type{});
        else deposit(buf ^ 1);
        if (u + 1 < u1) settle();
    }
    l += __shfl_xor(l, 32);
    if (row0 + 32 * wave + col >= rows) return;
    // register 4 c + e of tile t is element 32 t + 8 c + 4 h + e
    if (a.parts == 1) {
        const float r = l > 0.f ? a.v_scale / l : 0.f;
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *reinterpret_cast<uint2 *>(a.out + q_at + 32 * t + 8 * c + 4 * h) =
                    make_uint2(pack_bf16x2(o[t][4 * c] * r, o[t][4 * c + 1] * r), pack_bf16x2(o[t][4 * c + 2] * r, o[t][4 * c + 3] * r));
        return;
    }
    const int64_t slot = ((int64_t)item * a.kv_heads + head) * kRows + 32 * wave + col;
    if (h == 0) a.ml[slot] = make_float2(m, l);
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const f32x4 v = {o[t][4 * c], o[t][4 * c + 1], o[t][4 * c + 2], o[t][4 * c + 3]};
            *reinterpret_cast<f32x4 *>(a.part + slot * D + 32 * t + 8 * c + 4 * h) = v;
        }
}

}  // namespace

hipError_t launch_attn_tiles(const AttnArgs &a, int D, bool e4m3, hipStream_t stream) {
    const dim3 grid((unsigned)(a.items * a.kv_heads));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
    if (D == 64) {
        if (e4m3) go(attn_tiles_kernel<64, true>); else go(attn_tiles_kernel<64, false>);
    } else {
        if (e4m3) go(attn_tiles_kernel<128, true>); else go(attn_tiles_kernel<128, false>);
    }
    return hipGetLastError();
}

}  // namespace dmr
