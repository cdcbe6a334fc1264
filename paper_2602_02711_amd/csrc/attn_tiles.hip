// dmr_attn_paged for many rows to a key head: a workgroup of four waves has 128 (token, query head) rows of one request and one key
// head, 32 to a wave, and walks along the keys up to its last row's, 64 at a time, staged in LDS for all four waves.
//
// S^T = K Q^T on 32 x 32 x 16 MFMAs leaves lane l with the scores of query l % 32 for 16 keys of each 32, so the running maximum and
// sum are per-lane numbers, and the weights, rounded to bf16 in place, are the B operand of O^T += V^T P^T, whose columns are
// the queries again.  Row r of a score tile is key 8 (r / 4 % 2) + 4 (r / 8 % 2) + r % 4 of block r / 16: the order in which lane half
// l / 32 then holds 8 consecutive keys of each 16, as the pieces of the value pool do.
//
// The keys and values of the next 64 arrive while these are worked on: bf16 ones by loads into the other half of the buffer, e4m3
// ones through registers, where a thread makes them bf16 once for all four waves.  One barrier for each 64 keys.
#include "attn.hpp"
#include "lds_loads.hpp"

namespace dmr {

namespace {

constexpr int kRows = 128;      // of a tile
constexpr int kUnit = 64;       // keys staged at a time
constexpr float kMost = 4096.f; // a lane's 32 weights of a unit may sum to this before the reference of its row's exponents is moved

typedef __attribute__((ext_vector_type(2))) __bf16 pair_bf16;

template <int D, bool E4M3>
__global__ __launch_bounds__(256, 2) void attn_tiles_kernel(AttnArgs a) {
    constexpr int BLOCK = 16 * D * 2;                         // bytes of a block as bf16
    constexpr int SRC = E4M3 ? 16 * D : 16 * D * 2;           // and in the cache
    constexpr int STAGE = 4 * BLOCK;                          // keys of a unit, and values
    __shared__ __align__(16) uint8_t lds[4 * STAGE];          // [2][keys, values]
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const int head = (int)blockIdx.x % a.kv_heads, item = (int)blockIdx.x / a.kv_heads;
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
    const int wave_least = __builtin_amdgcn_readfirstlane(seen_by(row0 + 32 * wave));
    const int wave_most = __builtin_amdgcn_readfirstlane(row0 + 32 * wave < rows ? seen_by(row0 + 32 * wave + 31) : 0);
    const int units = most > 0 ? (most + kUnit - 1) / kUnit : 0;
    const int u0 = (int)((int64_t)units * part / a.parts), u1 = (int)((int64_t)units * (part + 1) / a.parts);

    Frag q[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) q[s].u = *reinterpret_cast<const uint4 *>(a.q + q_at + 16 * s + 8 * h);
    f32x16 o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) o[t] = f32x16{};
    // scores come out of the first product less the row's reference, the negative of which it starts from
    f32x16 lag = f32x16{};
    float l = 0.f;
    const int last_block = (rq.keys - 1) >> 4;
    const int key_row = 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3), key_block = col >> 4;

    // staging: with bf16, load i of a block is 4 KB (2 KB where D is 64: two waves' worth each); e4m3 pieces in registers
    constexpr int CHUNKS = E4M3 ? 4 * SRC / 4096 : 0;         // 16-byte pieces of a unit's keys, and values, for each thread
    u32x4_t hk[CHUNKS ? CHUNKS : 1], hv[CHUNKS ? CHUNKS : 1];
    auto request = [&](int u, int buf) {
        if constexpr (E4M3) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int piece = i * 256 + tid, blk = piece / (SRC / 16), p = piece % (SRC / 16);
                const int64_t src = block_offset<SRC>(a, pages, min(4 * u + blk, last_block), head) + 16 * p;
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
                } else {
                    // half of a block's keys and half of its values to each pair of waves
                    const uint8_t *from = wave & 2 ? a.v : a.k;
                    uint8_t *to = dst + (wave & 2 ? STAGE : 0) + blk * BLOCK + (wave & 1) * 1024;
                    load16_to_lds(from + src, BLOCK, to, (uint32_t)((tid & 127) * 16), 0);
                }
            }
        }
    };
    auto arrive = [&](int buf) {
        if constexpr (E4M3) {
            uint8_t *dst = lds + buf * (2 * STAGE);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int piece = i * 256 + tid, blk = piece / (SRC / 16), p = piece % (SRC / 16);
                uint8_t *dk = dst + blk * BLOCK + (p >> 4) * 512 + (p & 15) * 16;      // pieces 2 p' and 2 p' + 1 of a token
                *reinterpret_cast<uint4 *>(dk) = bf16_of_e4m3(hk[i][0], hk[i][1]);
                *reinterpret_cast<uint4 *>(dk + 256) = bf16_of_e4m3(hk[i][2], hk[i][3]);
                uint8_t *dv = dst + STAGE + blk * BLOCK + p * 16;                      // tokens 0 .. 7 and 8 .. 15 of an element
                *reinterpret_cast<uint4 *>(dv) = bf16_of_e4m3(hv[i][0], hv[i][1]);
                *reinterpret_cast<uint4 *>(dv + D * 16) = bf16_of_e4m3(hv[i][2], hv[i][3]);
            }
            wait_lds();
        } else {
            wait_loads<0>();
        }
        bare_barrier();
    };

    // EDGE: some key of the unit is not seen by some row of the wave, or lies behind the request's last
    auto unit = [&](int first, int buf, bool start, auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
        const uint8_t *sk = lds + buf * (2 * STAGE) + key_block * BLOCK + h * 256 + key_row * 16;
        const uint8_t *sv = lds + buf * (2 * STAGE) + STAGE + h * (D * 16) + col * 16;
        Frag k[2][D / 16], v[2][D / 16];
        auto read_values = [&](int half) {
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                Frag w[D / 32];
                read_frags<D / 32, 512>(sv + (2 * half + st) * BLOCK, sv + (2 * half + st) * BLOCK, w);
#pragma unroll
                for (int t = 0; t < D / 32; ++t) v[half][st * (D / 32) + t] = w[t];
            }
        };
        f32x16 s[2];
        read_frags<D / 16, 512>(sk, sk, k[0]);
        read_frags<D / 16, 512>(sk + 2 * BLOCK, sk + 2 * BLOCK, k[1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int st = 0; st < D / 16; ++st)
                s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[half][st].v, q[st].v, st ? s[half] : lag, 0, 0, 0);
            if (half == 0) {
                read_values(0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // register i of half is key first + 32 half + 16 (i / 8) + 8 h + i % 8
        if constexpr (EDGE) {
            const int left = seen - first - 8 * h;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[half][i] = 32 * half + 16 * (i >> 3) + (i & 7) < left ? s[half][i] : -INFINITY;
        }
        Frag p[2][2];
        float sum;
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            sum = 0.f;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const uint32_t w = pack_bf16x2(exp2_fast(s[half][i] * a.scale_log2), exp2_fast(s[half][i + 1] * a.scale_log2));
                    p[half][i >> 3].w[(i & 7) >> 1] = w;
                    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair_bf16, w), __builtin_bit_cast(pair_bf16, 0x3F803F80u), sum, false);
                }
            if (pass || !(start || __any(!(sum <= kMost)))) break;
            float top = -INFINITY;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[half][i]);
            top = fmaxf(top, __shfl_xor(top, 32));
            if (top == -INFINITY || !(start || top > 0.f)) top = 0.f;
            lag -= top;
            s[0] -= top;
            s[1] -= top;
            if (!start) {
                const float fade = exp2_fast(-top * a.scale_log2);
                l *= fade;
#pragma unroll
                for (int t = 0; t < D / 32; ++t) o[t] *= fade;
            }
        }
        l += sum;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half == 0) read_values(1);
            if constexpr (EDGE) {      // values of slots behind the last key may hold anything, and 0 x NaN is NaN
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const int left = rq.keys - (first + 32 * half + 16 * st + 8 * h);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t keep = (2 * w < left ? 0xFFFFu : 0u) | (2 * w + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int t = 0; t < D / 32; ++t) v[half][st * (D / 32) + t].w[w] &= keep;
                    }
                }
            }
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int t = 0; t < D / 32; ++t)
                    o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[half][st * (D / 32) + t].v, p[half][st].v, o[t], 0, 0, 0);
        }
    };

    if (u0 < u1) {
        request(u0, 0);
        arrive(0);
    }
    for (int u = u0; u < u1; ++u) {
        const int buf = (u - u0) & 1, first = u * kUnit;
        if (u + 1 < u1) request(u + 1, buf ^ 1);
        if (first + kUnit <= wave_least) unit(first, buf, u == u0, std::false_type{});
        else if (first < wave_most) unit(first, buf, u == u0, std::true_type{});
        if (u + 1 < u1) arrive(buf ^ 1);
    }
    l += __shfl_xor(l, 32);
    if (row0 + 32 * wave + col >= rows) return;
    // register 4 c + e of tile t is element 32 t + 8 c + 4 h + e
    if (a.parts == 1) {
        const float r = l > 0.f ? a.v_scale / l : 0.f;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *reinterpret_cast<uint2 *>(a.out + q_at + 32 * t + 8 * c + 4 * h) =
                    make_uint2(pack_bf16x2(o[t][4 * c] * r, o[t][4 * c + 1] * r), pack_bf16x2(o[t][4 * c + 2] * r, o[t][4 * c + 3] * r));
        return;
    }
    const int64_t slot = ((int64_t)item * a.kv_heads + head) * kRows + 32 * wave + col;
    if (h == 0) a.ml[slot] = make_float2(l > 0.f ? -lag[0] * a.scale_log2 : kNoKey, l);
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
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
