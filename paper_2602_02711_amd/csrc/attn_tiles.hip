// dmr_attn_paged for many rows to a key head: a workgroup of four waves has 128 (token, query head) rows of one request and one key
// head, 32 to a wave, and walks along the keys up to its last row's, 64 at a time, staged in LDS for all four waves.
//
// S^T = K Q^T on 32 x 32 x 16 MFMAs leaves lane l with the scores of query l % 32 for 16 keys of each 32, so the running maximum and
// sum are per-lane numbers, and the weights, rounded to bf16 in place, are the B operand of O^T += V^T P^T, whose columns are
// the queries again.  Row r of a score tile is key key_of_row(r): the order in which lane half l / 32 then holds 8 consecutive
// keys of each 16, as the pieces of the value pool do.
#include "attn.hpp"

namespace dmr {

namespace {

constexpr int kRows = 128;      // of a tile
constexpr int kUnit = 64;       // keys staged at a time

template <int D, bool E4M3>
__global__ __launch_bounds__(256, 1) void attn_tiles_kernel(AttnArgs a) {
    constexpr int BLOCK = 16 * D * 2;                         // bytes of a block as bf16
    constexpr int SRC = E4M3 ? 16 * D : 16 * D * 2;           // and in the cache
    constexpr int PIECES = SRC / 16;                          // of 16 bytes
    __shared__ __align__(16) uint8_t sk[4 * BLOCK], sv[4 * BLOCK];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, h = lane >> 5;
    const int head = (int)blockIdx.x % a.kv_heads, item = (int)blockIdx.x / a.kv_heads;
    const int part = item % a.parts;
    const Share sh = share_of_tile(a, item / a.parts, kRows, lane);
    if (sh.b < 0) return;
    const Request rq = sh.rq;
    const int tile = sh.tile;
    const int rows = rq.n * a.G, row0 = tile * kRows;
    const int32_t *pages = a.table + (int64_t)sh.b * a.width;
    // this lane's query; rows past the last repeat it
    const int row = min(row0 + 32 * wave + col, rows - 1), token = row / a.G, qh = head * a.G + row % a.G;
    const int64_t q_at = ((int64_t)(rq.first + token) * a.q_heads + qh) * D;
    const int seen = rq.keys - rq.n + token + 1;              // keys this lane's query sees
    const int most = rq.keys - rq.n + min(row0 + kRows - 1, rows - 1) / a.G + 1;      // and the tile's last one
    const int units = most > 0 ? (most + kUnit - 1) / kUnit : 0;
    const int u0 = (int)((int64_t)units * part / a.parts), u1 = (int)((int64_t)units * (part + 1) / a.parts);

    Frag q[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) q[s].u = *reinterpret_cast<const uint4 *>(a.q + q_at + 16 * s + 8 * h);
    f32x16 o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) o[t] = f32x16{};
    float m = kNoKey, l = 0.f;
    const int last_block = (rq.keys - 1) >> 4;
    const int key_row = 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3), key_block = col >> 4;

    for (int u = u0; u < u1; ++u) {
        __syncthreads();
#pragma unroll
        for (int blk = 0; blk < 4; ++blk) {
            const int64_t src = block_offset<SRC>(a, pages, min(4 * u + blk, last_block), head);
            for (int p = tid; p < PIECES; p += 256) {
                const uint4 kp = *reinterpret_cast<const uint4 *>(a.k + src + 16 * p);
                const uint4 vp = *reinterpret_cast<const uint4 *>(a.v + src + 16 * p);
                if constexpr (E4M3) {
                    uint8_t *dk = sk + blk * BLOCK + (p >> 4) * 512 + (p & 15) * 16;      // pieces 2 p' and 2 p' + 1 of a token
                    *reinterpret_cast<uint4 *>(dk) = bf16_of_e4m3(kp.x, kp.y);
                    *reinterpret_cast<uint4 *>(dk + 256) = bf16_of_e4m3(kp.z, kp.w);
                    uint8_t *dv = sv + blk * BLOCK + p * 16;                              // tokens 0 .. 7 and 8 .. 15 of an element
                    *reinterpret_cast<uint4 *>(dv) = bf16_of_e4m3(vp.x, vp.y);
                    *reinterpret_cast<uint4 *>(dv + D * 16) = bf16_of_e4m3(vp.z, vp.w);
                } else {
                    *reinterpret_cast<uint4 *>(sk + blk * BLOCK + 16 * p) = kp;
                    *reinterpret_cast<uint4 *>(sv + blk * BLOCK + 16 * p) = vp;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int base = u * kUnit + 32 * half;
            f32x16 s = f32x16{};
#pragma unroll
            for (int st = 0; st < D / 16; ++st) {
                Frag k;
                k.u = *reinterpret_cast<const uint4 *>(sk + (2 * half + key_block) * BLOCK + (2 * st + h) * 256 + key_row * 16);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.v, q[st].v, s, 0, 0, 0);
            }
            // register i is key base + 16 (i / 8) + 8 h + i % 8
            float x[16], top = kNoKey;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = base + 16 * (i >> 3) + 8 * h + (i & 7);
                x[i] = key < seen ? s[i] * a.scale_log2 : -INFINITY;
                top = fmaxf(top, x[i]);
            }
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m, top), fade = exp2_fast(m - m_new);
            m = m_new;
            l *= fade;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= fade;
            Frag p[2];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float e0 = exp2_fast(x[i] - m), e1 = exp2_fast(x[i + 1] - m);
                const uint32_t w = pack_bf16x2(e0, e1);
                p[i >> 3].w[(i & 7) >> 1] = w;
                l += __uint_as_float(w << 16) + __uint_as_float(w & 0xFFFF0000u);
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                // values of slots behind the last key may hold anything: 0 x NaN is NaN
                const int left = rq.keys - (base + 16 * st + 8 * h);
                uint32_t mask[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) mask[w] = (2 * w < left ? 0xFFFFu : 0u) | (2 * w + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
                for (int t = 0; t < D / 32; ++t) {
                    Frag v;
                    v.u = *reinterpret_cast<const uint4 *>(sv + (2 * half + st) * BLOCK + h * (D * 16) + (32 * t + col) * 16);
#pragma unroll
                    for (int w = 0; w < 4; ++w) v.w[w] &= mask[w];
                    o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v, p[st].v, o[t], 0, 0, 0);
                }
            }
        }
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
    if (h == 0) a.ml[slot] = make_float2(m, l);
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
