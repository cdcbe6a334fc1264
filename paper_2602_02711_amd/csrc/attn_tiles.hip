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

template <int D, bool E4M3>
__global__ __launch_bounds__(256, 1) void attn_tiles_kernel(AttnArgs a) {
    constexpr int BLOCK = 16 * D * 2;                         // bytes of a block as bf16
    constexpr int SRC = E4M3 ? 16 * D : 16 * D * 2;           // and in the cache
    constexpr int PIECES = SRC / 16;                          // of 16 bytes
    __shared__ __align__(16) uint8_t sk[4 * BLOCK], sv[4 * BLOCK];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, h = lane >> 5;
    const int head = (int)blockIdx.x % a.kv_heads, item = (int)blockIdx.x / a.kv_heads;
    int tile = item / a.parts;
    const int part = item - tile * a.parts;

    // which request has this tile
    int b = -1;
    Request rq{0, 0, 0};
    for (int base = 0; base < a.requests; base += 64) {
        const int i = base + lane;
        const Request r = i < a.requests ? request_at(a, i) : Request{0, 0, 0};
        const int64_t tiles = ((int64_t)r.n * a.G + kRows - 1) / kRows;
        int64_t upto = tiles;
        for (int d = 1; d < 64; d *= 2) {
            const int64_t u = __shfl_up(upto, d);
            if (lane >= d) upto += u;
        }
        const uint64_t above = __ballot(upto > tile);
        if (above) {
            const int l = __builtin_ctzll(above);
            tile -= (int)__shfl(upto - tiles, l);
            b = base + l;
            rq = Request{__shfl(r.first, l), __shfl(r.n, l), __shfl(r.keys, l)};
            break;
        }
        tile -= (int)__shfl(upto, 63);
    }
    if (b < 0) return;
    const int rows = rq.n * a.G, row0 = tile * kRows;
    const int32_t *pages = a.table + (int64_t)b * a.width;
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

// Parts of a tile's keys joined: out = sum_j 2^(m_j - M) o_j / sum_j 2^(m_j - M) l_j, M the largest m_j.  A wave has a row.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int tile_rows) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int head = (int)blockIdx.x % a.kv_heads;
    int tile = (int)blockIdx.x / a.kv_heads;
    const int slot_tile = tile;
    int b = -1;
    Request rq{0, 0, 0};
    for (int base = 0; base < a.requests; base += 64) {
        const int i = base + lane;
        const Request r = i < a.requests ? request_at(a, i) : Request{0, 0, 0};
        const int64_t tiles = ((int64_t)r.n * a.G + tile_rows - 1) / tile_rows;
        int64_t upto = tiles;
        for (int d = 1; d < 64; d *= 2) {
            const int64_t u = __shfl_up(upto, d);
            if (lane >= d) upto += u;
        }
        const uint64_t above = __ballot(upto > tile);
        if (above) {
            const int l = __builtin_ctzll(above);
            tile -= (int)__shfl(upto - tiles, l);
            b = base + l;
            rq = Request{__shfl(r.first, l), __shfl(r.n, l), __shfl(r.keys, l)};
            break;
        }
        tile -= (int)__shfl(upto, 63);
    }
    if (b < 0) return;
    const int rows = rq.n * a.G, in_tile = (int)blockIdx.y * 4 + wave, row = tile * tile_rows + in_tile;
    if (row >= rows) return;
    const int64_t slot0 = ((int64_t)slot_tile * a.parts * a.kv_heads + head) * tile_rows + in_tile, step = (int64_t)a.kv_heads * tile_rows;
    float M = kNoKey;
    for (int j = 0; j < a.parts; ++j) M = fmaxf(M, a.ml[slot0 + j * step].x);
    float L = 0.f, acc[D / 64] = {};
    for (int j = 0; j < a.parts; ++j) {
        const float2 ml = a.ml[slot0 + j * step];
        const float w = exp2_fast(ml.x - M);
        L += w * ml.y;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) acc[e] += w * a.part[(slot0 + j * step) * D + lane + 64 * e];
    }
    const int64_t at = ((int64_t)(rq.first + row / a.G) * a.q_heads + head * a.G + row % a.G) * D;
    const float r = L > 0.f ? a.v_scale / L : 0.f;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) a.out[at + lane + 64 * e] = f32_to_bf16(acc[e] * r);
}

}  // namespace

// Tiles that `rows` rows of `requests` requests can make, each of at most max_query.
AttnPlan plan_attn(int64_t rows, int64_t requests, int q_heads, int kv_heads, int64_t max_query) {
    const int64_t G = q_heads / kv_heads;
    AttnPlan p;
    p.tile_rows = kRows;
    const int64_t by_request = requests * ((std::min(max_query, rows) * G + kRows - 1) / kRows), by_row = rows * G / kRows + requests;
    const int64_t tiles = std::min(by_request, by_row);
    p.parts = (int)std::max<int64_t>(1, std::min<int64_t>(32, 512 / std::max<int64_t>(1, tiles * kv_heads)));
    p.items = tiles * p.parts;
    p.split = p.parts > 1;
    return p;
}

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

hipError_t launch_attn_join(const AttnArgs &a, int tile_rows, int D, hipStream_t stream) {
    const dim3 grid((unsigned)(a.items / a.parts * a.kv_heads), (unsigned)(tile_rows / 4));
    if (D == 64) hipLaunchKernelGGL(attn_join_kernel<64>, grid, dim3(256), 0, stream, a, tile_rows);
    else hipLaunchKernelGGL(attn_join_kernel<128>, grid, dim3(256), 0, stream, a, tile_rows);
    return hipGetLastError();
}

}  // namespace dmr
