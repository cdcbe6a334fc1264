// The plan of a dmr_attn_paged call, and the kernel that joins what a split call's workgroups left.
#include "attn.hpp"
#include "glue.hpp"

namespace dmr {

namespace {

// out = sum_j 2^(m_j - M) o_j / sum_j 2^(m_j - M) l_j over a tile's parts, M the largest m_j, in the order of the parts.  A workgroup has
// a row: each wave takes every fourth part, a lane D / 64 elements.  UNIT: that of the attn_few kernel that split, 0: attn_tiles.
template <int D, int UNIT>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int tile_rows) {
    constexpr int E = D / 64;
    __shared__ float sums[4][D + 1];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, in_tile = (int)blockIdx.y;
    const int head = (int)blockIdx.x % a.kv_heads, at = (int)blockIdx.x / a.kv_heads;
    Share sh;
    if constexpr (UNIT > 0) {
        sh = share_of_item<UNIT, true>(a, at, lane);
    } else {
        sh = share_of_tile(a, at, tile_rows, lane);
        sh.first_item = at * a.parts;
    }
    const int row = sh.tile * tile_rows + in_tile;
    if (sh.b < 0 || row >= sh.rq.n * a.G || sh.parts <= 1) return;      // one part: its workgroup has stored the result
    const int64_t slot0 = ((int64_t)sh.first_item * a.kv_heads + head) * tile_rows + in_tile, step = (int64_t)a.kv_heads * tile_rows;
    float M = kNoKey;
    for (int j = lane; j < sh.parts; j += 64) M = fmaxf(M, a.ml[slot0 + j * step].x);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
    float L = 0.f, acc[E] = {};
#pragma unroll 4
    for (int j = wave; j < sh.parts; j += 4) {
        const float2 ml = a.ml[slot0 + j * step];
        const float *o = a.part + (slot0 + j * step) * D + lane * E;
        const float w = exp2_fast(ml.x - M);
        L = fmaf(w, ml.y, L);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(w, o[e], acc[e]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sums[wave][lane * E + e] = acc[e];
    if (lane == 0) sums[wave][D] = L;
    __syncthreads();
    const int d = (int)threadIdx.x;
    if (d >= D / 2) return;
    const float l = (sums[0][D] + sums[1][D]) + (sums[2][D] + sums[3][D]);
    const float r = l > 0.f ? a.v_scale / l : 0.f;
    float o[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) o[e] = ((sums[0][2 * d + e] + sums[1][2 * d + e]) + (sums[2][2 * d + e] + sums[3][2 * d + e])) * r;
    const int64_t out = ((int64_t)(sh.rq.first + row / a.G) * a.q_heads + head * a.G + row % a.G) * D;
    reinterpret_cast<uint32_t *>(a.out + out)[d] = pack_bf16x2(o[0], o[1]);
}

}  // namespace

AttnPlan plan_attn(int64_t rows, int64_t requests, int q_heads, int kv_heads, int64_t max_query, int64_t capacity, bool e4m3) {
    const int64_t G = q_heads / kv_heads, most = std::min(max_query, rows) * G;
    AttnPlan p;
    p.few = most <= 32;
    if (p.few) {
        p.tile_rows = most <= 16 ? 16 : 32;
        // Parts: about what the chip holds at once of these workgroups, two (e4m3) to four (bf16, whose waves hold less) a CU.  Between
        // half and twice that a decode step of the 7B-class decoder varies by 10 %.  us with 512 / 1024 in all: 1 x 32768 keys 27.8 /
        // 29.4 (e4m3 19.1 / 22.7), 16 x 300..9000 62.2 / 58.6 (38.9 / 36.7), 32 x 1003 27.5 / 28.3 (18.6 / 21.6).  A large ragged
        // batch gets finer parts, so that the last ones to start end soon: 96 x 1..8100 287 us with 96 to a head, 268 with 256.
        const int64_t wanted = (e4m3 ? 512 : 1024) / kv_heads;
        // no split, and no second launch, where the table is short (one request of 256 keys 4.8 us against 7.3; of 1003 13.1 against
        // 8.1, as one CU reads 40 bytes a ns at most) or the requests fill the chip many times over
        p.split = requests * kv_heads < 8192 && capacity > 256;
        p.parts = p.split ? (int)std::max<int64_t>(1, std::max(wanted, 2 * requests)) : 0;
        p.items = requests + p.parts;
        return p;
    }
    p.tile_rows = 128;
    // tiles that so many rows of so many requests can make
    const int64_t tiles = std::min(requests * ((most + p.tile_rows - 1) / p.tile_rows), rows * G / p.tile_rows + requests);
    p.parts = (int)std::max<int64_t>(1, std::min<int64_t>(32, env_int("DMR_ATTN_PARTS", 512) / std::max<int64_t>(1, tiles * kv_heads)));
    p.items = tiles * p.parts;
    p.split = p.parts > 1;
    return p;
}

hipError_t launch_attn_join(const AttnArgs &a, const AttnPlan &p, int rows, int D, bool e4m3, hipStream_t stream) {
    const int64_t tiles = p.few ? a.requests : a.items / p.parts;
    const dim3 grid((unsigned)(tiles * a.kv_heads), (unsigned)std::min(rows, p.tile_rows));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, p.tile_rows); };
    auto split_by = [&](auto unit) {
        constexpr int U = decltype(unit)::value;
        if (D == 64) go(attn_join_kernel<64, U>); else go(attn_join_kernel<128, U>);
    };
    if (!p.few) split_by(std::integral_constant<int, 0>{});
    else if (e4m3) split_by(std::integral_constant<int, few_unit(true)>{});
    else split_by(std::integral_constant<int, few_unit(false)>{});
    return hipGetLastError();
}

}  // namespace dmr
