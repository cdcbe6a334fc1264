// The plan of a dmr_attn_paged call, and the kernel that joins what a split call's workgroups left.
#include "attn.hpp"
#include "glue.hpp"

namespace dmr {

namespace {

// out = sum_j 2^(m_j - M) o_j / sum_j 2^(m_j - M) l_j over a tile's parts, M the largest m_j, in the order of the parts.
//
// FEW, after attn_few, whose tiles are few rows of many parts: a workgroup has a row, each wave every fourth part, a lane D / 64
// elements.  Else, after attn_tiles, the other way round: a wave has a row, and up to 32 parts.  (A workgroup for each row took
// 35 us for the two parts of 1024 rows of 32 heads, a wave 10.)
template <int D, bool FEW>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int tile_rows) {
    constexpr int E = D / 64;
    typedef float __attribute__((ext_vector_type(E))) elements;
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int head = (int)blockIdx.x % a.kv_heads, at = (int)blockIdx.x / a.kv_heads;
    Share sh;
    int in_tile;
    if constexpr (FEW) {
        const int2 split = a.split[at];      // not written for a request without rows
        sh = Share{at, 0, 0, split.y, split.x, request_at(a, at)};
        in_tile = (int)blockIdx.y;
    } else {
        sh = share_of_tile(a, at, tile_rows, lane);
        sh.first_item = at * a.parts;
        in_tile = (int)blockIdx.y * 4 + wave;
    }
    const int row = sh.tile * tile_rows + in_tile;
    if (sh.b < 0 || row >= sh.rq.n * a.G || sh.parts <= 1) return;      // one part: its workgroup has stored the result
    const int64_t slot0 = ((int64_t)sh.first_item * a.kv_heads + head) * tile_rows + in_tile, step = (int64_t)a.kv_heads * tile_rows;
    const int64_t out = ((int64_t)(sh.rq.first + row / a.G) * a.q_heads + head * a.G + row % a.G) * D;
    auto wave_max = [](float v) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
        return v;
    };
    elements acc = {};
    if constexpr (!FEW) {
        const float2 ml = lane < sh.parts ? a.ml[slot0 + lane * step] : make_float2(kNoKey, 0.f);
        const float w = exp2_fast(ml.x - wave_max(ml.x)), L = wave64_sum(w * ml.y);
        const elements *o = reinterpret_cast<const elements *>(a.part + slot0 * D) + lane;
#pragma unroll 4
        for (int j = 0; j < sh.parts; ++j)
            acc += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), j)) * o[j * step * 64];
        acc *= L > 0.f ? a.v_scale / L : 0.f;
        if constexpr (E == 2) reinterpret_cast<uint32_t *>(a.out + out)[lane] = pack_bf16x2(acc[0], acc[1]);
        else a.out[out + lane] = f32_to_bf16(acc[0]);
        return;
    }
    __shared__ float sums[4][D];
    __shared__ float2 mls[4];
    // a wave's parts eight at a time, requested with their references, which they then fade to
    constexpr int AHEAD = 8;
    float m = kNoKey, L = 0.f;
    for (int j0 = wave; j0 < sh.parts; j0 += 4 * AHEAD) {
        float2 ml[AHEAD];
        elements o[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int64_t at_j = slot0 + min(j0 + 4 * i, sh.parts - 1) * step;
            ml[i] = a.ml[at_j];
            o[i] = reinterpret_cast<const elements *>(a.part + at_j * D)[lane];
        }
        float to = m;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) to = fmaxf(to, ml[i].x);
        const float fade = exp2_fast(m - to);
        m = to;
        L *= fade;
        acc *= fade;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float w = j0 + 4 * i < sh.parts ? exp2_fast(ml[i].x - m) : 0.f;
            L = fmaf(w, ml[i].y, L);
            acc += w * o[i];
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sums[wave][lane * E + e] = acc[e];
    if (lane == 0) mls[wave] = make_float2(m, L);
    __syncthreads();
    const int d = (int)threadIdx.x;
    if (d >= D / 2) return;
    const float M = fmaxf(fmaxf(mls[0].x, mls[1].x), fmaxf(mls[2].x, mls[3].x));
    float l = 0.f, o[2] = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = exp2_fast(mls[w].x - M);
        l = fmaf(f, mls[w].y, l);
        o[0] = fmaf(f, sums[w][2 * d], o[0]);
        o[1] = fmaf(f, sums[w][2 * d + 1], o[1]);
    }
    const float r = l > 0.f ? a.v_scale / l : 0.f;
    o[0] *= r;
    o[1] *= r;
    reinterpret_cast<uint32_t *>(a.out + out)[d] = pack_bf16x2(o[0], o[1]);
}

}  // namespace

AttnPlan plan_attn(int64_t rows, int64_t requests, int q_heads, int kv_heads, int D, bool e4m3, int64_t max_query, int64_t capacity) {
    const int64_t G = q_heads / kv_heads, most = std::min(max_query, rows) * G;
    AttnPlan p;
    p.few = most <= 32;
    p.max_tiles = 1;
    if (p.few) {
        p.tile_rows = most <= 16 ? 16 : 32;
        // Parts: about what the chip holds at once of these workgroups, two (e4m3; one with D = 128 and 32 rows, whose parts come in two
        // rounds) to four (bf16, whose waves hold less) a CU.  Between
        // half and twice that a decode step of the 7B-class decoder varies by 10 %.  us with 512 / 1024 in all: 1 x 32768 keys 27.8 /
        // 29.4 (e4m3 19.1 / 22.7), 16 x 300..9000 62.2 / 58.6 (38.9 / 36.7), 32 x 1003 27.5 / 28.3 (18.6 / 21.6).  A large ragged
        // batch gets finer parts, so that the last ones to start end soon: 96 x 1..8100 287 us with 96 to a head, 268 with 256.
        const int64_t wanted = (e4m3 ? 512 : 1024) / kv_heads;
        // no split, and no second launch, where the table is short (one request of 256 keys 4.8 us against 7.3; of 1003 13.1 against
        // 8.1, as one CU reads 40 bytes a ns at most) or the requests fill the chip several times over, where a workgroup's sums over
        // all their lengths, and the join, cost more than an even end gains: us unsplit / split, 256 requests of 8 key heads with 300 keys
        // each 62 / 79 (e4m3 40 / 70), 1000 193 / 203 (106 / 129), 1 .. 2000 222 / 211 (107 / 149); 512 with 1000 355 / 390 (202 / 289);
        // 2048 of one head with 1000 169 / 293 (100 / 274).  The price is a batch with a history many times the others', which one
        // workgroup to a head then reads alone: 256 with 500 keys and one of 32768 499 / 148 (291 / 115), 1 .. 1000 and two
        // of 131071 1744 / 290 (1067 / 188); 600 of one head, the same two, 1616 / 78 (1013 / 64).
        p.split = capacity > 256 && requests <= 512 && requests * kv_heads < 2048;
        p.parts = p.split ? (int)std::max<int64_t>(1, std::max(wanted, 2 * requests)) : 0;
        p.items = requests + p.parts;
        return p;
    }
    p.tile_rows = 128;
    // tiles that so many rows of so many requests can make
    p.max_tiles = (int)((most + p.tile_rows - 1) / p.tile_rows);
    const int64_t tiles = std::min(requests * p.max_tiles, rows * G / p.tile_rows + requests);
    // Parts: the least estimated time, in ns, among those that two workgroups a CU can serve at once.  A workgroup alone on its CU takes
    // 17 ns for a key of its tile, two take 29 (D = 64: 0.6 of that); joining costs a launch and the partial results' way to memory and
    // back.  us with 1 part / as many as 256 / 512 workgroups: 64 rows over 2000 keys 39 / 19 / 26, 300 over 8000 137 / 63 / 61, 512
    // over 32768 543 / 311 / 272, 1024 over 1024 25 / 25 / 35, over 16000 288 / 293 / 258, 8 x 12 over 4000 72 / 31 / 43.  The capacity
    // stands for the longest request: with a table of 131072 tokens instead of one as long as that, 64 over 2000 26 instead of 16, 1024
    // over 1024 36 instead of 25, 300 over 8000 59 instead of 67, 8192 over 8192 level.
    const int64_t wgs = std::max<int64_t>(1, tiles * kv_heads), most_parts = std::max<int64_t>(1, std::min<int64_t>(32, 2 * kCus / wgs));
    auto estimate = [&](int64_t parts) {
        const double key = (D == 64 ? 0.6 : 1.0) * (wgs * parts <= kCus ? 17.0 : 29.0);
        return (double)capacity / (double)parts * key +
               (parts > 1 ? 4000.0 + (double)parts * (double)rows * q_heads * D * 8.0 / 4000.0 : 0.0);
    };
    p.parts = (int)most_parts;
    if (capacity < INT64_MAX)
        for (int64_t n = most_parts - 1; n > 0; --n)
            if (estimate(n) <= estimate(p.parts)) p.parts = (int)n;
    p.items = tiles * p.parts;
    p.split = p.parts > 1;
    return p;
}

hipError_t launch_attn_join(const AttnArgs &a, const AttnPlan &p, int rows, int D, hipStream_t stream) {
    const int64_t tiles = p.few ? a.requests : a.items / p.parts;
    const dim3 grid((unsigned)(tiles * a.kv_heads), (unsigned)(p.few ? std::min(rows, p.tile_rows) : (std::min(rows, p.tile_rows) + 3) / 4));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, p.tile_rows); };
    if (p.few) {
        if (D == 64) go(attn_join_kernel<64, true>); else go(attn_join_kernel<128, true>);
    } else {
        if (D == 64) go(attn_join_kernel<64, false>); else go(attn_join_kernel<128, false>);
    }
    return hipGetLastError();
}

}  // namespace dmr
