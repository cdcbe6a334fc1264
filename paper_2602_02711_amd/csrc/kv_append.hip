// dmr_kv_append: the qkv projection's output to queries, and to keys and values in the paged cache.
//
// One thread holds 8 consecutive elements of a head (16 bytes), so D / 8 lanes hold a head and a norm is a sum over a DPP row or
// half of one.  The partner of an element under DMR_ROPE_HALVES lies D / 16 lanes away, two DPP moves at most.  The turn of pair i is
// formed as position * inv_freq[i] / 2 pi in 64 bits and reduced there to within half a turn, which the hardware's sine and cosine (they
// take turns) then get in 32 bits: an angle of 10^6 rad is as good as a small one.
// Bound by memory: every byte of d_qkv is read once and every result written once.
#include "attn.hpp"
#include "glue.hpp"

namespace dmr {

namespace {

struct AppendArgs {
    const uint16_t *qkv, *gamma_q, *gamma_k;
    const float *inv_freq;
    const int32_t *positions, *slots;
    uint16_t *q;
    uint8_t *k, *v;
    int64_t cache_slots;
    int32_t q_heads, kv_heads, page_shift;
    float eps;
    struct Scale {
        float step, inv;      // of an e4m3 cache, and its reciprocal
    } k_scale, v_scale;
};

// Sum over aligned groups of 16 (8) lanes, in every lane of the group.
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
    if constexpr (LANES == 16) return row16_sum(v);
    v += dpp_move<0xB1>(v);      // quad_perm 1 0 3 2
    v += dpp_move<0x4E>(v);      // quad_perm 2 3 0 1
    return v + dpp_move<0x141>(v);   // row_half_mirror: the other quad of the eight
}
// The value of the lane LANES / 2 away within the group.
template <int LANES>
__device__ __forceinline__ float other_half(float v) {
    if constexpr (LANES == 16) return dpp_move<0x128>(v);    // row_ror 8
    return dpp_move<0x141>(dpp_move<0x1B>(v));               // lane j ^ 3, then 7 - j: j ^ 4
}

// Cosine and sine of the pairs that a lane holds: its 8 elements of one half, or 4 adjacent pairs.
template <int D, bool ADJACENT>
struct Turn {
    static constexpr int PAIRS = ADJACENT ? 4 : 8;
    float cs[PAIRS], sn[PAIRS];
    __device__ __forceinline__ void at(const AppendArgs &a, int64_t t, int lane) {
        if (!a.inv_freq) return;
        const double pos = (double)a.positions[t];
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) {
            const int pair = ADJACENT ? 4 * lane + e : (8 * lane + e) & (D / 2 - 1);
            const double turns = pos * ((double)a.inv_freq[pair] * 0.15915494309189533577);
            const float f = (float)(turns - __builtin_rint(turns));
            cs[e] = __builtin_amdgcn_cosf(f);
            sn[e] = __builtin_amdgcn_sinf(f);
        }
    }
};

// mean(x^2) + eps of the head whose elements the group's lanes hold, eight each; x may come back times a power of two, and the result then
// is of those.  A square below 2^-100 has lost bits of its terms and one above 2^100 may have overflowed: there the elements are brought
// to where neither happens (the smallest, 2^-133, to 2^-33; the largest, below 2^128, to 2^58) and summed again.
template <int LANES>
__device__ __forceinline__ float head_square(const uint4 &raw, float eps, float (&x)[8]) {
    constexpr float kPer = 1.0f / (8 * LANES);
    float square = fmaf(head_sum<LANES>(sumsq_piece(raw)), kPer, eps);
    if (!(square >= 0x1p-100f && square <= 0x1p100f)) {      // or no number; lanes of a head come here together
        const float by = square > 1.f ? 0x1p-70f : 0x1p100f;
        float own = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] *= by;
            own = fmaf(x[e], x[e], own);
        }
        square = fmaf(head_sum<LANES>(own), kPer, eps * by * by);
    }
    return square;
}

// A lane's 8 elements of query or key head h, normed and turned.  A head of zeros stays zeros, one with a NaN is NaN throughout.
template <int D, bool ADJACENT>
__device__ __forceinline__ void norm_and_turn(const AppendArgs &a, const uint4 &raw, int h, int lane, const Turn<D, ADJACENT> &turn, float (&x)[8]) {
    constexpr int LANES = D / 8;
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        x[2 * p] = __uint_as_float(w[p] << 16);
        x[2 * p + 1] = __uint_as_float(w[p] & 0xFFFF0000u);
    }
    const uint16_t *gamma = h < a.q_heads ? a.gamma_q : a.gamma_k;
    if (gamma) {
        const float square = head_square<LANES>(raw, a.eps, x), scale = square == 0.f ? 0.f : __builtin_amdgcn_rsqf(square);
        const uint4 g = reinterpret_cast<const uint4 *>(gamma)[lane];
        const uint32_t gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            x[2 * p] = (x[2 * p] * scale) * __uint_as_float(gw[p] << 16);
            x[2 * p + 1] = (x[2 * p + 1] * scale) * __uint_as_float(gw[p] & 0xFFFF0000u);
        }
    }
    if (!a.inv_freq) return;
    if constexpr (ADJACENT) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = x[2 * e], v = x[2 * e + 1];
            x[2 * e] = u * turn.cs[e] - v * turn.sn[e];
            x[2 * e + 1] = v * turn.cs[e] + u * turn.sn[e];
        }
    } else {
        const bool upper = lane >= LANES / 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float o = other_half<LANES>(x[e]);
            x[e] = x[e] * turn.cs[e] + (upper ? o : -o) * turn.sn[e];
        }
    }
}

__device__ __forceinline__ uint4 as_bf16(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
// Four values over the scale to e4m3, to nearest even, past the range to the largest; NaN stays NaN.  The quotient is that of an fp32
// division: the product with the reciprocal may lie a step or two beside it, and a tie of e4m3 would then go the other way (2 of 1000 values
// over 7 / 256), so what the product leaves of the value, exact in one FMA, is divided and added.  (8192 rows of the 7B-class decoder 41.0 ->
// 41.9 us, 2048 14.2 -> 14.7, few rows level.)  The first bound keeps an infinity from leaving no number and may lose a NaN (a median of three
// does), which the remainder brings back; the second must not.
__device__ __forceinline__ uint32_t as_e4m3(float a, float b, float c, float d, const AppendArgs::Scale &s) {
    auto over = [&](float v) {
        const float q = __builtin_amdgcn_fmed3f(v * s.inv, -448.f, 448.f), exact = fmaf(fmaf(-q, s.step, v), s.inv, q);
        return __builtin_elementwise_maximum(__builtin_elementwise_minimum(exact, 448.f), -448.f);
    };
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(over(a), over(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(over(c), over(d), lo, true);
}
__device__ __forceinline__ float bf16_at(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// Where the cache has slot `slot` of head kvh: block of 16 tokens, token in the block.
struct Place {
    int64_t block;
    int tok;
};
__device__ __forceinline__ Place place_of(const AppendArgs &a, int64_t slot, int kvh) {
    const int per_page = a.page_shift - 4, in_page = (int)slot & ((1 << a.page_shift) - 1);
    return Place{((((slot >> a.page_shift) * a.kv_heads + kvh) << per_page) + (in_page >> 4)), in_page & 15};
}

// A lane's 8 elements of a key to their piece.
template <int D, bool E4M3>
__device__ __forceinline__ void store_key(const AppendArgs &a, const Place &at, int lane, const float (&x)[8]) {
    if constexpr (E4M3)
        *reinterpret_cast<uint2 *>(a.k + at.block * (16 * D) + (lane >> 1) * 256 + at.tok * 16 + (lane & 1) * 8) =
            make_uint2(as_e4m3(x[0], x[1], x[2], x[3], a.k_scale), as_e4m3(x[4], x[5], x[6], x[7], a.k_scale));
    else
        *reinterpret_cast<uint4 *>(a.k + at.block * (32 * D) + lane * 256 + at.tok * 16) = as_bf16(x);
}

// Element d of a value to its place in the piece of its 8 or 16 tokens.
template <int D, bool E4M3>
__device__ __forceinline__ void store_value(const AppendArgs &a, const Place &at, int d, uint16_t v) {
    if constexpr (E4M3)
        a.v[at.block * (16 * D) + d * 16 + at.tok] = (uint8_t)as_e4m3(bf16_at(v), 0.f, 0.f, 0.f, a.v_scale);
    else
        reinterpret_cast<uint16_t *>(a.v)[at.block * (16 * D) + (at.tok >> 3) * (D * 8) + d * 8 + (at.tok & 7)] = v;
}

// Rows, as the 7B-class decoder has it (32 + 8 heads of 128; us by rows / by tiles): 512 8.1 / 8.5 (e4m3 7.7 / 10.6), 640 9.3 / 8.7 (9.2 / 10.7), 768
// 12.8 / 9.3 (11.5 / 11.2).  Wider layouts cross earlier (64 + 8 of 128: 430 rows, e4m3 600), narrower ones later: 768 rows of 28 + 4 of 128 7.4 / 8.5
// (7.6 / 10.6), of 8 + 2 4.8 / 7.5 (4.3 / 9.6), of 16 + 8 of 64 6.3 / 5.6 (5.2 / 7.3), of 4 + 1 of 64 3.1 / 5.1 (3.4 / 6.9).
constexpr int kTilesFrom = 640;

// Few rows: a workgroup has 256 / (D / 8) heads of one row.
template <int D, bool E4M3, bool ADJACENT>
__global__ __launch_bounds__(256) void append_rows_kernel(AppendArgs a) {
    constexpr int LANES = D / 8, SLOTS = 256 / LANES;
    const int lane = (int)threadIdx.x % LANES, h = (int)blockIdx.y * SLOTS + (int)threadIdx.x / LANES;
    const int64_t t = blockIdx.x;
    const int heads = a.q_heads + 2 * a.kv_heads, rotated = a.q_heads + a.kv_heads;
    if (h >= heads) return;      // lanes of a head leave together
    const uint4 raw = reinterpret_cast<const uint4 *>(a.qkv)[(t * heads + h) * LANES + lane];
    const int64_t slot = a.slots[t];
    const bool kept = slot >= 0 && slot < a.cache_slots;
    if (h >= rotated) {
        if (!kept) return;
        const Place at = place_of(a, slot, h - rotated);
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) store_value<D, E4M3>(a, at, 8 * lane + e, (uint16_t)(w[e >> 1] >> (16 * (e & 1))));
        return;
    }
    Turn<D, ADJACENT> turn;
    turn.at(a, t, lane);
    float x[8];
    norm_and_turn<D, ADJACENT>(a, raw, h, lane, turn, x);
    if (h < a.q_heads) reinterpret_cast<uint4 *>(a.q)[(t * a.q_heads + h) * LANES + lane] = as_bf16(x);
    else if (kept) store_key<D, E4M3>(a, place_of(a, slot, h - a.q_heads), lane, x);
}

// Many rows.  A workgroup has TOKENS rows of up to 4 query or key heads, whose angles it forms once and whose loads are all in flight
// together; or 64 rows of one value head, which it turns in LDS: tokens that fill a piece of the cache leave as one store
// of 16 bytes, the others, at the ends of a run of slots, element by element.  (With a thread's 8 elements of one token stored
// one by one a wave's store fell into 64 lines: 8192 rows 77 us.)  The projection is read, and queries are written, past the caches:
// 53 -> 41 us for 8192 rows of the 7B-class decoder, 4.9 .. 5.0 TB/s, where a copy of as many bytes takes 39 (into e4m3 42 us, 4.4 TB/s).
constexpr int kHeadsAtOnce = 4, kValueRows = 64;
template <int D, bool E4M3, bool ADJACENT>
__global__ __launch_bounds__(256) void append_tiles_kernel(AppendArgs a, int rows, int chunks) {
    constexpr int LANES = D / 8, TOKENS = 256 / LANES, RUN = E4M3 ? 16 : 8;
    __shared__ __align__(16) uint16_t tile_of[kValueRows][D + 8];
    __shared__ int slot_of[kValueRows];
    __shared__ uint8_t lead[kValueRows], alone[kValueRows];
    const int tid = (int)threadIdx.x, heads = a.q_heads + 2 * a.kv_heads, rotated = a.q_heads + a.kv_heads;
    const int works = chunks * (kValueRows / TOKENS) + a.kv_heads;      // of a tile of kValueRows rows
    const int tile = (int)blockIdx.x / works, work = (int)blockIdx.x % works;
    if (work >= a.kv_heads) {
        const int lane = tid % LANES, sub = (work - a.kv_heads) / chunks, first = (work - a.kv_heads) % chunks * kHeadsAtOnce;
        const int64_t t = (int64_t)tile * kValueRows + sub * TOKENS + tid / LANES;
        if (t >= rows) return;
        const int n = min(kHeadsAtOnce, rotated - first);
        u32x4_t raw[kHeadsAtOnce];
        const u32x4_t *src = reinterpret_cast<const u32x4_t *>(a.qkv) + (t * heads + first) * LANES + lane;
#pragma unroll
        for (int i = 0; i < kHeadsAtOnce; ++i) raw[i] = __builtin_nontemporal_load(src + min(i, n - 1) * LANES);
        const int64_t slot = a.slots[t];
        const bool kept = slot >= 0 && slot < a.cache_slots;
        Turn<D, ADJACENT> turn;
        turn.at(a, t, lane);
#pragma unroll
        for (int i = 0; i < kHeadsAtOnce; ++i) {
            if (i >= n) break;
            const int h = first + i;
            float x[8];
            norm_and_turn<D, ADJACENT>(a, make_uint4(raw[i][0], raw[i][1], raw[i][2], raw[i][3]), h, lane, turn, x);
            if (h < a.q_heads) {
                const uint4 w = as_bf16(x);
                __builtin_nontemporal_store(u32x4_t{w.x, w.y, w.z, w.w}, reinterpret_cast<u32x4_t *>(a.q) + (t * a.q_heads + h) * LANES + lane);
            } else if (kept) {
                store_key<D, E4M3>(a, place_of(a, slot, h - a.q_heads), lane, x);
            }
        }
        return;
    }
    const int kvh = work;
    const int64_t t0 = (int64_t)tile * kValueRows;
    const int here = (int)min((int64_t)kValueRows, rows - t0);
#pragma unroll
    for (int i = 0; i < kValueRows / TOKENS; ++i) {
        const int r = i * TOKENS + tid / LANES, lane = tid % LANES;
        const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(a.qkv) + ((t0 + min(r, here - 1)) * heads + rotated + kvh) * LANES + lane);
        *reinterpret_cast<u32x4_t *>(&tile_of[r][8 * lane]) = v;
    }
    if (tid < kValueRows) {
        const int64_t slot = tid < here ? a.slots[t0 + tid] : -1;
        slot_of[tid] = slot >= 0 && slot < a.cache_slots ? (int)slot : -1;
    }
    __syncthreads();
    if (tid < kValueRows) {      // whether this row begins a whole piece
        bool whole = tid + RUN <= kValueRows && slot_of[tid] >= 0 && slot_of[tid] % RUN == 0;
        for (int i = 1; i < RUN; ++i) whole = whole && slot_of[min(tid + i, kValueRows - 1)] == slot_of[tid] + i;
        lead[tid] = whole;
    }
    __syncthreads();
    if (tid < kValueRows) {
        bool in_piece = false;
        for (int i = 0; i < RUN; ++i) in_piece = in_piece || (tid >= i && lead[tid - i]);
        alone[tid] = slot_of[tid] >= 0 && !in_piece;
    }
    __syncthreads();
    for (int r = tid / D; r < here; r += 256 / D) {
        const int d = tid % D;
        if (lead[r]) {
            const Place at = place_of(a, slot_of[r], kvh);
            if constexpr (E4M3) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = as_e4m3(bf16_at(tile_of[r + 4 * i][d]), bf16_at(tile_of[r + 4 * i + 1][d]), bf16_at(tile_of[r + 4 * i + 2][d]),
                                   bf16_at(tile_of[r + 4 * i + 3][d]), a.v_scale);
                *reinterpret_cast<uint4 *>(a.v + at.block * (16 * D) + d * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = (uint32_t)tile_of[r + 2 * i][d] | ((uint32_t)tile_of[r + 2 * i + 1][d] << 16);
                *reinterpret_cast<uint4 *>(a.v + at.block * (32 * D) + (at.tok >> 3) * (D * 16) + d * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else if (alone[r]) {
            store_value<D, E4M3>(a, place_of(a, slot_of[r], kvh), d, tile_of[r][d]);
        }
    }
}

}  // namespace

hipError_t launch_kv_append(const CacheView &c, const uint16_t *qkv, int64_t rows, int q_heads, const uint16_t *gamma_q,
                            const uint16_t *gamma_k, float eps, const float *inv_freq, bool adjacent, const int32_t *positions,
                            const int32_t *slots, uint16_t *q, hipStream_t stream) {
    const AppendArgs a{qkv, gamma_q, gamma_k, inv_freq, positions, slots, q, c.k, c.v, c.pages << c.page_shift,
                       q_heads, c.kv_heads, c.page_shift, eps, {c.k_scale, 1.0f / c.k_scale}, {c.v_scale, 1.0f / c.v_scale}};
    const int heads = q_heads + 2 * c.kv_heads, tokens = 256 * 8 / c.D;
    auto with = [&](auto d, auto e, auto adj) {
        constexpr int D = decltype(d)::value;
        constexpr bool E = decltype(e)::value, A = decltype(adj)::value;
        if (rows < env_int("DMR_APPEND_TILES", kTilesFrom)) {
            const dim3 grid((unsigned)rows, (unsigned)((heads + tokens - 1) / tokens));
            hipLaunchKernelGGL(HIP_KERNEL_NAME(append_rows_kernel<D, E, A>), grid, dim3(256), 0, stream, a);
        } else {
            const int tiles = (int)((rows + kValueRows - 1) / kValueRows), chunks = (q_heads + c.kv_heads + kHeadsAtOnce - 1) / kHeadsAtOnce;
            const int64_t blocks = (int64_t)tiles * (chunks * (kValueRows / tokens) + c.kv_heads);
            hipLaunchKernelGGL(HIP_KERNEL_NAME(append_tiles_kernel<D, E, A>), dim3((unsigned)blocks), dim3(256), 0, stream, a, (int)rows, chunks);
        }
    };
    auto pairs = [&](auto d, auto e) {
        if (adjacent) with(d, e, std::true_type{}); else with(d, e, std::false_type{});
    };
    auto type = [&](auto d) {
        if (c.e4m3) pairs(d, std::true_type{}); else pairs(d, std::false_type{});
    };
    if (c.D == 64) type(std::integral_constant<int, 64>{}); else type(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace dmr
