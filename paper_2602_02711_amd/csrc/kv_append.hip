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
    int32_t q_heads, kv_heads, page_shift, heads_per_group;
    float eps, inv_k_scale, inv_v_scale;
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

__device__ __forceinline__ float e4m3_range(float x) { return __builtin_amdgcn_fmed3f(x, -448.f, 448.f); }

template <int D, bool E4M3, bool ADJACENT>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    constexpr int LANES = D / 8, SLOTS = 256 / LANES;
    const int lane = (int)threadIdx.x % LANES, head0 = (int)threadIdx.x / LANES;
    const int64_t t = blockIdx.x;
    const int heads = a.q_heads + 2 * a.kv_heads, rotated = a.q_heads + a.kv_heads;
    const int64_t slot = a.slots[t];
    const bool kept = slot >= 0 && slot < a.cache_slots;
    const int per_page = a.page_shift - 4, in_page = (int)slot & ((1 << a.page_shift) - 1);
    const int64_t page = slot >> a.page_shift;
    const int block = in_page >> 4, tok = in_page & 15;
    const int first = (int)blockIdx.y * a.heads_per_group, last = min(first + a.heads_per_group, heads);

    // cosine and sine of this lane's pairs: 8 elements of one half, or 4 adjacent pairs
    constexpr int PAIRS = ADJACENT ? 4 : 8;
    float cs[PAIRS], sn[PAIRS];
    if (a.inv_freq && first < rotated) {
        const double pos = (double)a.positions[t];
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) {
            const int pair = ADJACENT ? 4 * lane + e : (8 * lane + e) & (D / 2 - 1);
            const double turns = pos * ((double)a.inv_freq[pair] * 0.15915494309189533577);
            const float f = (float)(turns - __builtin_rint(turns));
            cs[e] = __builtin_amdgcn_cosf(f);
            sn[e] = __builtin_amdgcn_sinf(f);
        }
    } else {
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) cs[e] = 1.f, sn[e] = 0.f;
    }
    for (int base = first; base < last; base += SLOTS) {
        const int h = base + head0;
        const bool live = h < last;
        // lanes of a head leave together; others' DPP moves stay within their own head
        if (!live) continue;
        const uint4 raw = reinterpret_cast<const uint4 *>(a.qkv)[(t * heads + h) * LANES + lane];
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        float x[8];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            x[2 * p] = __uint_as_float(w[p] << 16);
            x[2 * p + 1] = __uint_as_float(w[p] & 0xFFFF0000u);
        }
        if (h < rotated) {
            const uint16_t *gamma = h < a.q_heads ? a.gamma_q : a.gamma_k;
            if (gamma) {
                const float scale = rms_scale(head_sum<LANES>(sumsq_piece(raw)), 1.0f / D, a.eps);
                const uint4 g = reinterpret_cast<const uint4 *>(gamma)[lane];
                const uint32_t gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    x[2 * p] = (x[2 * p] * scale) * __uint_as_float(gw[p] << 16);
                    x[2 * p + 1] = (x[2 * p + 1] * scale) * __uint_as_float(gw[p] & 0xFFFF0000u);
                }
            }
            if (a.inv_freq) {
                if constexpr (ADJACENT) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float u = x[2 * e], v = x[2 * e + 1];
                        x[2 * e] = u * cs[e] - v * sn[e];
                        x[2 * e + 1] = v * cs[e] + u * sn[e];
                    }
                } else {
                    const bool upper = lane >= LANES / 2;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float o = other_half<LANES>(x[e]);
                        x[e] = x[e] * cs[e] + (upper ? o : -o) * sn[e];
                    }
                }
            }
        }
        if (h < a.q_heads) {
            reinterpret_cast<uint4 *>(a.q)[(t * a.q_heads + h) * LANES + lane] =
                make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
            continue;
        }
        if (!kept) continue;
        const bool key = h < rotated;
        const int kvh = h - (key ? a.q_heads : rotated);
        const int64_t at = ((page * a.kv_heads + kvh) << per_page) + block;
        if constexpr (E4M3) {
            const float inv = key ? a.inv_k_scale : a.inv_v_scale;
            uint32_t c[2];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                int r = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[4 * p] * inv), e4m3_range(x[4 * p + 1] * inv), 0, false);
                c[p] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[4 * p + 2] * inv), e4m3_range(x[4 * p + 3] * inv), r, true);
            }
            if (key) {
                *reinterpret_cast<uint2 *>(a.k + at * (16 * D) + (lane >> 1) * 256 + tok * 16 + (lane & 1) * 8) = make_uint2(c[0], c[1]);
            } else {
                uint8_t *dst = a.v + at * (16 * D) + lane * 128 + tok;
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e * 16] = (uint8_t)(c[e >> 2] >> (8 * (e & 3)));
            }
        } else {
            if (key) {
                *reinterpret_cast<uint4 *>(a.k + at * (32 * D) + lane * 256 + tok * 16) =
                    make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
            } else {
                uint16_t *dst = reinterpret_cast<uint16_t *>(a.v + at * (32 * D)) + (tok >> 3) * (D * 8) + lane * 64 + (tok & 7);
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e * 8] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));    // values go as they came
            }
        }
    }
}

}  // namespace

hipError_t launch_kv_append(const CacheView &c, const uint16_t *qkv, int64_t rows, int q_heads, const uint16_t *gamma_q,
                            const uint16_t *gamma_k, float eps, const float *inv_freq, bool adjacent, const int32_t *positions,
                            const int32_t *slots, uint16_t *q, hipStream_t stream) {
    AppendArgs a{qkv, gamma_q, gamma_k, inv_freq, positions, slots, q, c.k, c.v, c.pages << c.page_shift,
                 q_heads, c.kv_heads, c.page_shift, 0, eps, 1.0f / c.k_scale, 1.0f / c.v_scale};
    const int heads = q_heads + 2 * c.kv_heads, slots_per_group = 256 * 8 / c.D;
    // few rows: a workgroup for every 16 (32) heads; many: one for all of a row's heads, which share its angles
    a.heads_per_group = rows >= 512 ? heads : slots_per_group;
    const dim3 grid((unsigned)rows, (unsigned)((heads + a.heads_per_group - 1) / a.heads_per_group));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
    auto with = [&](auto d, auto e) {
        constexpr int D = decltype(d)::value;
        constexpr bool E = decltype(e)::value;
        if (adjacent) go(append_kernel<D, E, true>); else go(append_kernel<D, E, false>);
    };
    auto type = [&](auto d) {
        if (c.e4m3) with(d, std::true_type{}); else with(d, std::false_type{});
    };
    if (c.D == 64) type(std::integral_constant<int, 64>{}); else type(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace dmr
