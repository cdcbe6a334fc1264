// The attention block's shared declarations: how the paged cache lies in memory, what the kernels are given, and the launchers.
//
// Layout of a pool: [page][kv head][16-token block], a block 16 x D elements in pieces of 16 bytes (pc elements: 8 bf16, 16 e4m3),
// keys [D / pc][16][pc], values [16 / pc][D][pc].  It is the order of MFMA operands: with scores formed as K Q^T and outputs as
// V^T P^T both products take the cache as their A operand, 8 elements along the contraction per lane, so a wave fetches an operand
// as whole pieces that lie side by side, straight into registers, and no transposition is left for the kernels.  The scores come
// out of the first product with a query per lane column and keys along the registers, which is how the second one wants its B
// operand once the keys are taken in the matching order (key_of_row in the kernels): probabilities never leave their lane.
#pragma once
#include <type_traits>

#include "common.hpp"

namespace dmr {

constexpr int kBlockTokens = 16;      // tokens of a cache block

struct AttnArgs {
    const uint16_t *q;
    uint16_t *out;
    const uint8_t *k, *v;
    const int32_t *start, *lens, *table;
    float *part;              // [item][kv head][tile rows][D] unnormalised outputs
    float2 *ml;               // [item][kv head][tile rows]: reference of the exponents (log2 units), sum
    int2 *split;              // attn_few: [request] first item, parts, for attn_join
    int32_t rows, requests, width, q_heads, kv_heads, G, pages, page_shift;
    float scale_log2;         // softmax scale * key scale * log2(e)
    float v_scale;
    int32_t items;            // per kv head, of the grid
    int32_t max_tiles;        // of a request
    int32_t parts;            // attn_tiles: parts of every tile's keys;  attn_few: as share_of_item says, 0: one item per request
};

// A request as its device arrays have it, kept inside the buffers whatever they hold.
struct Request {
    int first, n, keys;       // rows first .. first + n - 1, the last n of `keys` keys
};
__device__ __forceinline__ Request request_at(const AttnArgs &a, int b) {
    Request r;
    r.first = min(max(a.start[b], 0), a.rows);
    r.n = min(max(a.start[b + 1], r.first), a.rows) - r.first;
    r.keys = min(max(a.lens[b], 0), a.width << a.page_shift);
    return r;
}

// Units of UNIT keys in `keys` of them, which may be up to 2^31 - 16: the sum before the division passes 31 bits.
template <int UNIT>
__device__ __forceinline__ int units_in(int keys) { return (int)(((uint32_t)keys + (UNIT - 1)) / UNIT); }

// First byte of a block of 16 tokens of one head: `block` of the request whose row of the table is given.
template <int BLOCK_BYTES>
__device__ __forceinline__ int64_t block_offset(const AttnArgs &a, const int32_t *row, int block, int head) {
    const int per_page = a.page_shift - 4;
    const int page = min(max(row[block >> per_page], 0), a.pages - 1);
    return (((((int64_t)page * a.kv_heads + head) << per_page) + (block & ((1 << per_page) - 1)))) * BLOCK_BYTES;
}

// The same for a block that all lanes ask for: a scalar load where the compiler can tell that they do (attn_tiles), a vector load where it
// cannot (attn_few, whose wave index it takes for a lane's own).
template <int BLOCK_BYTES>
__device__ __forceinline__ int64_t uniform_block_offset(const AttnArgs &a, const int32_t *row, int block, int head) {
    typedef const __attribute__((address_space(4))) int32_t *constant_i32;
    const int per_page = a.page_shift - 4;
    const int page = min(max(((constant_i32)(uintptr_t)row)[block >> per_page], 0), a.pages - 1);
    return (((((int64_t)page * a.kv_heads + head) << per_page) + (block & ((1 << per_page) - 1)))) * BLOCK_BYTES;
}

// Inclusive scan over the wave's lanes under `op`, whose neutral element is 0.
template <typename Op>
__device__ __forceinline__ uint32_t wave_scan(uint32_t v, Op op) {
    auto from = [](uint32_t u, auto ctrl, auto rows) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    };
    typedef std::integral_constant<int, 0xF> all;
    v = op(v, from(v, std::integral_constant<int, 0x111>{}, all{}));      // row_shr 1, 2, 4, 8: within rows of 16
    v = op(v, from(v, std::integral_constant<int, 0x112>{}, all{}));
    v = op(v, from(v, std::integral_constant<int, 0x114>{}, all{}));
    v = op(v, from(v, std::integral_constant<int, 0x118>{}, all{}));
    v = op(v, from(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{}));      // row_bcast 15: rows 1 and 3
    v = op(v, from(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{}));      // row_bcast 31: rows 2 and 3
    return v;
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    return wave_scan(v, [](uint32_t a, uint32_t b) { return a + b; });
}
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }

// What an item of a split call does: part `part` of `parts` of the keys of rows tile `tile` of request b; its partial result, and
// those of the tile's other parts, are at items first_item .. first_item + parts - 1.  b < 0: nothing.
struct Share {
    int b, tile, part, parts, first_item;
    Request rq;
};

// Item -> tile where every tile has a.parts parts: request b has ceil(n G / tile_rows) tiles, and no more than max_query asks for, so
// that one with more rows takes no other's.
__device__ __forceinline__ Share share_of_tile(const AttnArgs &a, int tile, int tile_rows, int lane) {
    for (int base = 0; base < a.requests; base += 64) {
        const int i = base + lane;
        const Request r = i < a.requests ? request_at(a, i) : Request{0, 0, 0};
        const uint32_t tiles = (uint32_t)min((int)(((int64_t)r.n * a.G + tile_rows - 1) / tile_rows), a.max_tiles), upto = wave_scan(tiles);
        const uint64_t above = __ballot((int)upto > tile);
        if (above) {
            const int l = __builtin_ctzll(above);
            return Share{base + l, tile - (int)lane_value(upto - tiles, l), 0, a.parts, 0,
                         Request{(int)lane_value(r.first, l), (int)lane_value(r.n, l), (int)lane_value(r.keys, l)}};
        }
        tile -= (int)lane_value(upto, 63);
    }
    return Share{-1, 0, 0, 0, 0, Request{0, 0, 0}};
}

// One tile per request, its keys in as many parts as its length asks for.  With U units of UNIT keys in the whole batch and
// C = max(kMinUnits, ceil(U / a.parts)), a request of u units has ceil(u / C) parts, one at least: no more than a.parts + requests
// items, whatever the lengths.  A batch that gives every CU a workgroup and whose longest request is no longer than 3 / 2 of the mean
// is not split.  Each workgroup forms the same sums from the lengths on the device, so that a captured call splits the lengths
// of its replay.  (Whether a call is split at all, plan_attn decides from the batch's size.)
constexpr int kMinUnits = 4;      // a unit for each wave of a workgroup
template <int UNIT>
__device__ __forceinline__ Share share_of_item(const AttnArgs &a, int item, int lane) {
    uint64_t total = 0;
    uint32_t longest = 0, some = 0;
    // (64 requests of 2^31 keys each would have 2^32 units: one less for such a request keeps a round's sum in 32 bits)
    auto units_of = [](const Request &r) { return r.n > 0 ? std::min((uint32_t)units_in<UNIT>(r.keys), (1u << 26) - 1) : 0u; };
    auto request_of = [&](int i) { return i < a.requests ? request_at(a, i) : Request{0, 0, 0}; };
    Request r;      // of this lane, in the round at hand: up to 64 requests are read once
    for (int base = 0; base < a.requests; base += 64) {
        r = request_of(base + lane);
        const uint32_t u = units_of(r);
        total += lane_value(wave_scan(u), 63);
        longest = std::max(longest, lane_value(wave_scan(u, [](uint32_t x, uint32_t y) { return std::max(x, y); }), 63));
        some += (uint32_t)__popcll(__ballot(r.n > 0));
    }
    const uint32_t parts = (uint32_t)a.parts;
    const uint32_t even = total >> 31 ? (uint32_t)((total + parts - 1) / parts) : ((uint32_t)total + parts - 1) / parts;
    uint32_t C = std::max((uint32_t)kMinUnits, even);
    if (some * (uint32_t)a.kv_heads >= (uint32_t)kCus && (uint64_t)longest * some * 2 <= total * 3) C = std::max(C, longest);
    int before = 0;
    for (int base = 0; base < a.requests; base += 64) {
        if (a.requests > 64) r = request_of(base + lane);
        const uint32_t items = r.n > 0 ? std::max(1u, (units_of(r) + C - 1) / C) : 0u, upto = wave_scan(items);
        const uint64_t above = __ballot(before + (int)upto > item);
        if (above) {
            const int l = __builtin_ctzll(above), first = before + (int)lane_value(upto - items, l);
            return Share{base + l, 0, item - first, (int)lane_value(items, l), first,
                         Request{(int)lane_value(r.first, l), (int)lane_value(r.n, l), (int)lane_value(r.keys, l)}};
        }
        before += (int)lane_value(upto, 63);
    }
    return Share{-1, 0, 0, 0, 0, Request{0, 0, 0}};
}

// Eight e4m3 bytes to eight bf16 (exact).
__device__ __forceinline__ uint4 bf16_of_e4m3(uint32_t lo, uint32_t hi) {
    auto pair = [](uint32_t w, auto upper) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, decltype(upper)::value));
    };
    return make_uint4(pair(lo, std::false_type{}), pair(lo, std::true_type{}), pair(hi, std::false_type{}), pair(hi, std::true_type{}));
}

// 2^x, x <= 0 or -inf.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kNoKey = -3.0e38f;    // "largest score" of a row that has seen no key: finite, so that differences stay numbers

struct CacheView {
    uint8_t *k, *v;
    int64_t pages;
    int32_t page_shift, kv_heads, D;
    bool e4m3;
    float k_scale, v_scale;
};

hipError_t launch_kv_assign(int64_t requests, int64_t rows, int64_t width, int page_shift, int64_t capacity, const int32_t *new_tokens,
                            const int32_t *lens, const int32_t *free_pages, const int32_t *free_count, int32_t *table,
                            int32_t *start, int32_t *kv_lens, int32_t *positions, int32_t *slots, int32_t *left, hipStream_t stream);
hipError_t launch_kv_append(const CacheView &c, const uint16_t *qkv, int64_t rows, int q_heads, const uint16_t *gamma_q,
                            const uint16_t *gamma_k, float eps, const float *inv_freq, bool adjacent, const int32_t *positions,
                            const int32_t *slots, uint16_t *q, hipStream_t stream);

// How a call of dmr_attn_paged is split, from what the host knows: pure arithmetic, the same for the workspace query and the launch.
struct AttnPlan {
    bool few;                 // attn_few: one tile of 16 or 32 rows per request
    int tile_rows;            // (token, query head) rows of a tile
    int64_t items;            // workgroups per kv head
    int parts, max_tiles;     // AttnArgs
    bool split;               // several items may belong to one tile: partial results, joined by a second kernel
};
constexpr int few_unit(bool e4m3) { return e4m3 ? 64 : 32; }      // keys that a wave of attn_few takes at a time
// `capacity`: tokens that a row of the block table can name; INT64_MAX gives a plan with no fewer items than any capacity's.
AttnPlan plan_attn(int64_t rows, int64_t requests, int q_heads, int kv_heads, int D, bool e4m3, int64_t max_query, int64_t capacity);
hipError_t launch_attn_tiles(const AttnArgs &a, int D, bool e4m3, hipStream_t stream);
hipError_t launch_attn_few(const AttnArgs &a, const AttnPlan &p, int D, bool e4m3, hipStream_t stream);
// Joins the parts that a split call left; `rows` of a tile at most.
hipError_t launch_attn_join(const AttnArgs &a, const AttnPlan &p, int rows, int D, hipStream_t stream);

}  // namespace dmr
