// dmr_kv_assign: pages, positions and slots of a step from the requests' lengths.
//
// With need_b the pages that request b lacks and upto_b their running sum, the j-th new page of b is the page
// free - 1 - (upto_b - need_b + j) of the stack: two prefix sums (rows, then needs, since what a request needs counts only if its
// rows fit) and independent look-ups.  The work is a few KB whatever the batch, so a call is bound by its launch and by the chain of
// dependent reads lengths -> pages -> slots.  Up to 1024 requests it is one launch: every workgroup forms the sums, the first one
// writes the requests' results, and each has 2048 rows, whose slots it takes from the old entries of the table or straight from
// the stack.  A step that updates its lengths in place has one workgroup up to 4096 rows; beyond that, and beyond 1024 requests, a second
// kernel has the rows (200 requests, 16100 rows: 10.4 us a call in two launches, 7.4 in one).
#include "attn.hpp"

namespace dmr {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kRowsAlone = 4096, kRowsEach = 2048;
constexpr int32_t kRefused = INT32_MIN;

// Inclusive sum over the workgroup on top of `carry`, which moves on to the total.  A wave's own sum fits 32 bits.
__device__ __forceinline__ int64_t block_scan(uint32_t v, int64_t &carry, uint32_t *sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t in_wave = wave_scan(v);
    __syncthreads();                       // `sums` of the scan before
    if (lane == 63) sums[wave] = in_wave;
    __syncthreads();
    int64_t before = carry;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += sums[w];
        carry += sums[w];
    }
    return before + in_wave;
}

// First index in [lo, hi) whose value is above t; hi if none.
template <typename V>
__device__ __forceinline__ int first_above(const V *v, int lo, int hi, int64_t t) {
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((int64_t)v[mid] > t) hi = mid; else lo = mid + 1;
    }
    return lo;
}

__global__ __launch_bounds__(kThreads) void assign_kernel(int requests, int rows, int64_t width, int page_shift, int64_t capacity,
                                                          const int32_t *new_tokens, const int32_t *lens, const int32_t *free_pages,
                                                          const int32_t *free_count, int32_t *table, int32_t *start,
                                                          int32_t *kv_lens, int32_t *positions, int32_t *slots, int32_t *left,
                                                          int rows_each) {
    __shared__ uint32_t sums[kWaves];
    __shared__ uint32_t upto[kThreads];        // new pages of this round's requests, running sum over those that got theirs
    __shared__ int32_t first_col[kThreads];    // column of a request's first new page
    __shared__ int32_t end_row[kThreads], row_to_pos[kThreads];
    __shared__ int refused_sum;
    const int tid = (int)threadIdx.x;
    const bool writes = blockIdx.x == 0;
    const int64_t free = min(max((int64_t)*free_count, (int64_t)0), capacity);
    const int round = (1 << page_shift) - 1;
    int64_t rows_sum = 0, need_sum = 0, taken = 0;
    if (tid == 0) {
        refused_sum = 0;
        if (requests == 0 && writes) start[0] = 0;
    }
    int refused = 0;
    for (int base = 0; base < requests; base += kThreads) {
        const int b = base + tid;
        const bool live = b < requests;
        const int64_t len = live ? (int64_t)lens[b] : 0, old = len < 0 ? -1 - len : len;
        // a count past `rows` is refused whatever it is: rows + 1 keeps the sums short
        const int64_t more = live ? min(max((int64_t)new_tokens[b], (int64_t)0), (int64_t)rows + 1) : 0;
        const int64_t end = block_scan((uint32_t)more, rows_sum, sums);
        const int64_t first = (old + round) >> page_shift, last = (old + more + round) >> page_shift;
        const bool fits = last <= width && end <= rows;
        const uint32_t need = live && fits ? (uint32_t)(last - first) : 0u;
        const int64_t mine = block_scan(need, need_sum, sums);
        const bool good = fits && (need == 0 || mine <= free);
        // requests that get pages come before all that are refused for want of them, so their needs add up to `mine` themselves
        const uint32_t got = good ? need : 0u;
        const int64_t taken_before = taken;
        const int64_t got_upto = block_scan(got, taken, sums);
        upto[tid] = (uint32_t)(got_upto - taken_before);
        first_col[tid] = (int32_t)min(first, width);
        end_row[tid] = (int32_t)min(end, (int64_t)rows);
        row_to_pos[tid] = good ? (int32_t)(old - (end - more)) : kRefused;
        if (live && writes) {
            start[b] = (int32_t)min(end - more, (int64_t)rows);
            if (b == requests - 1) start[requests] = (int32_t)min(end, (int64_t)rows);
            kv_lens[b] = (int32_t)(good ? old + more : -1 - old);
            refused += good ? 0 : 1;
        }
        __syncthreads();
        const int here = min(kThreads, requests - base);
        const uint32_t pages = (uint32_t)(taken - taken_before);
        for (uint32_t n = (uint32_t)tid; n < pages && writes; n += kThreads) {
            const int r = first_above(upto, 0, here, n);
            const uint32_t before = r ? upto[r - 1] : 0u;
            table[(int64_t)(base + r) * width + first_col[r] + (int)(n - before)] = free_pages[free - 1 - (taken_before + n)];
        }
    }
    if (refused) atomicAdd(&refused_sum, refused);
    __syncthreads();
    if (tid == 0 && writes) {
        left[0] = (int32_t)(free - taken);
        left[1] = refused_sum;
    }
    // rows of this workgroup (requests <= kThreads: the sums of the one round are still there)
    const int first_row = (int)blockIdx.x * rows_each, last_row = min(first_row + rows_each, rows);
    for (int t = first_row + tid; t < last_row; t += kThreads) {
        const int r = first_above(end_row, 0, requests, t);
        int pos = 0, slot = -1;
        if (r < requests && row_to_pos[r] != kRefused) {
            pos = row_to_pos[r] + t;
            const int col = pos >> page_shift;
            const int page = col < first_col[r] ? table[(int64_t)r * width + col]
                                                : free_pages[free - 1 - ((r ? upto[r - 1] : 0u) + (uint32_t)(col - first_col[r]))];
            slot = (int)((uint32_t)page << page_shift) + (pos & round);
        }
        positions[t] = pos;
        slots[t] = slot;
    }
}

__global__ __launch_bounds__(256) void rows_kernel(int requests, int rows, int64_t width, int page_shift, const int32_t *table,
                                                   const int32_t *start, const int32_t *kv_lens, int32_t *positions, int32_t *slots) {
    const int t0 = (int)blockIdx.x * 256, t = t0 + (int)threadIdx.x;
    // requests of this workgroup's first and last row (uniform), then the thread's own among them
    const int lo = first_above(start + 1, 0, requests, t0), hi = first_above(start + 1, lo, requests, min(t0 + 255, rows - 1));
    if (t >= rows) return;
    const int b = first_above(start + 1, lo, min(hi + 1, requests), t);
    int pos = 0, slot = -1;
    if (b < requests && kv_lens[b] >= 0) {
        pos = kv_lens[b] - start[b + 1] + t;
        slot = (int)((uint32_t)table[(int64_t)b * width + (pos >> page_shift)] << page_shift) + (pos & ((1 << page_shift) - 1));
    }
    positions[t] = pos;
    slots[t] = slot;
}

bool overlap(const int32_t *a, int64_t na, const int32_t *b, int64_t nb) {
    return reinterpret_cast<uintptr_t>(a) < reinterpret_cast<uintptr_t>(b + nb) && reinterpret_cast<uintptr_t>(b) < reinterpret_cast<uintptr_t>(a + na);
}

}  // namespace

hipError_t launch_kv_assign(int64_t requests, int64_t rows, int64_t width, int page_shift, int64_t capacity, const int32_t *new_tokens,
                            const int32_t *lens, const int32_t *free_pages, const int32_t *free_count, int32_t *table,
                            int32_t *start, int32_t *kv_lens, int32_t *positions, int32_t *slots, int32_t *left, hipStream_t stream) {
    const bool in_place = overlap(lens, requests, kv_lens, requests) || overlap(free_count, 1, left, 2);
    const bool one = requests <= kThreads && (rows <= kRowsAlone || !in_place);
    const int each = !one ? 0 : rows <= kRowsAlone ? kRowsAlone : kRowsEach;
    const int groups = one && rows > kRowsAlone ? (int)((rows + kRowsEach - 1) / kRowsEach) : 1;
    hipLaunchKernelGGL(assign_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, (int)requests, (int)rows, width, page_shift, capacity,
                       new_tokens, lens, free_pages, free_count, table, start, kv_lens, positions, slots, left, each);
    if (!one && rows > 0)
        hipLaunchKernelGGL(rows_kernel, dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, stream, (int)requests, (int)rows, width, page_shift,
                           table, start, kv_lens, positions, slots);
    return hipGetLastError();
}

}  // namespace dmr
