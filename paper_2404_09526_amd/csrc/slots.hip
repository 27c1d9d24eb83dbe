// Block tables and slot lists on the GPU, from request lengths.
//   esp_extend_block_table: request b gets the pages that its tokens from old_lens[b] up to new_lens[b] need, in order of the requests from a
//     list of free ones: n_b = ceil(new / page) - ceil(old / page), entry ceil(old / page) + e of its row is free page sum_{b' < b} n_b' + e;
//   esp_build_slots: the pool slots of the requests' tokens, one request after another: token i of request b is at
//     table[row_b][i / page] * page + i % page; the offsets of the requests are the prefix sums of their counts.
// Both are a prefix sum over the requests and then a map over its total, all elements alike; with a few hundred requests what counts is
// the chain of round trips, so both are one launch: every workgroup takes the prefix sum itself (the lengths are a few KB in the L2),
// 1024 requests at a time, and then its share of the elements.
#include "esp_common.h"

namespace esp {

constexpr int kSlotThreads = 256;
constexpr int kSlotRequests = 1024;               // of a round: four a thread
constexpr int kSlotChunk = kSlotThreads * 4;      // elements of a workgroup at a time: four a thread, next to each other

__device__ __forceinline__ int32_t clip32(int64_t x, int32_t most) { return (int32_t)(x < most ? x : most); }

// Prefix sums of the counts of up to 1024 requests: off[i] = min(base + sum of the counts before request i, limit) for i = 0 .. n, and
// base moves on.  count(i) is asked for once for each request by one thread.
template <class Count>
__device__ __forceinline__ void scan_counts(int32_t n, int64_t& base, int32_t limit, int32_t* off, int64_t* wave_sum, Count count) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t c[4];
    int64_t mine = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = 4 * (int)threadIdx.x + u;
        c[u] = i < n ? count(i) : 0;
        mine += c[u];
    }
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t below = __shfl_up(upto, d);
        if (lane >= d) upto += below;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int64_t before = base, all = base;
#pragma unroll
    for (int w = 0; w < kSlotThreads / 64; ++w) {
        if (w < wave) before += wave_sum[w];
        all += wave_sum[w];
    }
    before += upto - mine;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = 4 * (int)threadIdx.x + u;
        if (i < n) off[i] = clip32(before, limit);
        before += c[u];
    }
    if (threadIdx.x == 0) off[n] = clip32(all, limit);
    base = all;
    __syncthreads();
}

// the request of element j: the last i with off[i] <= j (off[0] <= j < off[n])
__device__ __forceinline__ int find_request(const int32_t* off, int n, int32_t j) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= j) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int32_t pages_of(int32_t len, int32_t page) { return len <= 0 ? 0 : (int32_t)(((uint32_t)len - 1) / (uint32_t)page) + 1; }

__global__ __launch_bounds__(kSlotThreads) void extend_table_kernel(const int32_t* __restrict__ free_pages, int32_t n_free, const int32_t* __restrict__ req_row,
                                                                    const int32_t* __restrict__ old_lens, const int32_t* __restrict__ new_lens,
                                                                    int32_t B, int32_t page, int32_t* __restrict__ table, int32_t rows, int32_t width,
                                                                    int32_t* __restrict__ taken) {
    __shared__ int32_t off[kSlotRequests + 1];
    __shared__ int64_t wave_sum[kSlotThreads / 64];
    __shared__ int2 at[kSlotRequests];             // row, and its entry where the request's new pages begin
    int64_t base = 0;
    if (B == 0 && blockIdx.x == 0 && threadIdx.x == 0) taken[0] = 0;
    for (int64_t r0 = 0; r0 < B; r0 += kSlotRequests) {
        const int32_t n = (int32_t)min((int64_t)kSlotRequests, B - r0);
        scan_counts(n, base, INT32_MAX, off, wave_sum, [&](int i) {
            const int32_t b = (int32_t)r0 + i, row = req_row ? req_row[b] : b, from = pages_of(old_lens[b], page);
            const int32_t to = min(pages_of(new_lens[b], page), width);
            at[i] = make_int2(row, from);
            return row >= 0 && row < rows && to > from ? to - from : 0;
        });
        if (blockIdx.x == 0)
            for (int i = threadIdx.x; i <= n; i += kSlotThreads) taken[r0 + i] = off[i];
        const int32_t first = off[0], end = off[n];
        // chunk c of the elements is workgroup c % gridDim.x's, whatever round it falls into
        const int64_t c0 = first / kSlotChunk, turn = ((int64_t)blockIdx.x - c0 % gridDim.x + gridDim.x) % gridDim.x;
        for (int64_t c = c0 + turn; c * kSlotChunk < end; c += gridDim.x) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t j = c * kSlotChunk + u * kSlotThreads + threadIdx.x;
                if (j < first || j >= end) continue;
                const int i = find_request(off, n, (int32_t)j);
                table[(int64_t)at[i].x * width + at[i].y + ((int32_t)j - off[i])] = j < n_free ? free_pages[j] : -1;
            }
        }
        __syncthreads();                           // read: the next round may overwrite it
    }
}

__global__ __launch_bounds__(kSlotThreads) void build_slots_kernel(const int32_t* __restrict__ table, int32_t rows, int32_t width, int32_t page,
                                                                   const int32_t* __restrict__ req_row, const int32_t* __restrict__ first_token,
                                                                   const int32_t* __restrict__ lens, int32_t B, int32_t keep_first, int32_t keep_last,
                                                                   int32_t pos_first, int32_t pos_stride, int32_t capacity,
                                                                   int32_t* __restrict__ seq_offsets, int32_t* __restrict__ slots, int32_t* __restrict__ pos) {
    __shared__ int32_t off[kSlotRequests + 1];
    __shared__ int64_t wave_sum[kSlotThreads / 64];
    // Token of element e of a request: first + e, and from element `head` on `jump` more (a window's first tokens come before it).
    struct Request { int32_t row, first, head, jump; };
    __shared__ Request of[kSlotRequests];
    int64_t base = 0;
    if (B == 0 && blockIdx.x == 0 && threadIdx.x == 0) seq_offsets[0] = 0;
    for (int64_t r0 = 0; r0 < B; r0 += kSlotRequests) {
        const int32_t n = (int32_t)min((int64_t)kSlotRequests, B - r0);
        scan_counts(n, base, capacity, off, wave_sum, [&](int i) {
            const int32_t b = (int32_t)r0 + i, len = max(lens[b], 0), f = first_token ? max(first_token[b], 0) : 0;
            const int32_t tail = max(len - keep_last, 0), head = max(min(keep_first, tail) - f, 0), from = max(f, tail);
            of[i] = Request{req_row ? req_row[b] : b, f, head, from - f - head};
            return head + max(len - from, 0);
        });
        if (blockIdx.x == 0)
            for (int i = threadIdx.x; i <= n; i += kSlotThreads) seq_offsets[r0 + i] = off[i];
        const int32_t first = off[0], end = off[n];
        const int64_t c0 = first / kSlotChunk, turn = ((int64_t)blockIdx.x - c0 % gridDim.x + gridDim.x) % gridDim.x;
        for (int64_t c = c0 + turn; c * kSlotChunk < end; c += gridDim.x) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t j = c * kSlotChunk + u * kSlotThreads + threadIdx.x;
                if (j < first || j >= end) continue;
                const int i = find_request(off, n, (int32_t)j);
                const Request r = of[i];
                const int32_t e = (int32_t)j - off[i];
                const uint32_t t = (uint32_t)r.first + e + (e >= r.head ? r.jump : 0), p = t / (uint32_t)page;
                int32_t slot = -1;
                if (r.row >= 0 && r.row < rows && p < (uint32_t)width) {
                    const int32_t entry = table[(int64_t)r.row * width + p];
                    if (entry >= 0) slot = (int32_t)((uint32_t)entry * page + (t - p * page));
                }
                slots[j] = slot;
                if (pos) pos[j] = (int32_t)((uint32_t)pos_first + t * (uint32_t)pos_stride);
            }
        }
        __syncthreads();
    }
}

static unsigned slot_grid(int64_t elements) {
    const int64_t chunks = (elements + kSlotChunk - 1) / kSlotChunk;
    return (unsigned)(chunks < 1 ? 1 : chunks > 2048 ? 2048 : chunks);
}

esp_status launch_extend_table(const int32_t* free_pages, int32_t n_free, const int32_t* req_row, const int32_t* old_lens, const int32_t* new_lens,
                               int32_t B, int32_t page, int32_t* table, int32_t rows, int32_t width, int32_t* taken, hipStream_t stream) {
    // (how many pages there are to place is not known here; a workgroup that finds none for it ends after the prefix sum)
    const int64_t most = (int64_t)B * width < n_free ? (int64_t)B * width : n_free;
    hipLaunchKernelGGL(extend_table_kernel, dim3(slot_grid(most) < 256 ? slot_grid(most) : 256), dim3(kSlotThreads), 0, stream, free_pages, n_free, req_row,
                       old_lens, new_lens, B, page, table, rows, width, taken);
    return check_launch("extend_table_kernel");
}

esp_status launch_build_slots(const int32_t* table, int32_t rows, int32_t width, int32_t page, const int32_t* req_row, const int32_t* first_token,
                              const int32_t* lens, int32_t B, int32_t keep_first, int32_t keep_last, int32_t pos_first, int32_t pos_stride,
                              int32_t capacity, int32_t* seq_offsets, int32_t* slots, int32_t* pos, hipStream_t stream) {
    hipLaunchKernelGGL(build_slots_kernel, dim3(slot_grid(capacity)), dim3(kSlotThreads), 0, stream, table, rows, width, page, req_row, first_token, lens,
                       B, keep_first, keep_last > 0 ? keep_last : INT32_MAX, pos_first, pos_stride, capacity, seq_offsets, slots, pos);
    return check_launch("build_slots_kernel");
}

}  // namespace esp
