// Block tables and slot lists on the GPU, from request lengths.
//   esp_extend_block_table: request b gets the pages that its tokens from old_lens[b] up to new_lens[b] need, in order of the requests from a
//     list of free ones: n_b = ceil(new / page) - ceil(old / page), entry ceil(old / page) + e of its row is free page sum_{b' < b} n_b' + e;
//   esp_build_slots: the pool slots of the requests' tokens, one request after another: token i of request b is at
//     table[row_b][i / page] * page + i % page; the offsets of the requests are the prefix sums of their counts.
// Both are a prefix sum over the requests and then a map over its total, all elements alike; with a few hundred requests what counts is
// the chain of round trips, so both are one launch: every workgroup takes the prefix sum itself (the lengths are a few KB in the L2),
// 1024 requests at a time, and then its share of the elements.
// Measured: the pages of 64 requests' next tokens 4.6 us, the slots of 16 requests of some 600 tokens 4.8 us, hardly more than an empty launch.  Long lists are
// bound by their bytes, written and of the table: 256 lists of 7.2 M slots in all, pages of one (57.5 MB), took 34 us with one slot a thread, with four, whole pieces
// of 16 bytes, 15.6 us, 3.7 TB/s.
#include "esp_common.h"

namespace esp {

constexpr int kSlotThreads = 256;
constexpr int kSlotRequests = 1024;               // of a round: four a thread
constexpr int kSlotMost = 1536;                   // workgroups: as many as fit the chip at once

struct Int4 { int32_t x, y, z, w; };               // 16 bytes that need not lie on 16

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
        // a thread's elements, and the workgroup's chunk of them: chunk c is workgroup c's, c + gridDim.x's, ...
        const int per = end - first <= kSlotThreads * (int64_t)gridDim.x ? 1 : 4, chunk = kSlotThreads * per;
        for (int64_t c = first / chunk + blockIdx.x; c * chunk < end; c += gridDim.x) {
            // four elements next to each other: one search, and where they are one request's whole pieces of 16 bytes
            const int64_t j0 = c * chunk + per * (int64_t)threadIdx.x;
            if (j0 + per <= first || j0 >= end) continue;
            int i = find_request(off, n, (int32_t)max(j0, (int64_t)first));
            if (per == 4 && j0 >= first && j0 + 4 <= off[i + 1] && j0 + 4 <= n_free) {
                *(Int4*)(table + ((int64_t)at[i].x * width + at[i].y + ((int32_t)j0 - off[i]))) = *(const Int4*)(free_pages + j0);
                continue;
            }
            int32_t page_no[4];                                     // all loads before the first store: one round trip
            int64_t to[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t j = j0 + u;
                to[u] = -1;
                if (u >= per || j < first || j >= end) continue;
                while (off[i + 1] <= j) ++i;
                to[u] = (int64_t)at[i].x * width + at[i].y + ((int32_t)j - off[i]);
                page_no[u] = j < n_free ? free_pages[j] : -1;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (to[u] >= 0) table[to[u]] = page_no[u];
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
    const bool power = (page & (page - 1)) == 0;
    const int shift = __builtin_ctz(page);
    auto page_of = [&](uint32_t t) { return power ? t >> shift : t / (uint32_t)page; };
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
        const int per = end - first <= kSlotThreads * (int64_t)gridDim.x ? 1 : 4, chunk = kSlotThreads * per;
        for (int64_t c = first / chunk + blockIdx.x; c * chunk < end; c += gridDim.x) {
            const int64_t j0 = c * chunk + per * (int64_t)threadIdx.x;
            if (j0 + per <= first || j0 >= end) continue;
            int i = find_request(off, n, (int32_t)max(j0, (int64_t)first));
            Request r = of[i];
            const int32_t e0 = (int32_t)j0 - off[i];
            // four elements next to each other that are four tokens next to each other, in a row that has them all
            if (per == 4 && j0 >= first && j0 + 4 <= off[i + 1] && (e0 >= r.head || e0 + 4 <= r.head) && r.row >= 0 && r.row < rows) {
                const uint32_t t = (uint32_t)r.first + e0 + (e0 >= r.head ? r.jump : 0), p = page_of(t);
                if (p < (uint32_t)width && page_of(t + 3) < (uint32_t)width) {
                    const int32_t* const entries = table + ((int64_t)r.row * width + p);
                    Int4 slot;
                    if (page == 1) {
                        slot = *(const Int4*)entries;
                        slot = {max(slot.x, -1), max(slot.y, -1), max(slot.z, -1), max(slot.w, -1)};
                    } else {
                        int32_t to[4];
                        const int32_t last = page_of(t + 3) - p;     // of the four's entries: 0 (all on one page), 1, or with pages of two or three tokens 2
                        const int32_t entry[3] = {entries[0], entries[min(1, last)], entries[last]};
                        uint32_t at = t - p * page, of_page = 0;
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int32_t x = of_page == 0 ? entry[0] : of_page == 1 ? entry[1] : entry[2];
                            to[u] = x >= 0 ? (int32_t)((uint32_t)x * page + at) : -1;
                            if (++at == (uint32_t)page) { at = 0; ++of_page; }
                        }
                        slot = {to[0], to[1], to[2], to[3]};
                    }
                    *(Int4*)(slots + j0) = slot;
                    const uint32_t at = (uint32_t)pos_first + t * (uint32_t)pos_stride;
                    if (pos) *(Int4*)(pos + j0) = {(int32_t)at, (int32_t)(at + pos_stride), (int32_t)(at + 2 * (uint32_t)pos_stride), (int32_t)(at + 3 * (uint32_t)pos_stride)};
                    continue;
                }
            }
            int32_t entry[4];                                       // all loads before the first store: one round trip
            uint32_t token[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t j = j0 + u;
                if (u >= per || j < first || j >= end) continue;
                while (off[i + 1] <= j) ++i;
                r = of[i];
                const int32_t e = (int32_t)j - off[i];
                token[u] = (uint32_t)r.first + e + (e >= r.head ? r.jump : 0);
                const uint32_t p = page_of(token[u]);
                entry[u] = r.row >= 0 && r.row < rows && p < (uint32_t)width ? table[(int64_t)r.row * width + p] : -1;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t j = j0 + u;
                if (u >= per || j < first || j >= end) continue;
                slots[j] = entry[u] >= 0 ? (int32_t)((uint32_t)entry[u] * page + (token[u] - page_of(token[u]) * page)) : -1;
                if (pos) pos[j] = (int32_t)((uint32_t)pos_first + token[u] * (uint32_t)pos_stride);
            }
        }
        __syncthreads();
    }
}

static unsigned slot_grid(int64_t elements) {
    const int64_t chunks = (elements + kSlotThreads - 1) / kSlotThreads;
    return (unsigned)(chunks < 1 ? 1 : chunks > kSlotMost ? kSlotMost : chunks);
}

esp_status launch_extend_table(const int32_t* free_pages, int32_t n_free, const int32_t* req_row, const int32_t* old_lens, const int32_t* new_lens,
                               int32_t B, int32_t page, int32_t* table, int32_t rows, int32_t width, int32_t* taken, hipStream_t stream) {
    // (how many pages there are to place is not known here; a workgroup that finds none for it ends after the prefix sum.  So there are at most two to a CU:
    // a step has few new pages, and of a list that is longer each takes several chunks.)
    const int64_t most = (int64_t)B * width < n_free ? (int64_t)B * width : n_free;
    hipLaunchKernelGGL(extend_table_kernel, dim3(slot_grid(most) < 512 ? slot_grid(most) : 512), dim3(kSlotThreads), 0, stream, free_pages, n_free, req_row,
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
