// esp_evict_slots: of each request's list the entries that stay: its first ones, its last ones, and of the others those with the largest sums (of
// attention weights), up to a budget; both lists keep the order that the entries had.  Four bytes of a list entry and four of its slot's sum are read,
// four written: what counts is the number of steps that depend on each other.
//
// The smallest sum that stays is found by its digits, from the highest on: sums as unsigned numbers that order alike, 11, 11 and 10 bits, a histogram
// of the digit among the entries that have the digits found so far, and the digit in which the count of larger ones passes what is to be kept.  Of
// entries equal to it the first ones stay.  Counts are whole numbers: the order in which they are added does not matter.
//   Where no list is longer than 2048 entries each is one workgroup's: entries in its registers, histograms in its LDS, one launch.
//   Otherwise a first launch takes the sums of all entries, a lane's each from another line of memory: a CU is given some 0.15 lines a cycle, so 16384
//   entries that one CU took for itself were 44 us, spread over all of them 3.  Lists of up to 16384 are one workgroup's again: 16 lists of 32 .. 4096
//   2.7 and 7.3 us, most of it three times a histogram, a search and a wait; 162 of 45 .. 11760 21 us, in chunks 27, 4 of 16000 24 and 25.
//   Where one is longer, those of more than 4096 are cut into chunks of 4096: each digit is a launch over all of them, with a histogram per request in
//   the workspace; with the last one a chunk leaves what it would keep for each last digit, so that the next launch can write its part behind those
//   before it.  64 lists of 1024 .. 131072: sums 9.6 us, digits 5.2, 5.4 and 6.2, lists 9.8.
#include "evict.h"

namespace esp {

constexpr int kEvThreads = 1024;                  // of a workgroup
constexpr int kEvRounds = 4;                      // entries of a thread
constexpr int kEvShort = kEvRounds * kEvThreads;  // entries of a request that is one workgroup's
constexpr int kEvFew = 256, kEvFewRounds = 8, kEvOneLaunch = kEvFewRounds * kEvFew;   // where all lists are this short, and no other launch comes before
constexpr int kEvMiddle = 16 * kEvThreads;        // the same, where none is longer
constexpr int kEvChunk = kEvRounds * kEvThreads;  // of the longer ones
constexpr int kEvBins = 2048, kEvHist = 2 * kEvBins + 1024;   // of a digit at most; of the three digits
constexpr int kEvFrom = 1025 + 7;                 // (a multiple of 16 bytes)
// Requests up to which a workgroup adds up those before its own by itself, in one launch.  That work goes by their square, and is still the less of the
// two: 1024 lists of 4 .. 64 8.3 us, by the two launches for longer lists 17.1; 8192 of 1 .. 64 54 against 92, of 64 .. 1024 89 against 169; past it
// 16384 of 1 .. 64 156 against 181, 24576 314 against 277.
constexpr int32_t kEvOwnOffsets = 8192;

// where the launches for long lists keep what they share
struct EvictSpace {
    int32_t* chunk_first;                         // [B + 1] chunks of the long requests before this one
    int32_t* number;                              // [B] of this one among the long ones
    uint32_t* keys;                               // [total]
    int32_t* hist;                                // [long requests][kEvHist]
    uint2* found;                                 // [long requests][2] digits so far, and how many entries that have them are still to be taken
    uint16_t* from;                               // [chunks][kEvFrom] entries that stay if those with the digits found and a last digit from d on do
};
static int64_t long_most(int32_t total) { return (int64_t)total / (kEvShort + 1); }
static int64_t chunks_most(int32_t total) { return (int64_t)total / kEvChunk + long_most(total); }
static size_t evict_space(EvictSpace* s, char* at, int32_t B, int32_t total) {
    size_t n = 0;
    auto take = [&](size_t bytes) { char* p = at + n; n += (bytes + 255) / 256 * 256; return p; };
    const size_t longs = (size_t)long_most(total), chunks = (size_t)chunks_most(total);
    EvictSpace x;
    x.chunk_first = (int32_t*)take(((size_t)B + 1) * 4);
    x.number = (int32_t*)take((size_t)B * 4);
    x.keys = (uint32_t*)take((size_t)total * 4);
    x.hist = (int32_t*)take(longs * kEvHist * 4);
    x.found = (uint2*)take(longs * 2 * 8);
    x.from = (uint16_t*)take(chunks * kEvFrom * 2);
    if (s) *s = x;
    return n;
}
size_t evict_workspace_bytes(int32_t B, int32_t total_tokens, int32_t max_len) {
    return max_len <= kEvOneLaunch && B <= kEvOwnOffsets ? 256 : evict_space(nullptr, nullptr, B, total_tokens) + 256;
}

// Sums as unsigned numbers that order alike: NaN above all, both zeros the same; an entry without a slot in the pool below all.
__device__ __forceinline__ uint32_t key_of(const EvictArgs& a, int32_t slot) {
    if (slot < 0 || slot >= a.num_slots) return 0;
    const float x = a.sums[slot];
    if (x != x) return 0xffffffffu;
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// how many of a request's n entries stay
__device__ __forceinline__ int32_t stays(const EvictArgs& a, int32_t b, int32_t n) {
    int64_t m = a.budgets ? a.budgets[b] : a.budget;
    const int64_t always = (int64_t)a.keep_first + a.keep_last;
    if (m < always) m = always;
    return m < n ? (int32_t)m : n;
}
__device__ __forceinline__ bool always_stays(const EvictArgs& a, uint32_t i, int32_t n) { return i < (uint32_t)a.keep_first || (int64_t)i >= (int64_t)n - a.keep_last; }

// Sum of the wavefront's lanes up to this one.
__device__ __forceinline__ int32_t upto_lane(int32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);    // from 1, 2, 4 and 8 lanes below within a row of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // the last lane of rows 0 and 2 to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // and of the lower half to the upper
    return x;
}
// Sums over the workgroup's threads before this one's, and of all.
template <int WAVES>
__device__ __forceinline__ int32_t before(int32_t x, int32_t& all, int32_t* s_wave) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t upto = upto_lane(x);
    __syncthreads();
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    const int32_t w = upto_lane(lane < WAVES ? s_wave[lane] : 0);
    all = __builtin_amdgcn_readlane(w, 63);
    return (wave > 0 ? __shfl(w, wave - 1) : 0) + upto - x;
}

// The digit in which the count of entries, from the highest digit on, passes `want` (at least 1, at most the histogram's sum), how many of its entries
// are still to be taken, and whether those are all that it has.  By one wavefront: a lane has BINS / 64 digits in a row.  Digit d's count lies at
// place(d), so that lanes read different banks.
template <int BINS> __device__ __forceinline__ int place(uint32_t d) { return (int)((d & (BINS / 64 - 1)) * 64 + d / (BINS / 64)); }
struct Digit { uint32_t digit; int32_t want, all; };
template <int BINS, class P>
__device__ __forceinline__ Digit find_digit(P hist, int32_t want) {
    constexpr int N = BINS / 64;
    const int lane = threadIdx.x & 63, down = 63 - lane;             // lane 0 has the highest ones
    int32_t sum = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) sum += hist[k * 64 + down];
    const int32_t upto = upto_lane(sum);
    uint64_t hit = __builtin_amdgcn_ballot_w64(upto >= want);
    const int l = hit ? __builtin_ctzll(hit) : 63;
    const int32_t rest = want - __builtin_amdgcn_readlane(upto - sum, l);
    const int32_t h = lane < N ? hist[(N - 1 - lane) * 64 + (63 - l)] : 0, fine = upto_lane(h);
    hit = __builtin_amdgcn_ballot_w64(fine >= rest);
    const int k = hit ? __builtin_ctzll(hit) : N - 1;
    const int32_t left = rest - __builtin_amdgcn_readlane(fine - h, k);
    return {(uint32_t)((63 - l) * N + N - 1 - k), left, left == __builtin_amdgcn_readlane(h, k)};
}
__device__ __forceinline__ uint32_t digit_of(uint32_t key, int pass) { return pass == 0 ? key >> 21 : pass == 1 ? key >> 10 & 2047 : key & 1023; }
__device__ __forceinline__ int place_of(uint32_t key, int pass) { return pass == 2 ? place<1024>(digit_of(key, pass)) : place<kEvBins>(digit_of(key, pass)); }
__device__ __forceinline__ bool has_digits(uint32_t key, uint32_t so_far, int pass) { return pass == 0 || (pass == 1 ? key >> 21 == so_far >> 21 : key >> 10 == so_far >> 10); }
__device__ __forceinline__ uint32_t with_digit(uint32_t so_far, uint32_t digit, int pass) { return so_far | digit << (pass == 0 ? 21 : pass == 1 ? 10 : 0); }

template <int WAVES, int J>
struct EvictShared {
    int32_t hist[kEvHist];
    int32_t wave[WAVES];
    int32_t table[2][J * WAVES];
    Digit digit[3];
};

// Entries with a flag before this one's, in the order of i = threads * j + thread (J rounds, flags[j] the round's flags of this wavefront): the table's
// entry for (j, wavefront) plus the wavefront's own before the lane.
template <int WAVES, int J>
__device__ __forceinline__ void count_flags(const uint64_t (&flags)[J], int32_t* table) {
    constexpr int N = (J * WAVES + 63) / 64;                        // entries of a lane, in a row
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (lane == j) table[j * WAVES + wave] = __builtin_popcountll(flags[j]);
    __syncthreads();
    if (wave == 0) {
        int32_t x[N], sum = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) { x[e] = lane * N + e < J * WAVES ? table[lane * N + e] : 0; sum += x[e]; }
        int32_t from = upto_lane(sum) - sum;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (lane * N + e < J * WAVES) table[lane * N + e] = from;
            from += x[e];
        }
    }
    __syncthreads();
}
template <int WAVES>
__device__ __forceinline__ int32_t flags_before(uint64_t flags, int j, const int32_t* table) {
    return table[j * WAVES + (threadIdx.x >> 6)] + __builtin_popcountll(flags & ((1ull << (threadIdx.x & 63)) - 1));
}

__device__ __forceinline__ void put(const EvictArgs& a, bool keep, int64_t kept_at, int64_t freed_at, int32_t slot, int32_t pos) {
    if (keep) {
        if (kept_at < a.kept_capacity) {
            a.kept_slots[kept_at] = slot;
            if (a.kept_pos) a.kept_pos[kept_at] = pos;
        }
    } else if (freed_at < a.freed_capacity) {
        a.freed_slots[freed_at] = slot;
    }
}

// A request of up to J entries for each of the workgroup's threads.  Without keys: they are taken here, and the places of its lists added up (and
// written); otherwise both are there.
template <int THREADS, int J>
__device__ void evict_one(const EvictArgs& a, int32_t b, const uint32_t* keys, EvictShared<THREADS / 64, J>& s) {
    constexpr int WAVES = THREADS / 64;
    const int32_t s0 = a.seq_offsets[b], n = min(a.seq_offsets[b + 1], a.total_tokens) - s0;
    int32_t slot[J], pos[J];
    const int rounds = n > 0 ? (n + THREADS - 1) / THREADS : 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int32_t i = j * THREADS + (int32_t)threadIdx.x;
        slot[j] = j < rounds && i < n ? a.slot_idx[s0 + i] : -1;
        pos[j] = a.kept_pos && j < rounds && i < n ? a.token_pos[s0 + i] : 0;
    }
    const int32_t m = n > 0 ? stays(a, b, n) : 0, want = m - a.keep_first - a.keep_last;
    const bool choose = m < n && want > 0;
    if (choose)
        for (int x = threadIdx.x; x < kEvHist; x += THREADS) s.hist[x] = 0;
    int64_t kept_at, freed_at;
    if (!keys) {
        int32_t stay = 0, all;
        for (int32_t x = threadIdx.x; x < b; x += THREADS) {
            const int32_t nx = min(a.seq_offsets[x + 1], a.total_tokens) - a.seq_offsets[x];
            if (nx > 0) stay += stays(a, x, nx);
        }
        before<WAVES>(stay, all, s.wave);
        kept_at = all;
        freed_at = (int64_t)min(s0, a.total_tokens) - kept_at;
        if (threadIdx.x == 0) {
            a.kept_offsets[b] = (int32_t)min(kept_at, (int64_t)a.kept_capacity);
            a.freed_offsets[b] = (int32_t)min(freed_at, (int64_t)a.freed_capacity);
            if (b == a.B - 1) {
                a.kept_offsets[a.B] = (int32_t)min(kept_at + m, (int64_t)a.kept_capacity);
                a.freed_offsets[a.B] = (int32_t)min(freed_at + max(n, 0) - m, (int64_t)a.freed_capacity);
            }
        }
    } else {
        kept_at = a.kept_offsets[b];                                // (a cut list ends there: nothing is written past the capacity either way)
        freed_at = a.freed_offsets[b];
    }
    if (n <= 0) return;
    uint64_t keep[J];
    if (choose) {                                                   // (then no entry is both among the first and the last)
        uint32_t key[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int32_t i = j * THREADS + (int32_t)threadIdx.x;
            key[j] = j >= rounds || i >= n ? 0 : keys ? keys[s0 + i] : key_of(a, slot[j]);
        }
        Digit d = {0, want, 0};
        uint32_t so_far = 0;
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            int32_t* const hist = s.hist + pass * kEvBins;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int32_t i = j * THREADS + (int32_t)threadIdx.x;
                if (j < rounds && i < n && !always_stays(a, i, n) && has_digits(key[j], so_far, pass)) atomicAdd(&hist[place_of(key[j], pass)], 1);
            }
            __syncthreads();
            if (threadIdx.x < 64) {
                d = pass == 2 ? find_digit<1024>(hist, d.want) : find_digit<kEvBins>(hist, d.want);
                if (threadIdx.x == 0) s.digit[pass] = d;
            }
            __syncthreads();
            d = s.digit[pass];
            so_far = with_digit(so_far, d.digit, pass);
        }
        uint64_t equal[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int32_t i = j * THREADS + (int32_t)threadIdx.x;
            const bool in = j < rounds && i < n, fixed = in && always_stays(a, i, n);
            equal[j] = __builtin_amdgcn_ballot_w64(in && !fixed && key[j] == so_far);
            keep[j] = __builtin_amdgcn_ballot_w64(fixed || (in && key[j] > so_far));
        }
        if (d.all) {                                                // all of the equal ones stay
#pragma unroll
            for (int j = 0; j < J; ++j) keep[j] |= equal[j];
        } else {
            count_flags<WAVES, J>(equal, s.table[0]);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const bool taken = (equal[j] >> (threadIdx.x & 63) & 1) && flags_before<WAVES>(equal[j], j, s.table[0]) < d.want;
                keep[j] |= __builtin_amdgcn_ballot_w64(taken);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int32_t i = j * THREADS + (int32_t)threadIdx.x;
            keep[j] = __builtin_amdgcn_ballot_w64(j < rounds && i < n && (m == n || always_stays(a, i, n)));
        }
    }
    count_flags<WAVES, J>(keep, s.table[1]);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int32_t i = j * THREADS + (int32_t)threadIdx.x;
        if (j >= rounds || i >= n) continue;
        const int32_t at = flags_before<WAVES>(keep[j], j, s.table[1]);
        put(a, keep[j] >> (threadIdx.x & 63) & 1, kept_at + at, freed_at + i - at, slot[j], pos[j]);
    }
}

template <int THREADS, int J>
__global__ __launch_bounds__(THREADS) void evict_short_kernel(EvictArgs a, const uint32_t* keys) {
    __shared__ EvictShared<THREADS / 64, J> s;
    const int64_t b = wide_block();
    if (b < a.B) evict_one<THREADS, J>(a, (int32_t)b, keys, s);
}

// The first launch: workgroup 0 adds up where the lists of every request begin, and its chunks; the others take the sums as keys, and clear the histograms.
__global__ __launch_bounds__(kEvThreads) void evict_keys_kernel(EvictArgs a, EvictSpace w, int64_t hist_total) {
    __shared__ int32_t s_wave[kEvThreads / 64];
    const int64_t block = wide_block();
    if (block > 0) {
        const int64_t i = (block - 1) * kEvThreads + threadIdx.x, others = ((int64_t)a.total_tokens + kEvThreads - 1) / kEvThreads * kEvThreads;
        if (i < a.total_tokens) w.keys[i] = key_of(a, a.slot_idx[i]);
        for (int64_t x = i; x < hist_total && i < others; x += others) w.hist[x] = 0;
        return;
    }
    int32_t kept = 0, freed = 0, chunks = 0, longs = 0;             // (none of them is more than total_tokens)
    for (int64_t base = 0; base < a.B; base += kEvThreads) {
        const int32_t b = (int32_t)min(base + threadIdx.x, (int64_t)a.B - 1);
        const bool in = base + threadIdx.x < a.B;
        const int32_t n = in ? max(min(a.seq_offsets[b + 1], a.total_tokens) - a.seq_offsets[b], 0) : 0;
        const int32_t m = n > 0 ? stays(a, b, n) : 0;
        const bool is_long = n > kEvShort;
        int32_t all_kept, all_freed, all_chunks, all_longs;
        const int32_t k = kept + before<kEvThreads / 64>(m, all_kept, s_wave), f = freed + before<kEvThreads / 64>(n - m, all_freed, s_wave);
        const int32_t c = chunks + before<kEvThreads / 64>(is_long ? (int32_t)(((int64_t)n + kEvChunk - 1) / kEvChunk) : 0, all_chunks, s_wave);
        const int32_t l = longs + before<kEvThreads / 64>(is_long ? 1 : 0, all_longs, s_wave);
        if (in) {
            a.kept_offsets[b] = min(k, a.kept_capacity);
            a.freed_offsets[b] = min(f, a.freed_capacity);
            w.chunk_first[b] = c;
            w.number[b] = is_long ? l : -1;
        }
        kept += all_kept; freed += all_freed; chunks += all_chunks; longs += all_longs;
    }
    if (threadIdx.x == 0) {
        a.kept_offsets[a.B] = min(kept, a.kept_capacity);
        a.freed_offsets[a.B] = min(freed, a.freed_capacity);
        w.chunk_first[a.B] = chunks;
    }
}

// Launches over the chunks of the long lists: histograms of a digit.  The last digit's launch leaves how many of a chunk would stay with each last digit.
template <int PASS>
__global__ __launch_bounds__(kEvThreads) void evict_digit_kernel(EvictArgs a, EvictSpace w, int32_t chunks) {
    constexpr int J = kEvRounds, WAVES = kEvThreads / 64;
    __shared__ int32_t s_hist[kEvBins], s_wave[WAVES];
    const int64_t at = wide_block();
    if (at >= chunks || at >= w.chunk_first[a.B]) return;
    const RequestAt r = request_of((int32_t)at, w.chunk_first, a.B, threadIdx.x & 63);
    const int32_t b = r.b, s0 = a.seq_offsets[b], n = min(a.seq_offsets[b + 1], a.total_tokens) - s0, m = stays(a, b, n), number = w.number[b];
    const uint32_t i0 = (uint32_t)((int32_t)at - w.chunk_first[b]) * kEvChunk;
    const int32_t want = m - a.keep_first - a.keep_last;
    if (m == n || want == 0) return;                                // nothing to choose
    int32_t* const hist = w.hist + (int64_t)number * kEvHist;
    uint2 found = {0, (uint32_t)want};
    if (PASS > 0) {
        if (PASS > 1) found = w.found[2 * number + PASS - 2];
        const Digit d = find_digit<kEvBins>((const int32_t*)hist + (PASS == 1 ? 0 : kEvBins), (int32_t)found.y);   // (every wavefront for itself)
        found = {with_digit(found.x, d.digit, PASS - 1), (uint32_t)d.want};
        if (i0 == 0 && threadIdx.x == 0) w.found[2 * number + PASS - 1] = found;
    }
    for (int x = threadIdx.x; x < kEvBins; x += kEvThreads) s_hist[x] = 0;
    __syncthreads();
    uint32_t key[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const uint32_t i = min(i0 + j * kEvThreads + threadIdx.x, (uint32_t)n - 1);
        key[j] = w.keys[s0 + i];
    }
    int32_t stay = 0;                                               // whatever the last digit is
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const uint32_t i = i0 + j * kEvThreads + threadIdx.x;   // (past 2^31 next to its end)
        if (i >= (uint32_t)n) continue;
        if (always_stays(a, i, n)) ++stay;
        else if (has_digits(key[j], found.x, PASS)) atomicAdd(&s_hist[place_of(key[j], PASS)], 1);
        else if (key[j] > found.x) ++stay;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < (PASS == 2 ? 1024 : kEvBins); x += kEvThreads)
        if (s_hist[x] != 0) atomicAdd(&hist[PASS * kEvBins + x], s_hist[x]);
    if (PASS == 2) {
        static_assert(kEvThreads == 1024, "a digit to each thread");
        uint16_t* const from = w.from + at * kEvFrom;
        const uint32_t d = 1023 - threadIdx.x;
        const int32_t count = s_hist[place<1024>(d)];
        int32_t all_stay, all;
        before<WAVES>(stay, all_stay, s_wave);
        const int32_t above = before<WAVES>(count, all, s_wave);
        from[d] = (uint16_t)(all_stay + above + count);             // (at most the chunk's 4096)
        if (threadIdx.x == 0) from[1024] = (uint16_t)all_stay;
    }
}

// Then each chunk writes what stays of it behind what stays of those before it.  This launch, which takes longest by itself, also has the short lists,
// in its first workgroups.
__global__ __launch_bounds__(kEvThreads, 8) void evict_chunk_kernel(EvictArgs a, EvictSpace w, int32_t chunks) {
    constexpr int J = kEvRounds, WAVES = kEvThreads / 64;
    __shared__ EvictShared<WAVES, kEvRounds> s;
    int64_t at = wide_block();
    if (at < a.B) {
        if (w.number[at] < 0) evict_one<kEvThreads, kEvRounds>(a, (int32_t)at, w.keys, s);
        return;
    }
    at -= a.B;
    if (at >= chunks || at >= w.chunk_first[a.B]) return;
    const RequestAt r = request_of((int32_t)at, w.chunk_first, a.B, threadIdx.x & 63);
    const int32_t b = r.b, s0 = a.seq_offsets[b], n = min(a.seq_offsets[b + 1], a.total_tokens) - s0, m = stays(a, b, n), number = w.number[b];
    const int32_t chunk = (int32_t)at - w.chunk_first[b];
    const uint32_t i0 = (uint32_t)chunk * kEvChunk;
    const int32_t want = m - a.keep_first - a.keep_last;
    const bool choose = m < n && want > 0;
    uint32_t keys[J];
    int32_t slot[J], pos[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {                                   // (all asked for before the first is waited for)
        const uint32_t i = min(i0 + j * kEvThreads + threadIdx.x, (uint32_t)n - 1);
        keys[j] = choose ? w.keys[s0 + i] : 0;
        slot[j] = a.slot_idx[s0 + i];
        pos[j] = a.kept_pos ? a.token_pos[s0 + i] : 0;
    }
    // what stays of the chunks before: for sure, and with the last of the equal ones (of which the first `take` of the request stay)
    uint32_t smallest = 0;
    int32_t take = 0, stay_before, same_before = 0;
    if (choose) {
        const uint2 found = w.found[2 * number + 1];
        const Digit d = find_digit<1024>((const int32_t*)w.hist + (int64_t)number * kEvHist + 2 * kEvBins, (int32_t)found.y);
        smallest = with_digit(found.x, d.digit, 2);
        take = d.want;
        int32_t stay = 0, same = 0;
        for (int32_t x = threadIdx.x; x < chunk; x += kEvThreads) {
            const uint16_t* const from = w.from + (at - chunk + x) * kEvFrom + d.digit;
            stay += from[1];
            same += from[0] - from[1];
        }
        before<WAVES>(stay, stay_before, s.wave);
        before<WAVES>(same, same_before, s.wave);
    } else {                                                        // all, or the first and the last
        const int64_t last = (int64_t)i0 - ((int64_t)n - a.keep_last);
        stay_before = m == n ? (int32_t)i0 : (int32_t)(min((int64_t)i0, (int64_t)a.keep_first) + (last > 0 ? last : 0));
    }
    uint64_t keep[J], equal[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const uint32_t i = i0 + j * kEvThreads + threadIdx.x;   // (past 2^31 next to its end)
        const bool in = i < (uint32_t)n, fixed = in && (m == n || always_stays(a, i, n));
        equal[j] = __builtin_amdgcn_ballot_w64(choose && in && !fixed && keys[j] == smallest);
        keep[j] = __builtin_amdgcn_ballot_w64(fixed || (choose && in && keys[j] > smallest));
    }
    const int32_t taken_before = min(same_before, take), rest = take - taken_before;
    count_flags<WAVES, J>(equal, s.table[0]);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const bool taken = (equal[j] >> (threadIdx.x & 63) & 1) && flags_before<WAVES>(equal[j], j, s.table[0]) < rest;
        keep[j] |= __builtin_amdgcn_ballot_w64(taken);
    }
    count_flags<WAVES, J>(keep, s.table[1]);
    const int64_t kept_before = (int64_t)stay_before + taken_before, kept_at = a.kept_offsets[b] + kept_before, freed_at = a.freed_offsets[b] + i0 - kept_before;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const uint32_t i = i0 + j * kEvThreads + threadIdx.x;   // (past 2^31 next to its end)
        if (i >= (uint32_t)n) continue;
        const int32_t flags = flags_before<WAVES>(keep[j], j, s.table[1]);
        put(a, keep[j] >> (threadIdx.x & 63) & 1, kept_at + flags, freed_at + (i - i0) - flags, slot[j], pos[j]);
    }
}

__global__ void evict_none_kernel(int32_t* kept_offsets, int32_t* freed_offsets) { *kept_offsets = *freed_offsets = 0; }

esp_status launch_evict(const EvictArgs& a, void* workspace, hipStream_t stream) {
    if (a.B == 0) {
        hipLaunchKernelGGL(evict_none_kernel, dim3(1), dim3(1), 0, stream, a.kept_offsets, a.freed_offsets);
        return check_launch("evict_none_kernel");
    }
    if (a.max_len <= kEvOneLaunch && a.B <= kEvOwnOffsets) {
        hipLaunchKernelGGL((evict_short_kernel<kEvFew, kEvFewRounds>), wide_grid(a.B), dim3(kEvFew), 0, stream, a, (const uint32_t*)nullptr);
        return check_launch("evict_short_kernel");
    }
    EvictSpace w;
    evict_space(&w, (char*)workspace, a.B, a.total_tokens);
    const int64_t chunks = a.max_len > kEvMiddle ? chunks_most(a.total_tokens) : 0, hist = chunks > 0 ? long_most(a.total_tokens) * kEvHist : 0;
    hipLaunchKernelGGL(evict_keys_kernel, wide_grid(1 + ((int64_t)a.total_tokens + kEvThreads - 1) / kEvThreads), dim3(kEvThreads), 0, stream, a, w, hist);
    esp_status st = check_launch("evict_keys_kernel");
    if (st != ESP_OK) return st;
    if (chunks == 0 && a.max_len > kEvShort) {
        hipLaunchKernelGGL((evict_short_kernel<kEvThreads, kEvMiddle / kEvThreads>), wide_grid(a.B), dim3(kEvThreads), 0, stream, a, (const uint32_t*)w.keys);
        return check_launch("evict_short_kernel");
    }
    if (chunks == 0) {
        hipLaunchKernelGGL((evict_short_kernel<kEvThreads, kEvRounds>), wide_grid(a.B), dim3(kEvThreads), 0, stream, a, (const uint32_t*)w.keys);
        return check_launch("evict_short_kernel");
    }
    hipLaunchKernelGGL(evict_digit_kernel<0>, wide_grid(chunks), dim3(kEvThreads), 0, stream, a, w, (int32_t)chunks);
    hipLaunchKernelGGL(evict_digit_kernel<1>, wide_grid(chunks), dim3(kEvThreads), 0, stream, a, w, (int32_t)chunks);
    hipLaunchKernelGGL(evict_digit_kernel<2>, wide_grid(chunks), dim3(kEvThreads), 0, stream, a, w, (int32_t)chunks);
    hipLaunchKernelGGL(evict_chunk_kernel, wide_grid(chunks + a.B), dim3(kEvThreads), 0, stream, a, w, (int32_t)chunks);
    return check_launch("evict kernels");
}

}  // namespace esp
