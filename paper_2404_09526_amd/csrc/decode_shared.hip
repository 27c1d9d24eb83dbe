// esp_partial_attn_decode_shared: decode of a batch whose requests come in groups that share a long prefix (a system prompt, a document): every
// request's query attends the pool rows of its group's prefix and its own.  Read once per request, as the plain decode call does, the prefix is
// n times its bytes; here it is read once per group.  The queries of a group are packed rows, (request, query head of the group) pairs of a
// KV head, and the columns of MFMA tiles:
//   S^T [keys x columns] = K Q^T,   O^T [128 x columns] += V^T P^T
// against the prefix in ranges of keys, a partial (accumulator, maximum, sum) per (range, row).  With few columns the prefix is bound by the
// memory, as the requests' own rows are, from some 200 columns on by the wavefronts' work on its tiles; so one launch works on both, prefix ranges and own
// ranges side by side, and what bounds the one is left over by the other (shared_order).  A second launch combines the partials of both kinds.
// Workgroups are of four wavefronts, two of them on a CU, so that one starts and ends beside the other's sweep, or of eight for long prefixes and little
// else, which read a tile of keys once for 256 columns: which, and ranges of what length, is estimated (shared_plan).
// Weights are rounded to bf16 for the product, as in the plain decode on the matrix cores (fp32 operands run at a sixteenth of the rate, and weights in two bf16 parts are
// twice the product); their sum is that of the rounded ones, and accumulators, maxima and sums are fp32.  Against 64 bits the result is off by 2.3e-3 of its size, 1.7e-3
// of it the rounding of O itself.
// Measured: 64 requests of some 750 tokens behind 2051, 32 / 8 heads, 52 us (207 MB); 16 behind 65536, 32 / 32, 213 (1.24 GB, 5.8 TB/s); 256 in three groups behind 65549,
// 40000 and 20011, 32 / 8, 412 (1.59 GB and 193 GFLOP); four short requests 7.3.  The plain decode on the joined lists (requests of 600 tokens each, 32 / 8 heads): 64
// behind 2000 90.7 -> 41.5 us, 2 behind 2000 13.5 -> 12.4, 16 behind 30000 227 -> 46; nothing to share: 64 requests in groups of one behind 100 38.6 -> 45.6.
#include <math.h>

#include "column_tile.h"
#include "decode_merge.h"

namespace esp {

constexpr int kSharedTile = kColKBytes + kColVBytes;
// A workgroup of the first launch has four wavefronts, two of them share a CU, or eight, which have it alone.
template <int WAVES>
struct SharedGeometry {
    static constexpr int half = WAVES * (kSharedTile / 2), most = 4096;   // of the tiles' LDS; keys of a prefix range: its slots lie in LDS
    static constexpr int own = 512;                                 // keys of an own range, a wavefront's: its slots too
    static constexpr int lds = 2 * half + most * 4;
    // tiles that wavefronts have for themselves lie before the lists; the blocks that rows are stored from, which are larger, may lie on them: they come last
    static_assert(WAVES * kSharedTile <= 2 * half && WAVES * (kColWaveBytes + 32 * 8) <= lds && WAVES * own <= most, "the wavefronts' tiles and blocks fit");
    static_assert(lds <= 16 * 1024 * 10 * WAVES / 8, "two of four, or one of eight, on a CU");
};
constexpr int kWholeWaves = 8;                                      // of a workgroup of the one-launch form
// The offset that a wide workgroup takes probabilities against is moved (and the accumulators with it) only where those of a tile sum up to more than
// this: moved with every new maximum, as the plain decode's, it moves in half of the tiles for some column of the 32.  Larger
// probabilities change nothing for their bf16 or the fp32 sums.
constexpr float kSharedSum = 4096.f;

// Partials of ranges of `range` keys: accumulators [rows][128], then (maximum, sum) pairs [rows], a row to a query head.  Those of a list that begins at token s0
// lie from slot s0 / range + (the list's number) on, a slot being Hq rows of a request, or of a prefix max_group times as many.  So groups of very different
// size would take the largest's room for every range; then a prefix's lie by request, `each` of Hq rows to one, as many as the longest prefix has (0: by slot).
struct SharedParts { float* acc; float* ml; int32_t range, each; };
// The work of the first launch: `prefix` workgroups on the prefix (units (range, KV head), `blocks` column blocks each) and `own` on the requests' own
// rows, in eights: among the first `first` eights first_prefix are the prefix's, up to number `mixed` the rest of those, spread evenly both times; own rows alone
// come last.
struct SharedWork {
    int32_t prefix, own, units, blocks, first, first_prefix, mixed;
    __device__ __forceinline__ uint32_t before(uint32_t eight) const {   // eights of the prefix among the first so many
        const uint32_t all = (uint32_t)prefix >> 3, n = first, of_n = first_prefix, m = mixed;
        if (eight < n) return (uint64_t)eight * of_n / n;
        return eight < m ? of_n + (uint64_t)(eight - n) * (all - of_n) / (m - n) : all;
    }
};

// V of the rows past the end of a tile that is not full.  K's repeat the last row, and their weight is 0: of V that would not do, as 0 times an infinity is not 0.
// (Cleared in LDS when V had landed, the call of four short requests took 0.2 us more.)
__device__ const u32x4 kZeroRow[kHeadDim / 8] = {};

// A wavefront on tiles of 32 keys of its own, number `first`, first + step, ...: their rows go to its block of the LDS, the next tile's K as soon
// as this one's scores are taken, its V as soon as this one's has been read.  list: the slots of all `seg` keys, in LDS (a load of them on the way would
// be waited for with everything that was asked for before it).
__device__ __forceinline__ void sweep_tiles(Columns& cols, const bf16x8 (&qf)[8], uint32_t lds_k, const char* kbase, const char* vbase, uint32_t row_bytes,
                                            int first, int step, int32_t seg, const int32_t* list, float scale_log2, int lane) {
    const int hi = lane >> 5;
    uint32_t slot[8];
    auto fetch_k = [&](int i) {
#pragma unroll
        for (int n = 0; n < 8; ++n) slot[n] = (uint32_t)list[min(32 * i + col_row(n, lane), seg - 1)];
#pragma unroll
        for (int n = 0; n < 8; ++n) load_to_lds_b128_at_nt(lds_k + 1024 * n, kbase + ((uint64_t)slot[n] * row_bytes + col_k_within(n, lane)));
    };
    auto fetch_v = [&](int i) {
        const int rows = seg - 32 * i;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const char* from = vbase + ((uint64_t)slot[n] * row_bytes + col_v_within(lane));
            if (rows < 32 && col_row(n, lane) >= rows) from = (const char*)kZeroRow + col_v_within(lane);
            load_to_lds_b128_at_nt(lds_k + kColKBytes + 1024 * n, from);
        }
    };
    if (32 * first >= seg) return;
    fetch_k(first);
    fetch_v(first);
    for (int i = first; 32 * i < seg; i += step) {
        const int rows = min(32, seg - 32 * i);
        const bool next = 32 * (i + step) < seg;
        wait_vm<8>();                                               // K has landed; V may be on its way
        floatx16 sc = cols.scores(qf);
        if (next) {
            asm volatile("" :: "v"(sc));                            // K has been read
            fetch_k(i + step);
        }
        if (rows < 32) {                                            // keys past the end are hidden
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + 4 * hi + (r & 3) >= rows) sc[r] = -INFINITY;
        }
        Columns::PFrag pf[2];
        cols.weigh(sc, scale_log2, pf);
        if (next) wait_vm<8>(); else wait_vm<0>();
        cols.accumulate(pf);
        if (next) fetch_v(i + step);
    }
}

// Ranges counted from each list's first token on (lists: offsets[b] .. offsets[b + 1]), all whole ones first, then what is left of each list: where
// range i is, as request_range (esp_common.h) finds it, but 64 N lists at a time, whose offsets are one round trip for both kinds where that is all.
// total: entries that there are (offsets past them stand for that end); longest: tokens of a list that count.  members: offsets of something else by list, whose bounds for the list that is found go to m0 and m1 (asked for together
// with its own).
struct ListRange { int32_t b, t0, t1, part, w; };                   // list; tokens; number within the list, and along all (s0 / range + part)
template <int N>
__device__ __forceinline__ ListRange find_range(int32_t i, int32_t range, int32_t B, const int32_t* offsets, int32_t total, int32_t longest, int lane, const int32_t* members,
                                                int32_t& m0, int32_t& m1) {
    int32_t s0[N], s1[N], of0[N], of1[N];
#pragma unroll 1
    for (int rest = 0; rest < 2; ++rest) {
#pragma unroll 1
        for (int base = 0; base < B; base += 64 * N) {
            if (rest == 0 || B > 64 * N) {
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    const int b = min(base + 64 * u + lane, B - 1);
                    s0[u] = min(offsets[b], total); s1[u] = min(offsets[b + 1], total);
                    if (members) { of0[u] = members[b]; of1[u] = members[b + 1]; }
                }
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                if (base + 64 * u >= B) break;
                const int32_t len = min(max(s1[u] - s0[u], 0), longest), whole = (uint32_t)len / (uint32_t)range;
                const int32_t n = base + 64 * u + lane >= B ? 0 : rest ? (len > whole * range ? 1 : 0) : whole;
                int32_t upto = n;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int32_t below = __shfl_up(upto, d);
                    if (lane >= d) upto += below;
                }
                const uint64_t hit = __builtin_amdgcn_ballot_w64(upto > i);
                if (hit) {
                    const int l = __builtin_ctzll(hit);
                    const int32_t start = __builtin_amdgcn_readlane(s0[u], l), left = __builtin_amdgcn_readlane(len, l);
                    const int32_t part = rest ? __builtin_amdgcn_readlane(whole, l) : i - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
                    const int32_t t0 = start + part * range;
                    if (members) { m0 = __builtin_amdgcn_readlane(of0[u], l); m1 = __builtin_amdgcn_readlane(of1[u], l); }
                    return {base + 64 * u + l, t0, t0 + min(range, left - part * range), part, start / range + part};
                }
                i -= __builtin_amdgcn_readlane(upto, 63);
            }
        }
    }
    return {0, 0, 0, 0, 0};                                            // the launch is an upper bound
}

// The requests' own rows: a wavefront alone on (a range of a request, KV head, up to 32 of its query heads), heads next to each other as in a
// pool row; its partial goes to that range's slot.
template <int WAVES>
__device__ __forceinline__ void shared_own(const SharedArgs& a, float scale_log2, const SharedParts& mine, int32_t index, unsigned char* smem, int wave, int lane) {
    const int qi = lane & 31, hi = lane >> 5;
    const int G = a.Hq / a.Hkv, chunks = (G + 31) / 32;
    const uint32_t unit = (uint32_t)index * WAVES + wave, i = unit / (uint32_t)(a.Hkv * chunks), rest = unit - i * (uint32_t)(a.Hkv * chunks);
    const int kvh = rest / (uint32_t)chunks, g0 = (rest - kvh * chunks) * 32, ng = min(32, G - g0), h0 = kvh * G + g0;
    int32_t none;
    const ListRange at = find_range<4>(i, mine.range, a.B, a.seq_offsets, a.total_tokens, INT32_MAX, lane, nullptr, none, none);
    const int32_t seg = at.t1 - at.t0;
    if (seg <= 0) return;
    int32_t* const list = (int32_t*)(smem + 2 * SharedGeometry<WAVES>::half) + wave * SharedGeometry<WAVES>::own;
    for (int j = lane; j < seg; j += 64) list[j] = a.slot_idx[at.t0 + j];
    bf16x8 qf[8];
    const int64_t row = (int64_t)at.b * a.Hq + h0 + min(qi, ng - 1);
    const uint16_t* qp = (const uint16_t*)a.q + row * kHeadDim + 8 * hi;
#pragma unroll
    for (int t = 0; t < 8; ++t) qf[t] = *(const bf16x8*)(qp + 16 * t);
    asm volatile("" :: "v"(qf[0]), "v"(qf[1]), "v"(qf[2]), "v"(qf[3]), "v"(qf[4]), "v"(qf[5]), "v"(qf[6]), "v"(qf[7]));   // here before the transfers, whose waits count
    const uint32_t lds_k = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem + wave * kSharedTile;
    Columns cols;
    cols.place(lds_k, lane);
    cols.clear();
    sweep_tiles(cols, qf, lds_k, a.k_pool + (uint32_t)kvh * (kHeadDim * 2), a.v_pool + (uint32_t)kvh * (kHeadDim * 2), (uint32_t)a.Hkv * (kHeadDim * 2), 0, 1, seg, list,
                scale_log2, lane);
    const float l = half_swap_sum(cols.l), l_r = half_swap_sum(cols.l_r), fix = l_r > 0.f ? l / l_r : 0.f;
    if (qi >= ng) return;
    const int64_t ph = (int64_t)(at.w + at.b) * a.Hq + h0 + qi;
    float* dst = mine.acc + ph * kHeadDim + 4 * hi;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *(float4*)(dst + 32 * db + 2 * r) = make_float4(cols.oacc[db][r] * fix, cols.oacc[db][r + 1] * fix, cols.oacc[db][r + 2] * fix, cols.oacc[db][r + 3] * fix);
    if (hi == 0) *(float2*)(mine.ml + ph * 2) = make_float2(cols.m, l);
}

// The prefix.  A workgroup has COLS tiles of 32 columns, a wavefront one, and the COLS wavefronts that have different
// columns (a team) share tiles of 32 keys in LDS, so that a row of K and V comes from memory once for 32 COLS columns; the WAVES / COLS teams take
// the tiles in turn, all teams' tiles are a step.
// A step of a wavefront is two phases that take about as long as each other: the scores of its tile become probabilities (vector ALU); then the
// products, the NEXT tile's scores and this one's V, without a wait, each followed by the LDS read of the operand that takes its place
// (matrix cores).  Of eight wavefronts the two of a SIMD are a phase apart, the barriers between phases keep them so; of four each has another workgroup's beside
// it, and one barrier a step is enough.  K's operands are thus read two steps ahead
// of the scores, V's one step ahead of their products, and each has a ring of COLS stages (16 KiB a wavefront together): group j of transfers is V of step j
// and K of step j + 1.
// A team of one wavefront shares nothing: it waits for its own rows only (sweep_tiles).
struct PrefixPart { ListRange at; int32_t b0, seg, n_all, kvh; };  // a range of group at.b's prefix: its keys, the group's first request and packed rows
template <int WAVES, int COLS, bool ONCE>
__device__ __forceinline__ void shared_prefix(const SharedArgs& a, float scale_log2, const SharedParts& parts, const PrefixPart& part, uint32_t cb, unsigned char* smem,
                                              int wave, int lane) {
    constexpr int TEAMS = WAVES / COLS, STEP = 32 * TEAMS, MOVES = 8 / COLS;   // MOVES: a wavefront's transfers of K, and of V, of a tile
    const int team = wave / COLS, ct = wave % COLS;
    const int qi = lane & 31, hi = lane >> 5;
    const ListRange& at = part.at;
    const int32_t t0 = at.t0, b0 = part.b0, seg = part.seg, n_all = part.n_all, kvh = part.kvh, G = a.Hq / a.Hkv;
    if (n_all <= (int32_t)cb * (32 * COLS)) return;
    const int32_t rho0 = cb * (32 * COLS) + ct * 32, n_rows = n_all - rho0;   // (columns of this wavefront, up to 32; none: it only moves tiles)

    int32_t* const list = (int32_t*)(smem + 2 * SharedGeometry<WAVES>::half);
    for (int i = threadIdx.x; i < seg; i += WAVES * 64) list[i] = a.prefix_slots[t0 + i];

    // row of this column within the group's queries (past the last: the last one's, whose results are not written)
    const int32_t rho = min(rho0 + qi, n_all - 1), of = rho / G;
    const int32_t row = of * a.Hq + kvh * G + (rho - of * G);
    bf16x8 qf[8];
    const uint16_t* qp = (const uint16_t*)a.q + ((int64_t)b0 * a.Hq + row) * kHeadDim + 8 * hi;
#pragma unroll
    for (int t = 0; t < 8; ++t) qf[t] = *(const bf16x8*)(qp + 16 * t);
    asm volatile("" :: "v"(qf[0]), "v"(qf[1]), "v"(qf[2]), "v"(qf[3]), "v"(qf[4]), "v"(qf[5]), "v"(qf[6]), "v"(qf[7]));   // here before the transfers, whose waits count

    const uint32_t row_bytes = (uint32_t)a.Hkv * (kHeadDim * 2);
    const char* kbase = a.k_pool + (uint32_t)kvh * (kHeadDim * 2);
    const char* vbase = a.v_pool + (uint32_t)kvh * (kHeadDim * 2);
    const uint32_t lds = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem;
    Columns cols;
    cols.clear();
    __syncthreads();                                                // the list is there
    if constexpr (COLS == 1) {
        cols.place(lds + wave * kSharedTile, lane);
        sweep_tiles(cols, qf, lds + wave * kSharedTile, kbase, vbase, row_bytes, wave, WAVES, seg, list, scale_log2, lane);
    } else {
        constexpr bool PHASES = WAVES == 8;
        constexpr int STAGES = COLS, kTile = kColKBytes;            // of K; V's is as large
        constexpr int kRing = STAGES * TEAMS * kTile;
        static_assert(2 * kRing == 2 * SharedGeometry<WAVES>::half, "both rings end where the list begins");
        const bool late = PHASES && wave >= WAVES / 2;                 // (wavefronts w and w + 4 are on one SIMD)
        const int steps = (seg + STEP - 1) / STEP;
        auto k_tile = [&](int i) { return lds + ((i % STAGES) * TEAMS + team) * kTile; };
        auto v_tile = [&](int i) { return lds + kRing + ((i % STAGES) * TEAMS + team) * kTile; };
        // A wavefront's rows of a tile are the same for K and V: slots are looked up a group ahead, and a row's place is kept from K's group to V's.
        uint32_t slot[MOVES];
        uint64_t place[MOVES];
        // ONCE: these columns are all that the group has, and the rows pass once; otherwise other workgroups find them in the L2.  (4 requests behind 100 thousand tokens are
        // 8 % faster past the caches, 100 behind 65536 8 % slower.)
        auto fetch_row = [](uint32_t to, const char* from) {
            if constexpr (ONCE) load_to_lds_b128_at_nt(to, from);
            else load_to_lds_b128_at(to, from);
        };
        auto look_up = [&](int i) {
#pragma unroll
            for (int x = 0; x < MOVES; ++x) slot[x] = (uint32_t)list[min(i * STEP + team * 32 + col_row(ct + COLS * x, lane), seg - 1)];
        };
        auto fetch_k = [&](int i) {
#pragma unroll
            for (int x = 0; x < MOVES; ++x) {
                const int n = ct + COLS * x;
                place[x] = (uint64_t)slot[x] * row_bytes;
                const uint32_t to = __builtin_amdgcn_readfirstlane(k_tile(i) + 1024 * n);
                fetch_row(to, kbase + (place[x] + col_k_within(n, lane)));
            }
        };
        auto fetch_v = [&](int i) {
#pragma unroll
            for (int x = 0; x < MOVES; ++x) {
                const uint32_t to = __builtin_amdgcn_readfirstlane(v_tile(i) + 1024 * (ct + COLS * x));
                fetch_row(to, vbase + (place[x] + col_v_within(lane)));
            }
        };
        auto fetch_group = [&](int j) {
            if (j < steps) fetch_v(j);
            if (j + 1 < steps) { fetch_k(j + 1); look_up(j + 2); }
        };
        // Group i + 1, of which the products of step i read, has landed: STAGES - 2 groups behind it may be on their way (the last one has no K).
        auto landed = [&](int i) {
            if (i + STAGES < steps) { wait_vm<2 * (STAGES - 2) * MOVES>(); return; }
            constexpr int kMore = COLS > 2 ? MOVES : 0, kEight = COLS == 8 ? MOVES : 0;   // (as many as the stages allow)
            const int left = steps - 2 - i;
            if (left <= 0) wait_vm<0>();
            else if (left == 1) wait_vm<kMore>();
            else if (left == 2) wait_vm<3 * kMore>();
            else if (left == 3) wait_vm<5 * kEight>();
            else if (left == 4) wait_vm<7 * kEight>();
            else if (left == 5) wait_vm<9 * kEight>();
            else wait_vm<11 * kEight>();
        };
        auto meet = [] {
            __builtin_amdgcn_sched_barrier(0);
            wg_barrier();
            __builtin_amdgcn_sched_barrier(0);
        };
        cols.place(0, lane);                                        // (offsets within a tile; of V behind K's)
        const uint32_t k_rd = cols.k_rd;
        bf16x8 kf[8];
        Columns::VFrag vf[8];
        auto read_k = [&](uint32_t tile, int t) { kf[t] = *(const ESP_LDS bf16x8*)(uintptr_t)((k_rd ^ (t << 5)) + tile); };
        auto read_v = [&](uint32_t tile, int p) {
            const uint32_t vp = cols.v_rd[p & 3] + (tile - kColKBytes + (16 * (p >> 2)) * 256);
            vf[p].s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ESP_LDS short4_t*)(uintptr_t)(vp));
            vf[p].s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ESP_LDS short4_t*)(uintptr_t)(vp + 8 * 256));
        };
        floatx16 sc;
        auto zero = [&] {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = 0.f;
        };

        look_up(0);
        fetch_k(0);
        look_up(1);
#pragma unroll 1
        for (int j = 0; j < STAGES - 1; ++j) fetch_group(j);
        landed(-1);
        meet();
        zero();
        if (n_rows > 0) {
#pragma unroll
            for (int t = 0; t < 8; ++t) read_k(k_tile(0), t);
#pragma unroll
            for (int t = 0; t < 8; ++t) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t], qf[t], sc, 0, 0, 0);
#pragma unroll
            for (int t = 0; t < 8; ++t) { read_k(k_tile(1), t); read_v(v_tile(0), t); }
        }
        meet();                                                     // K of steps 0 and 1 and V of step 0 are read
        fetch_group(STAGES - 1);
        if (late) { landed(0); meet(); }
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
            Columns::PFrag pf[2];
            if (n_rows > 0) {
                const int here = seg - i * STEP - team * 32;
                if (here < 32) {                                    // keys past the end are hidden, and their V, the last row's again, is 0 (as 0 times an infinity is not)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r >> 2) + 4 * hi + (r & 3) >= here) {
                            sc[r] = -INFINITY;
#pragma unroll
                            for (int db = 0; db < 4; ++db) vf[4 * (r >> 3) + db].s[(r >> 2) & 1][r & 3] = 0;   // (that key's element of the operands)
                        }
                }
                // Probabilities against the offset in use, without a look at the scores first; their sums tell whether it has to move.
                float sum, sum_r;
                auto weigh = [&] {
                    const float sub = cols.m == -INFINITY ? 0.f : cols.m;
                    sum = sum_r = 0.f;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[2 * c], scale_log2, -sub));
                        const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[2 * c + 1], scale_log2, -sub));
                        sum += p0 + p1;
                        const uint32_t pk = pack_bf16(p0, p1);
                        sum_r = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum_r, false);
                        pf[c >> 2].u[c & 3] = pk;
                    }
                };
                weigh();
                if (__builtin_amdgcn_ballot_w64(sum > kSharedSum || cols.m == -INFINITY) != 0) {
                    float top = sc[0];
#pragma unroll
                    for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
                    top = half_swap_max(top) * scale_log2;
                    // (a column that has seen nothing but -inf and NaN stays as it is: exp2(-inf - -inf) must not leak into sums that are zero)
                    const float to = fmaxf(cols.m, top), alpha = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(cols.m - to);
                    cols.m = to;
                    cols.l *= alpha; cols.l_r *= alpha;
#pragma unroll
                    for (int db = 0; db < 4; ++db)
#pragma unroll
                        for (int r = 0; r < 16; ++r) cols.oacc[db][r] *= alpha;
                    weigh();
                }
                cols.l += sum; cols.l_r += sum_r;
            }
            if (!late) landed(i);
            meet();
            // (past the last step there is nothing to read: what is there instead is never used)
            if (n_rows > 0) {
                __builtin_amdgcn_s_setprio(1);                      // (the other wavefront's vector instructions take what these leave, not the other way round)
                const uint32_t k_next = k_tile(i + 2), v_next = v_tile(i + 1);
                zero();
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t], qf[t], sc, 0, 0, 0);
                    read_k(k_next, t);
                    cols.oacc[t & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t].v, pf[t >> 2].v, cols.oacc[t & 3], 0, 0, 0);
                    read_v(v_next, t);
                    __builtin_amdgcn_sched_barrier(0);              // (in this order: the chain of the scores beside the sums of V, an operand's place taken over at once)
                }
                __builtin_amdgcn_s_setprio(0);
            }
            // every wavefront is done with the products of the step before this one, and with what they read
            fetch_group(i + STAGES);
            if (late) landed(i + 1);
            if (PHASES) meet();
        }
        if (PHASES && !late) meet();
    }
    // The wavefronts leave their columns as rows of 128 (and 4 of padding) floats in LDS, maxima and sums behind them; then every wavefront combines
    // the teams' rows and stores its share of them, 32 lanes a row.  (Stored from the accumulators, 16 bytes of 32 rows at a time, 256 such blocks took 11 us.)
    constexpr int kPitch = kHeadDim + 4;
    constexpr int kRowPairs = 16 * COLS / WAVES;                    // of a wavefront
    static_assert(32 * kPitch * 4 <= kColWaveBytes, "the rows fit");
    __syncthreads();                                                // the tiles are read
    {
        const float l = half_swap_sum(cols.l), l_r = half_swap_sum(cols.l_r), fix = l_r > 0.f ? l / l_r : 0.f;   // (the rounded probabilities were multiplied)
        float* mine = (float*)(smem + wave * kColWaveBytes) + qi * kPitch + 4 * hi;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4*)(mine + 32 * db + 2 * r) = make_float4(cols.oacc[db][r] * fix, cols.oacc[db][r + 1] * fix, cols.oacc[db][r + 2] * fix, cols.oacc[db][r + 3] * fix);
        if (hi == 0) ((float2*)(smem + WAVES * kColWaveBytes))[wave * 32 + qi] = make_float2(cols.m, l);
    }
    __syncthreads();
    // the range's rows for the group's first request, and how far apart those of two requests lie
    const int64_t slot = (parts.each ? (int64_t)b0 * parts.each + at.part : (int64_t)(at.w + at.b) * a.max_group) * a.Hq, apart = (int64_t)(parts.each ? parts.each : 1) * a.Hq;
#pragma unroll 1
    for (int i = 0; i < kRowPairs; ++i) {
        const int in = (wave * kRowPairs + i) * 2 + hi;              // of the workgroup's 32 COLS columns
        const int32_t col = cb * (32 * COLS) + in;
        if (col >= n_all) continue;
        const int w0 = in >> 5, at_row = in & 31;                   // team t's are those of wavefront w0 + COLS t
        float2 ml[TEAMS];
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < TEAMS; ++t) {
            ml[t] = ((const float2*)(smem + WAVES * kColWaveBytes))[(w0 + COLS * t) * 32 + at_row];
            mx = fmaxf(mx, ml[t].x);
        }
        float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
        float lsum = 0.f;
#pragma unroll
        for (int t = 0; t < TEAMS; ++t) {
            const float4 x = *(const float4*)((const float*)(smem + (w0 + COLS * t) * kColWaveBytes) + at_row * kPitch + 4 * qi);
            // a team that saw no key (sum 0) has nothing to add; a NaN sum shows in l * c
            const float c = ml[t].y > 0.f ? __builtin_amdgcn_exp2f(ml[t].x - mx) : 0.f;
            lsum += ml[t].y * c;
            out.x += x.x * c; out.y += x.y * c; out.z += x.z * c; out.w += x.w * c;
        }
        const int32_t req = col / G;
        const int64_t ph = slot + req * apart + kvh * G + (col - req * G);
        ((float4*)(parts.acc + ph * kHeadDim))[qi] = out;
        if (qi == 0) *(float2*)(parts.ml + ph * 2) = make_float2(mx, lsum);
    }
}

// Column tiles of a workgroup of so many wavefronts on the prefix of a group with so many packed rows.
__host__ __device__ __forceinline__ int shared_cols(int64_t rows, int waves) { return rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 || waves == 4 ? 4 : 8; }

template <int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void shared_partial_kernel(SharedArgs a, float scale_log2, SharedParts parts, SharedParts mine, SharedWork work) {
    __shared__ __attribute__((aligned(1024))) unsigned char smem[SharedGeometry<WAVES>::lds];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the eight that this workgroup is of, and how many before it are the prefix's: the workgroups of an eight lie on all XCDs in turn
    const uint32_t eight = blockIdx.x >> 3, of = blockIdx.x & 7, before = work.before(eight), after = work.before(eight + 1);
    if (after == before) {
        shared_own<WAVES>(a, scale_log2, mine, (eight - before) * 8 + of, smem, wave, lane);
        return;
    }
    // Unit: (range, KV head), heads next to each other as in a pool row.  The column blocks of a unit are in eights that follow each other: on one
    // XCD, whose L2 then has the rows.
    const uint32_t unit = before / work.blocks * 8 + of, cb = before % work.blocks;
    if (unit >= (uint32_t)work.units) return;
    PrefixPart part;
    part.kvh = unit % (uint32_t)a.Hkv;
    int32_t b1 = 0;
    part.b0 = 0;
    part.at = find_range<1>(unit / (uint32_t)a.Hkv, parts.range, a.n_groups, a.prefix_offsets, a.prefix_total, a.max_prefix, lane, a.group_offsets, part.b0, b1);
    part.n_all = min(min(b1, a.B) - part.b0, a.max_group) * (a.Hq / a.Hkv);
    part.seg = part.at.t1 - part.at.t0;
    if (part.seg <= 0 || part.n_all <= 0) return;
    if (part.n_all > 32 * WAVES) shared_prefix<WAVES, WAVES, false>(a, scale_log2, parts, part, cb, smem, wave, lane);
    else switch (shared_cols(part.n_all, WAVES)) {
        case 1: shared_prefix<WAVES, 1, true>(a, scale_log2, parts, part, cb, smem, wave, lane); break;
        case 2: shared_prefix<WAVES, 2, true>(a, scale_log2, parts, part, cb, smem, wave, lane); break;
        case 4: shared_prefix<WAVES, 4, true>(a, scale_log2, parts, part, cb, smem, wave, lane); break;
        default: shared_prefix<WAVES, WAVES, false>(a, scale_log2, parts, part, cb, smem, wave, lane);   // (eight: 2 % from the caches for less code)
    }
}

// Few short requests, in one launch: a workgroup has one request and KV head (a chunk of its query heads) and walks the prefix and the
// request's own rows as one list (as decode_whole.hip does with one); the prefix is read by each, from the caches, and no combination follows.
__global__ __launch_bounds__(kWholeWaves * 64, 2) void shared_whole_kernel(SharedArgs a, float scale_log2) {
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kWholeWaves * kColWaveBytes];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qi = lane & 31, hi = lane >> 5;
    const int b = blockIdx.x, kvh = blockIdx.y;
    const int32_t s0 = a.seq_offsets[b], s1 = min(a.seq_offsets[b + 1], a.total_tokens);   // (never past the slot list)
    int32_t p0 = 0, P = 0;
#pragma unroll 1
    for (int base = 0; base < a.n_groups; base += 64) {
        const int of = min(base + lane, a.n_groups - 1);
        const int32_t g0 = a.group_offsets[of], g1 = a.group_offsets[of + 1], from = a.prefix_offsets[of], to = min(a.prefix_offsets[of + 1], a.prefix_total);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(g0 <= b && b < g1);
        if (!hit) continue;
        const int l = __builtin_ctzll(hit);
        p0 = __builtin_amdgcn_readlane(from, l);
        if (b - __builtin_amdgcn_readlane(g0, l) < a.max_group) P = min(max(__builtin_amdgcn_readlane(to, l) - p0, 0), a.max_prefix);
        break;
    }
    const uint32_t n = (uint32_t)P + max(s1 - s0, 0);               // (without a sign: tiles that are looked ahead to may start past 2^31)
    const int32_t *const prefix = a.prefix_slots + p0, *const own = a.slot_idx + s0;
    auto tile_slots = [&](uint32_t i) {                             // lane: of tile row lane % 32 (rows past the end: the last)
        const uint32_t t = min(32 * i + qi, n - 1);
        return t < (uint32_t)P ? prefix[t] : own[t - P];
    };
    int32_t slots = 0, slots_next = 0;
    if (32 * wave < n) { slots = tile_slots(wave); slots_next = tile_slots(wave + kWholeWaves); }
    const int G = a.Hq / a.Hkv, g0 = blockIdx.z * 32, ng = min(32, G - g0);
    const uint32_t row_bytes = (uint32_t)a.Hkv * (kHeadDim * 2);
    const char* kbase = a.k_pool + (uint32_t)kvh * (kHeadDim * 2);
    const char* vbase = a.v_pool + (uint32_t)kvh * (kHeadDim * 2);
    const uint32_t lds_k = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem + wave * kColWaveBytes;
    const int64_t pair = (int64_t)b * a.Hq + kvh * G + g0 + min(qi, ng - 1);   // of this column (past the chunk: the last one's, nothing written)
    bf16x8 qf[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) qf[t] = *(const bf16x8*)((const uint16_t*)a.q + pair * kHeadDim + 16 * t + 8 * hi);
    asm volatile("" : "+v"(slots), "+v"(slots_next) : "v"(qf[0]), "v"(qf[1]), "v"(qf[2]), "v"(qf[3]), "v"(qf[4]), "v"(qf[5]), "v"(qf[6]), "v"(qf[7]));   // here before the transfers, whose waits count
    Columns cols;
    cols.place(lds_k, lane);
    cols.clear();
    auto fetch = [&](uint32_t to, const char* base, int32_t of, uint32_t i, bool is_k) {
        const uint32_t rows = n - 32 * i;                           // of the tile, or more
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const char* from = base + ((uint64_t)(uint32_t)__shfl(of, col_row(x, lane)) * row_bytes + (is_k ? col_k_within(x, lane) : col_v_within(lane)));
            if (!is_k && rows < 32 && col_row(x, lane) >= (int)rows) from = (const char*)kZeroRow + col_v_within(lane);
            load_to_lds_b128_at(to + 1024 * x, from);
        }
    };
    if (32 * wave < n) { fetch(lds_k, kbase, slots, wave, true); fetch(lds_k + kColKBytes, vbase, slots, wave, false); }
    for (uint32_t i = wave; 32 * i < n; i += kWholeWaves) {
        const int here = min(32u, n - 32 * i);
        const bool next = 32 * (i + kWholeWaves) < n;
        wait_vm<8>();                                               // K has landed; V may be on its way
        floatx16 sc = cols.scores(qf);
        if (next) {
            asm volatile("" :: "v"(sc));                            // K has been read
            fetch(lds_k, kbase, slots_next, i + kWholeWaves, true);
        }
        if (here < 32) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + 4 * hi + (r & 3) >= here) sc[r] = -INFINITY;
        }
        Columns::PFrag pf[2];
        cols.weigh(sc, scale_log2, pf);
        if (next) wait_vm<8>(); else wait_vm<0>();
        cols.accumulate(pf);
        if (next) {
            fetch(lds_k + kColKBytes, vbase, slots_next, i + kWholeWaves, false);
            slots_next = tile_slots(i + 2 * kWholeWaves);
        }
    }
    constexpr int N = 64 / kWholeWaves;
    float out[N], mx, lsum;
    cols.combine<kWholeWaves>(smem, wave, lane, out, mx, lsum);
    if (qi >= ng) return;
    const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;              // no token: 0; a NaN shows
    const int at = Columns::first_element<kWholeWaves>(wave, lane);
#pragma unroll
    for (int e = 0; e < N; e += 4)
        ((U32x2*)a.O)[(pair * kHeadDim + at + 2 * e) / 4] = U32x2{pack_bf16(out[e] * inv, out[e + 1] * inv), pack_bf16(out[e + 2] * inv, out[e + 3] * inv)};
    if (wave == 0 && hi == 0) a.LSE[pair] = lsum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(lsum)) * kLn2;
}

// Combination, as the plain decode's (decode.hip): groups of 32 lanes take a pair's partials in turn, four at a time, first those of the
// prefix, then its own.
template <int GROUPS>
__global__ __launch_bounds__(256) void shared_combine_kernel(SharedArgs a, int32_t pairs, SharedParts parts, SharedParts mine) {
    constexpr int U = 4;
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int64_t at = row_block() * (8 / GROUPS) + grp / GROUPS;
    if (at >= pairs) return;                                        // (a whole workgroup, or a pair is a wavefront and no barrier follows)
    const int pair = (int)at, g = grp % GROUPS;
    const int b = pair / a.Hq, h = pair - b * a.Hq;
    const int32_t s0 = a.seq_offsets[b], s1 = min(a.seq_offsets[b + 1], a.total_tokens);
    Weighted<4> sum;
    auto add = [&](const float* acc, const float* ml, int64_t first, int64_t step, int n) {
        for (int i = g; i < n; i += GROUPS * U) {
            float m[U], l[U], v[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = i + u * GROUPS;
                const int64_t ph = first + min(k, n - 1) * step;
                const float2 x = *(const float2*)(ml + ph * 2);
                const float4 o = load_once((const float4*)(acc + ph * kHeadDim + lane * 4));
                v[u][0] = o.x; v[u][1] = o.y; v[u][2] = o.z; v[u][3] = o.w;
                m[u] = x.x;
                l[u] = k < n ? x.y : 0.f;
            }
            sum.template add<false>(m, l, v);
        }
    };
    // the pair's group, and where its prefix lies: 64 groups at a time, their bounds asked for together
    const int l64 = threadIdx.x & 63;
#pragma unroll 1
    for (int base = 0; base < a.n_groups; base += 64) {
        const int of = min(base + l64, a.n_groups - 1);
        const int32_t g0 = a.group_offsets[of], g1 = a.group_offsets[of + 1], p0 = a.prefix_offsets[of], p1 = min(a.prefix_offsets[of + 1], a.prefix_total);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(g0 <= b && b < g1);
        if (!hit) continue;
        const int l = __builtin_ctzll(hit);
        const int32_t b0 = __builtin_amdgcn_readlane(g0, l), from = __builtin_amdgcn_readlane(p0, l), to = __builtin_amdgcn_readlane(p1, l);
        if (b - b0 < a.max_group && to > from) {
            const int64_t first = parts.each ? (int64_t)b * parts.each : (int64_t)(from / parts.range + base + l) * a.max_group + (b - b0);
            add(parts.acc, parts.ml, first * a.Hq + h, (int64_t)(parts.each ? 1 : a.max_group) * a.Hq, (min(to - from, a.max_prefix) - 1) / parts.range + 1);
        }
        break;
    }
    if (s1 > s0) add(mine.acc, mine.ml, ((int64_t)(s0 / mine.range) + b) * a.Hq + h, a.Hq, (s1 - s0 - 1) / mine.range + 1);

    float mx, Lt = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    if (GROUPS == 2) {
        mx = fmaxf(sum.M, __shfl_xor(sum.M, 32));
        const float c = __builtin_amdgcn_exp2f(sum.M - finite_offset(mx));
        Lt = sum.L * c;
        Lt += __shfl_xor(Lt, 32);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[e] = sum.acc[e] * c;
            o[e] += __shfl_xor(o[e], 32);
        }
    } else {
        __shared__ float sm[8], sl[8];
        __shared__ float4 sa[8][32];
        if (lane == 0) { sm[grp] = sum.M; sl[grp] = sum.L; }
        sa[grp][lane] = make_float4(sum.acc[0], sum.acc[1], sum.acc[2], sum.acc[3]);
        __syncthreads();
        if (g != 0) return;
        mx = sm[0];
#pragma unroll
        for (int u = 1; u < 8; ++u) mx = fmaxf(mx, sm[u]);
        const float ref = finite_offset(mx);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float c = __builtin_amdgcn_exp2f(sm[u] - ref);      // exp2(-inf) = 0 for an idle group
            const float4 t = sa[u][lane];
            Lt += sl[u] * c;
            o[0] += t.x * c; o[1] += t.y * c; o[2] += t.z * c; o[3] += t.w * c;
        }
    }
    if (g != 0) return;
    const float inv = Lt == 0.f ? 0.f : 1.0f / Lt;                  // no token anywhere: exactly 0
    ((U32x2*)a.O)[(int64_t)pair * (kHeadDim / 4) + lane] = U32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
    if (lane == 0) a.LSE[pair] = Lt == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(Lt)) * kLn2;
}

// The sizes of a call, and what its partials take.
struct SharedSizes {
    int32_t B, n_groups, prefix_total, max_prefix, max_group, total_tokens, Hq, Hkv;
    // Of so many times Hq rows: whole 256 bytes, and no more than 2^60 of them (such a call is refused).
    size_t bytes(int64_t times) const {
        const double all = (double)times * Hq * ((kHeadDim + 2) * sizeof(float));
        return all > 0x1p60 ? (size_t)1 << 60 : ((size_t)times * Hq * ((kHeadDim + 2) * sizeof(float)) + 255) / 256 * 256;
    }
    // Of the prefixes in ranges of so many keys, by request (to `each`) or by slot (0), whichever is less: a group's requests times its ranges, summed over all groups, can
    // be no more than either.
    int64_t prefix_rows(int32_t range, int32_t* each = nullptr) const {
        const int64_t most = ((int64_t)max_prefix + range - 1) / range, by_request = B * most, slots = (int64_t)prefix_total / range + n_groups;
        const bool by_slot = (double)slots * max_group < (double)by_request;
        if (each) *each = by_slot ? 0 : (int32_t)most;
        return by_slot ? slots * max_group : by_request;
    }
    int64_t own_rows(int32_t range) const { return total_tokens == 0 ? 0 : (int64_t)total_tokens / range + B; }   // (of requests of any lengths)
    // Room for them: for the shortest ranges, but beyond kRoom no more than the longest need.  It rises with every size, so a block that a call fits is large enough for all
    // smaller ones; the plan takes ranges that fit.  (Of 3000 drawn batches none would take others with more room; with 64 MiB 38 would, the worst for 20 % of its estimate.)
    static constexpr size_t kRoom = (size_t)128 << 20;
    static constexpr int32_t kLeast = 32, kMost = 4096, kOwnLeast = 64, kOwnMost = 512;   // keys of a range
    static size_t room(size_t most, size_t least) { return most < kRoom ? most : least > kRoom ? least : kRoom; }
    size_t prefix_room() const { return room(bytes(prefix_rows(kLeast)), bytes(prefix_rows(kMost))); }
    size_t own_room() const { return room(bytes(own_rows(kOwnLeast)), bytes(own_rows(kOwnMost))); }
    bool alone() const { return prefix_total == 0 || max_prefix == 0 || max_group == 0; }   // no prefix: the plain decode
    size_t workspace() const {
        const size_t plain = decode_workspace_bound(B, total_tokens, Hq, Hkv);
        if (alone()) return plain;
        const size_t all = prefix_room() + own_room();
        return all > plain ? all : plain;
    }
};

// The ranges of both kinds, and the workgroups that they are.
struct SharedPlan {
    int32_t range, own_range;                                       // keys of a range
    int32_t each;                                                   // partials of the prefix by request, or by slot (SharedParts)
    int64_t units, blocks, own;                                     // (range, KV head) pairs, column blocks of each; workgroups on own rows
    double us;                                                      // the estimate
    int waves, kind;                                                // of a workgroup: wavefronts, column tiles for an average group (2^kind)
    double share, last;                                             // the prefix's share of the time of all workgroups; a workgroup of it, of the whole launch
};
// Rounds of the chip from which on the order is not an even mixture (shared_order).
constexpr double kOneAfter = 1.6;
// Two workgroups of four wavefronts on a CU, or one of eight.  Of these estimates of the first launch's time, in us, with what its partials cost beside it, the least:
// a workgroup on the prefix takes a start and its steps, one on own rows a start and a time for each 32 keys of a wavefront, on a chip that they do not fill less of
// it; all of them together, spread evenly, and at the end a part of the longest, or of what comes last (shared_order), or, where they are only a few rounds of the chip,
// whole rounds; the longest alone; all rows at the memory's rate.  What is not known is how the groups differ: several are taken to be as large as their average.
// Fitted to 247 batches (1 .. 250 requests in 1 .. 5 groups, prefixes of 0 .. 130000 tokens, thirteen head layouts) with up to 130 choices each; of 60 others the estimates' choice was
// 4.8 % from the best on average, 25 % at most (3 + 10 + 52 requests behind 7798, 45217 and 197, 64 / 8 heads).  Four wavefronts at their best were the better by 6 % on average; eight were it for few long ranges (3 + 18 + 2 requests behind 47634, 102 and 3466 tokens,
// 32 / 4 heads, 30 us with eight, 44 with four; 16 behind 130000, 32 / 8, 115 and 127) and by 2 % for much work of more than 128 columns and nothing else.  So
// eight are taken where their estimate is 6 %, with more than 128 columns 8 %, the less (where it is less at all: 2 .. 3 % more time on average).
static SharedPlan shared_plan_for(int waves, const SharedSizes& of) {
    const int32_t B = of.B, n_groups = of.n_groups, prefix_total = of.prefix_total, max_group = of.max_group, total_tokens = of.total_tokens, Hq = of.Hq, Hkv = of.Hkv;
    constexpr double kOwnStart = 5.5, kOwnTile = 3.6, kTail = 0.15, kTailOwn = 0.44, kTailBoth = 0.23, kFewRounds = 3, kWholeRound = 1.1, kPartial = 0.0055, kBytesPerUs = 5.95e6;
    constexpr double kAlone = 0.43, kBlocks = 0.865;                // of a step's time: on a chip that is hardly filled; where blocks of four tiles find rows in the L2
    struct Times { double start, step; };
    constexpr Times kTimes[4] = {{5.6, 4.15}, {12.1, 1.57}, {8.3, 1.48}, {15.5, 1.04}};   // of a workgroup with 1, 2, 4, 8 column tiles
    constexpr int32_t kRanges[] = {SharedSizes::kLeast, 64, 128, 256, 384, 512, 768, 1024, 1536, 2048, SharedSizes::kMost};
    constexpr int32_t kOwnRanges[] = {SharedSizes::kOwnLeast, 128, 192, 256, 384, SharedSizes::kOwnMost};
    static_assert(kRanges[10] == SharedGeometry<4>::most && kRanges[10] == SharedGeometry<8>::most && kOwnRanges[5] == SharedGeometry<4>::own, "their slots lie in LDS");
    const size_t room = of.prefix_room(), own_room = of.own_room();
    SharedPlan p = {};
    const int64_t G = Hq / Hkv, chunks = (G + 31) / 32, mean = n_groups > 1 ? (B + n_groups / 2) / n_groups : max_group, rows = (mean > 1 ? mean : 1) * G;
    const int cols = shared_cols(rows, waves), kind = __builtin_ctz(cols);
    const double at_once = 256 * (8 / waves);
    const int64_t step = 32 * (waves / cols), wide = Hkv * ((rows + 32 * cols - 1) / (32 * cols));
    const double own_tiles = (double)total_tokens / 32 * Hkv * chunks / waves;
    const double memory = ((double)prefix_total + total_tokens) * Hkv * (4 * kHeadDim) / kBytesPerUs;
    auto own_wgs = [&](int32_t range) { return total_tokens == 0 ? 0 : (((int64_t)total_tokens / range + B) * Hkv * chunks + waves - 1) / waves; };
    p.us = HUGE_VAL;
    for (const int32_t range : kRanges) {
        if (of.bytes(of.prefix_rows(range)) > room) continue;       // (the longest fits)
        const double wgs = (ceil((double)prefix_total / range) + 0.5 * (n_groups - 1)) * wide;
        const double steps = (double)((range + step - 1) / step) * (kind == 2 && rows > 128 ? kBlocks : 1);
        for (const int32_t own_range : kOwnRanges) {
            if (of.bytes(of.own_rows(own_range)) > own_room) continue;
            const double own = (double)own_wgs(own_range), n = wgs + own, full = kAlone + (1 - kAlone) * fmin(1, n / at_once);
            const double one = kTimes[kind].start + kTimes[kind].step * steps * full, prefix_us = wgs * one;
            const double mine = kOwnStart + kOwnTile * full * own_range / 32, longest = total_tokens == 0 ? one : fmax(one, mine);
            const double sum = prefix_us + own * kOwnStart + own_tiles * kOwnTile * full;
            const double ends = own == 0 || n <= kOneAfter * at_once ? kTail * longest : kind <= 1 ? kTailOwn * mine : kTailBoth * (mine + one);
            double us = fmax(fmax(sum / at_once + ends, longest), memory);
            if (n <= kFewRounds * at_once) us = fmax(us, kWholeRound * ceil(n / at_once) * sum / n);
            us += wgs * cols * kPartial;
            if (us < p.us) {
                p.us = us; p.range = range; p.own_range = own_range;
                p.share = prefix_us / sum; p.last = one / (sum / at_once);
            }
            if (total_tokens == 0) break;
        }
        if (range >= prefix_total) break;
    }
    p.waves = waves;
    p.kind = kind;
    p.blocks = (max_group * G + 32 * waves - 1) / (32 * waves);     // (fewer column tiles than wavefronts are one block)
    p.units = ((int64_t)(prefix_total / p.range) + n_groups) * Hkv;
    of.prefix_rows(p.range, &p.each);
    p.own = own_wgs(p.own_range);
    return p;
}
static SharedPlan shared_plan(const SharedSizes& of) {
    const int32_t forced = forced_decode_plan();
    if (forced == 4 || forced == 8) return shared_plan_for(forced, of);
    const SharedPlan four = shared_plan_for(4, of), eight = shared_plan_for(8, of);
    return eight.us * (eight.kind == 3 ? 1.08 : 1.06) < four.us ? eight : four;
}
size_t decode_shared_workspace_bytes(int32_t B, int32_t n_groups, int32_t prefix_total, int32_t max_prefix, int32_t max_group, int32_t total_tokens,
                                     int32_t Hq, int32_t Hkv) {
    return SharedSizes{B, n_groups, prefix_total, max_prefix, max_group, total_tokens, Hq, Hkv}.workspace();
}

// Which calls run in one launch: those with no more workgroups than CUs whose estimate is the less.  In one launch: a start and an end, then the longest
// list's walk, or all lists' bytes from the caches, the prefix as often as there are requests; in ranges: what the plan says and a combination.  Measured on 280
// calls (1 .. 32 requests behind one prefix of 30 .. 4000 tokens, five head layouts; in ranges -> in one launch, us; * stays in ranges): two requests of
// 20 behind 300, 4 / 4 heads, 11.3 -> 8.5, of 300 behind 1000 11.6 -> 16.1*; 16 of 300 behind 30, 32 / 8, 14.8 -> 10.7, 16 of 20 behind 1000 15.6 -> 14.3, behind
// 2000 18.3 -> 22.1*; 32 of 300 behind 300, 32 / 1, 17.8 -> 14.3.  To the better form the choice loses 0.3 % on average, 26 % at most, on 60 batches that
// it was not fitted to 0.8 %, and 33 % at most (76 requests behind 837, 24 / 3).
static bool shared_whole(const SharedSizes& of, int32_t max_len, const SharedPlan& p) {
    const int32_t forced = forced_decode_plan();
    if ((int64_t)of.max_prefix + max_len > INT32_MAX) return false; // (a request's keys and tiles are counted in 32 bits)
    if (forced != 0) return forced == 2;
    const int64_t chunks = (of.Hq / of.Hkv + 31) / 32;
    if (of.B * (int64_t)of.Hkv * chunks > 256) return false;
    const double bytes = ((double)of.B * of.max_prefix + of.total_tokens) * of.Hkv * chunks * (4 * kHeadDim);
    const double whole = 6.75 + fmax(0.0065 * ((double)of.max_prefix + max_len), bytes / 9e6), ranges = 4.6 + 0.82 * p.us + 1.4 * p.kind;
    return whole < 0.97 * ranges;
}

int32_t query_decode_shared_plan(int32_t B, int32_t n_groups, int32_t prefix_total, int32_t max_prefix, int32_t max_group, int32_t total_tokens, int32_t max_len, int32_t Hq, int32_t Hkv) {
    const SharedSizes of = {B, n_groups, prefix_total, max_prefix, max_group, total_tokens, Hq, Hkv};
    if (of.alone()) return query_decode_plan(B, total_tokens, max_len, Hq, Hkv);
    const SharedPlan p = shared_plan(of);
    return shared_whole(of, max_len, p) ? 2 : p.waves;
}

// The order of the first launch.  Workgroups start in the order of their numbers as others end (on each XCD, and there on one shader engine after the other:
// one that is full holds up what comes behind).  What ends last should be short, and the prefix's workgroups are the long ones: so of those that start together as
// many are the prefix's as its share of the time, the rest follow evenly, and own rows alone fill the time that the last of the prefix take, and half as much
// again (their last ranges are short).  A prefix with few columns is bound by the memory as own rows are, nothing is gained side by side, and it comes first.
// Over 210 batches an even mixture takes 2.5 % more time, up to 63 % for one: 16 requests behind 65536 tokens, 32 / 32 heads, 245 us against 223; with eight wavefronts 1 + 110 + 12
// behind 12452, 947 and 28, 32 / 8, 71 against 56, and 96 + 100 + 60 behind 66, 40 and 20 thousand 442 against 418 (prefix first: 468 with four).  Up to 1.6 rounds of the chip it
// matters which ones the second gets, and evenly mixed is the better: 25 + 38 behind 16464 and 4705, 32 / 4, 48.6 against 53.1.  (Workgroups that take one piece of work after
// another by a counter: 416, and their loop costs others 4 % in the mean.)
static SharedWork shared_order(const SharedPlan& p, int64_t prefix, int64_t own) {
    SharedWork w = {(int32_t)prefix, (int32_t)own, (int32_t)p.units, (int32_t)p.blocks, 0, 0, 0};
    const int32_t P = w.prefix >> 3, N = w.own >> 3, all = P + N, round = 32 * (8 / p.waves);
    if (all <= kOneAfter * round) {
        w.first = w.mixed = all;
        w.first_prefix = P;
    } else if (p.kind <= 1) {
        w.first = w.first_prefix = w.mixed = P;
    } else {
        w.first = round;
        w.first_prefix = (int32_t)lround(round * p.share);
        if (w.first_prefix < round - N) w.first_prefix = round - N;
        if (w.first_prefix > P) w.first_prefix = P;
        w.mixed = all - (int32_t)(N * fmin(1.0, 1.5 * p.last));
        if (w.mixed < round + P - w.first_prefix) w.mixed = round + P - w.first_prefix;
    }
    return w;
}

esp_status launch_decode_shared(const SharedArgs& a, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const SharedSizes of = {a.B, a.n_groups, a.prefix_total, a.max_prefix, a.max_group, a.total_tokens, a.Hq, a.Hkv};
    if ((int64_t)a.B * a.Hq > INT32_MAX) return fail(ESP_ERR_INVALID_ARG, "decode (shared): too many rows for one launch");
    const size_t need = of.workspace();
    if (workspace_bytes < need) return fail(ESP_ERR_WORKSPACE, "decode (shared): workspace needs %zu bytes, got %zu", need, workspace_bytes);
    if (of.alone())                                                 // (on what that call asks for, so that the larger block changes nothing)
        return launch_decode(a.q, a.k_pool, a.v_pool, a.slot_idx, a.seq_offsets, a.B, a.total_tokens, a.max_len, a.Hq, a.Hkv, a.softmax_scale, a.O, a.LSE,
                             workspace, decode_workspace_bytes(a.B, a.total_tokens, a.Hq, a.Hkv), stream);
    const SharedPlan p = shared_plan(of);
    if (shared_whole(of, a.max_len, p)) {
        const int64_t chunks = (a.Hq / a.Hkv + 31) / 32;
        if (a.B > (int32_t)(UINT32_MAX / (kWholeWaves * 64)) || a.Hkv > 65535 || chunks > 65535)   // (only where a test asks for this form)
            return fail(ESP_ERR_UNSUPPORTED, "decode (shared): too many requests or heads for one launch of a workgroup each");
        hipLaunchKernelGGL(shared_whole_kernel, dim3(a.B, a.Hkv, (unsigned)chunks), dim3(kWholeWaves * 64), 0, stream, a, score_factor(a.softmax_scale));
        return check_launch("shared_whole_kernel");
    }
    const int32_t pairs = a.B * a.Hq;
    const int64_t prefix = (p.units + 7) / 8 * 8 * p.blocks, own = (p.own + 7) / 8 * 8;
    if (prefix + own > (int64_t)(UINT32_MAX / (p.waves * 64)) || p.units > INT32_MAX / 2)
        return fail(ESP_ERR_UNSUPPORTED, "decode (shared): too many heads, requests or groups for one launch");
    const int64_t rows = of.prefix_rows(p.range), own_rows = of.own_rows(p.own_range);
    float* const acc = (float*)workspace;
    const SharedParts parts = {acc, acc + rows * a.Hq * kHeadDim, p.range, p.each};
    float* const own_acc = (float*)((char*)workspace + of.bytes(rows));
    const SharedParts mine = {own_acc, own_acc + own_rows * a.Hq * kHeadDim, p.own_range, 0};
    const SharedWork work = shared_order(p, prefix, own);
    const dim3 grid((unsigned)(prefix + own)), block(p.waves * 64);
    if (p.waves == 8) hipLaunchKernelGGL(shared_partial_kernel<8>, grid, block, 0, stream, a, score_factor(a.softmax_scale), parts, mine, work);
    else hipLaunchKernelGGL(shared_partial_kernel<4>, grid, block, 0, stream, a, score_factor(a.softmax_scale), parts, mine, work);
    const esp_status st = check_launch("shared_partial_kernel");
    if (st != ESP_OK) return st;
    const int64_t most = (int64_t)a.max_prefix / p.range + a.max_len / p.own_range + 3;   // partials of a pair
#define ESP_COMBINE_LAUNCH(GROUPS)                                                                                                          \
    hipLaunchKernelGGL((shared_combine_kernel<GROUPS>), row_grid(((int64_t)pairs + 8 / GROUPS - 1) / (8 / GROUPS)), dim3(256), 0, stream, a, pairs, parts, mine)
    // A wavefront to a pair, which takes eight partials at a time, or a workgroup, which takes 32 and joins them through LDS: this where there are so many, or pairs
    // so few that a wavefront's rounds are all that the launch is.  On 210 batches that is 2 % less than a wavefront up to 64 partials (one request behind 14159
    // tokens beside three alone, 24 / 3 heads, 18.9 -> 15.2 us).
    if (most <= 8 || (most <= 64 && pairs > 2048)) ESP_COMBINE_LAUNCH(2);
    else ESP_COMBINE_LAUNCH(8);
#undef ESP_COMBINE_LAUNCH
    return check_launch("shared_combine_kernel");
}

}  // namespace esp
