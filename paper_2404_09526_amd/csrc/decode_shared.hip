// esp_partial_attn_decode_shared: decode of a batch whose requests come in groups that share a long prefix (a system prompt, a document): every
// request's query attends the pool rows of its group's prefix and its own.  Read once per request, as the plain decode call does, the prefix is
// n times its bytes; here it is read once per group.  The queries of a group are packed rows, (request, query head of the group) pairs of a
// KV head, and the columns of MFMA tiles:
//   S^T [keys x columns] = K Q^T,   O^T [128 x columns] += V^T P^T
// against the prefix in ranges of keys, a partial (accumulator, maximum, sum) per (range, row); the requests' own rows are the plain
// decode's partials; one kernel combines both.
#include <math.h>

#include "column_tile.h"
#include "decode_merge.h"

namespace esp {

constexpr int kSharedWaves = 4;

struct SharedParts { float* acc; float* ml; int32_t range; };

__global__ __launch_bounds__(kSharedWaves * 64, 2) void shared_prefix_kernel(SharedArgs a, float scale_log2, SharedParts parts) {
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kSharedWaves * kColWaveBytes];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qi = lane & 31, hi = lane >> 5;
    const int kvh = blockIdx.y, G = a.Hq / a.Hkv;
    const RequestRange at = request_range(blockIdx.x, parts.range, a.n_groups, a.prefix_offsets, lane);
    const int32_t t0 = at.t0, t1 = min(at.t1, a.prefix_total);      // (never past the slot list)
    const int32_t b0 = a.group_offsets[at.b], n_req = min(min(a.group_offsets[at.b + 1], a.B) - b0, a.max_group);
    const int32_t n_rows = n_req * G;                                // at most 32 in every group
    if (t0 >= t1 || n_rows <= 0) return;
    const int32_t seg = t1 - t0;
    const int32_t rho = min(qi, n_rows - 1), of = rho / G;
    const int32_t row = of * a.Hq + kvh * G + (rho - of * G);         // within the group's queries

    const uint32_t row_bytes = (uint32_t)a.Hkv * (kHeadDim * 2);
    const char* kbase = a.k_pool + (uint32_t)kvh * (kHeadDim * 2);
    const char* vbase = a.v_pool + (uint32_t)kvh * (kHeadDim * 2);
    const uint32_t lds_k = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem + wave * kColWaveBytes, lds_v = lds_k + kColKBytes;

    bf16x8 qf[8];
    const uint16_t* qp = (const uint16_t*)a.q + ((int64_t)b0 * a.Hq + row) * kHeadDim + 8 * hi;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        uint4 raw = *(const uint4*)(qp + 16 * t);
        if (qi >= n_rows) raw = make_uint4(0u, 0u, 0u, 0u);
        qf[t] = __builtin_bit_cast(bf16x8, raw);
    }
    Columns cols;
    cols.place(lds_k, lane);
    cols.clear();
    auto tile_slots = [&](int i) { return a.prefix_slots[t0 + 32 * i + min(qi, min(32, seg - 32 * i) - 1)]; };
    int32_t slots = 32 * wave < seg ? tile_slots(wave) : 0;
    for (int i = wave; 32 * i < seg; i += kSharedWaves) {
        const int rows = min(32, seg - 32 * i);
        uint64_t row_at[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            row_at[n] = (uint64_t)(uint32_t)__shfl(slots, col_row(n, lane)) * row_bytes;
            load_to_lds_b128_at(lds_k + 1024 * n, kbase + (row_at[n] + col_k_within(n, lane)));
        }
#pragma unroll
        for (int n = 0; n < 8; ++n) load_to_lds_b128_at(lds_v + 1024 * n, vbase + (row_at[n] + col_v_within(lane)));
        int32_t slots_next = 0;
        if (32 * (i + kSharedWaves) < seg) slots_next = tile_slots(i + kSharedWaves);
        wait_vm<8>();                                               // K has landed; V and the next slots may be on their way
        floatx16 sc = cols.scores(qf);
        if (rows < 32) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + 4 * hi + (r & 3) >= rows) sc[r] = -INFINITY;
        }
        Columns::PFrag pf[2];
        cols.weigh(sc, scale_log2, pf);
        wait_vm<0>();
        asm volatile("" :: "v"(slots_next));
        cols.accumulate(pf);
        slots = slots_next;
    }
    float out[64 / kSharedWaves], mx, lsum;
    cols.combine<kSharedWaves>(smem, wave, lane, out, mx, lsum);
    if (qi >= n_rows) return;
    const int64_t ph = (int64_t)(at.w + at.b) * a.max_group * a.Hq + row;
    float* dst = parts.acc + ph * kHeadDim + Columns::first_element<kSharedWaves>(wave, lane);
#pragma unroll
    for (int e = 0; e < 64 / kSharedWaves; e += 4) *(float4*)(dst + 2 * e) = make_float4(out[e], out[e + 1], out[e + 2], out[e + 3]);
    if (wave == 0 && hi == 0) *(float2*)(parts.ml + ph * 2) = make_float2(mx, lsum);
}

// More columns than one tile has: a workgroup of eight wavefronts has COLS tiles of 32 of them, a wavefront one, and the COLS wavefronts that
// have different columns (a team) share tiles of 32 keys in LDS, so that a row of K and V comes from memory once for 32 COLS columns; the 8 / COLS
// teams take the tiles in turn.  All teams' tiles are a step; COLS steps are on their way or at work (128 KiB of LDS in every form), and one
// barrier a step says both that its tiles are there and that the stage of the step before may be filled again.
constexpr int kWideWaves = 8;
constexpr int kWideTile = kColKBytes + kColVBytes;
constexpr int kWideMost = 4096;                                     // keys of a range: its slots lie in LDS

template <int COLS>
__global__ __launch_bounds__(kWideWaves * 64, 2) void shared_wide_kernel(SharedArgs a, float scale_log2, SharedParts parts, int32_t units, int32_t col_blocks) {
    constexpr int TEAMS = kWideWaves / COLS, STAGES = COLS, STEP = 32 * TEAMS, MOVES = 8 / COLS;   // MOVES: transfers of K, and of V, of a wavefront a step
    constexpr int kRing = STAGES * TEAMS * kWideTile, kLds = kRing + kWideMost * 4;
    static_assert(kRing + 1 >= 128 * 1024 && kWideWaves * kColWaveBytes <= kLds, "the blocks of the combination fit");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kLds];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int team = wave / COLS, ct = wave % COLS;
    const int qi = lane & 31, hi = lane >> 5;
    // unit: (range, KV head), heads next to each other as in a pool row.  The column blocks of a unit are eight workgroups apart: on one XCD, whose
    // L2 then has the rows.
    const uint32_t all = blockIdx.x, eight = all / (8u * col_blocks), rest = all - eight * (8u * col_blocks);
    const uint32_t unit = eight * 8 + (rest & 7), cb = rest >> 3;
    if (unit >= (uint32_t)units) return;
    const int kvh = unit % (uint32_t)a.Hkv, G = a.Hq / a.Hkv;
    const RequestRange at = request_range(unit / (uint32_t)a.Hkv, parts.range, a.n_groups, a.prefix_offsets, lane);
    const int32_t t0 = at.t0, t1 = min(at.t1, a.prefix_total);      // (never past the slot list)
    const int32_t b0 = a.group_offsets[at.b], n_req = min(min(a.group_offsets[at.b + 1], a.B) - b0, a.max_group);
    const int32_t seg = t1 - t0;
    if (seg <= 0 || n_req * G <= (int32_t)cb * (32 * COLS)) return;
    const int32_t rho0 = cb * (32 * COLS) + ct * 32, n_rows = min(32, n_req * G - rho0);   // (columns of this wavefront; none: it only moves tiles)

    int32_t* const list = (int32_t*)(smem + kRing);
    for (int i = threadIdx.x; i < seg; i += kWideWaves * 64) list[i] = a.prefix_slots[t0 + i];

    const int32_t rho = rho0 + max(min(qi, n_rows - 1), 0), rho_in = min(rho, n_req * G - 1), of = rho_in / G;
    const int32_t row = of * a.Hq + kvh * G + (rho_in - of * G);      // within the group's queries
    bf16x8 qf[8];
    const uint16_t* qp = (const uint16_t*)a.q + ((int64_t)b0 * a.Hq + row) * kHeadDim + 8 * hi;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        uint4 raw = *(const uint4*)(qp + 16 * t);
        if (qi >= n_rows) raw = make_uint4(0u, 0u, 0u, 0u);
        qf[t] = __builtin_bit_cast(bf16x8, raw);
    }
    asm volatile("" :: "v"(qf[0]), "v"(qf[1]), "v"(qf[2]), "v"(qf[3]), "v"(qf[4]), "v"(qf[5]), "v"(qf[6]), "v"(qf[7]));   // here before the transfers, whose waits count
    __syncthreads();

    const uint32_t row_bytes = (uint32_t)a.Hkv * (kHeadDim * 2);
    const char* kbase = a.k_pool + (uint32_t)kvh * (kHeadDim * 2);
    const char* vbase = a.v_pool + (uint32_t)kvh * (kHeadDim * 2);
    const uint32_t lds = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem;
    const int steps = (seg + STEP - 1) / STEP;
    auto fetch = [&](int i) {
        const uint32_t to = lds + ((i % STAGES) * TEAMS + team) * kWideTile;
        uint64_t row_at[MOVES];
#pragma unroll
        for (int x = 0; x < MOVES; ++x) {
            const int n = ct + COLS * x;
            row_at[x] = (uint64_t)(uint32_t)list[min(i * STEP + team * 32 + col_row(n, lane), seg - 1)] * row_bytes;
            load_to_lds_b128_at(to + 1024 * n, kbase + (row_at[x] + col_k_within(n, lane)));
        }
#pragma unroll
        for (int x = 0; x < MOVES; ++x) {
            const int n = ct + COLS * x;
            load_to_lds_b128_at(to + kColKBytes + 1024 * n, vbase + (row_at[x] + col_v_within(lane)));
        }
    };
    // the transfers of step i have landed: those of up to STAGES - 2 steps after it may be on their way
    auto landed = [&](int i) {
        const int after = min(steps - 1 - i, STAGES - 2);
        if (after <= 0) wait_vm<0>();
        else if (after == 1) wait_vm<2 * MOVES>();
        else if (after == 2) wait_vm<4 * MOVES>();
        else if (after == 3) wait_vm<6 * MOVES>();
        else if (after == 4) wait_vm<8 * MOVES>();
        else if (after == 5) wait_vm<10 * MOVES>();
        else wait_vm<12 * MOVES>();
    };
    for (int i = 0; i < STAGES - 1 && i < steps; ++i) fetch(i);

    Columns cols;
    cols.clear();
    for (int i = 0; i < steps; ++i) {
        landed(i);
        wg_barrier();
        if (i + STAGES - 1 < steps) fetch(i + STAGES - 1);
        const int here = seg - i * STEP - team * 32;                // keys of this tile
        if (n_rows <= 0 || here <= 0) continue;
        cols.place(lds + ((i % STAGES) * TEAMS + team) * kWideTile, lane);
        floatx16 sc = cols.scores(qf);
        if (here < 32) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + 4 * hi + (r & 3) >= here) sc[r] = -INFINITY;
        }
        Columns::PFrag pf[2];
        cols.weigh(sc, scale_log2, pf);
        cols.accumulate(pf);
    }
    float out[64 / TEAMS], mx, lsum;
    __syncthreads();                                                // the ring is read: it may hold the teams' results
    cols.combine<TEAMS, COLS>(smem + ct * kColWaveBytes, team, lane, out, mx, lsum);
    if (qi >= n_rows) return;
    const int64_t ph = (int64_t)(at.w + at.b) * a.max_group * a.Hq + row;
    float* dst = parts.acc + ph * kHeadDim + Columns::first_element<TEAMS>(team, lane);
#pragma unroll
    for (int e = 0; e < 64 / TEAMS; e += 4) *(float4*)(dst + 2 * e) = make_float4(out[e], out[e + 1], out[e + 2], out[e + 3]);
    if (team == 0 && hi == 0) *(float2*)(parts.ml + ph * 2) = make_float2(mx, lsum);
}

// Combination, as the plain decode's (decode.hip): groups of 32 lanes take a pair's partials in turn, four at a time, first those of the
// prefix, then its own.
template <int GROUPS>
__global__ __launch_bounds__(256) void shared_combine_kernel(SharedArgs a, int32_t pairs, SharedParts parts, DecodePartials mine) {
    constexpr int U = 4;
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int64_t at = row_block() * (8 / GROUPS) + grp / GROUPS;
    if (at >= pairs) return;                                        // (a whole workgroup, or a pair is a wavefront and no barrier follows)
    const int pair = (int)at, g = grp % GROUPS;
    const int b = pair / a.Hq, h = pair - b * a.Hq;
    const int32_t s0 = a.seq_offsets[b], s1 = a.seq_offsets[b + 1];
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
    if (a.prefix_total > 0) {
        const RequestAt in = request_of(b, a.group_offsets, a.n_groups, threadIdx.x & 63);
        const int32_t b0 = a.group_offsets[in.b], p0 = a.prefix_offsets[in.b], p1 = min(a.prefix_offsets[in.b + 1], a.prefix_total);
        if (b >= b0 && b < in.end && b - b0 < a.max_group && p1 > p0) {
            const int64_t rows = (int64_t)a.max_group * a.Hq;
            add(parts.acc, parts.ml, (int64_t)(p0 / parts.range + in.b) * rows + (int64_t)(b - b0) * a.Hq + h, rows, (p1 - p0 - 1) / parts.range + 1);
        }
    }
    if (s1 > s0) add(mine.acc, mine.ml, ((int64_t)(s0 / mine.range) + b) * a.Hq + h, a.Hq, own_partials(s0, s1, mine.range, mine.parts));

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

// Ranges of the prefix lists, which kernel has them, and the partials' slots.
struct SharedPlan { int32_t cols, range; };                         // cols: column tiles of a workgroup; 1: the kernel for one
static SharedPlan shared_plan(int32_t prefix_total, int32_t max_group, int32_t Hq, int32_t Hkv) {
    const int64_t rows = (int64_t)max_group * (Hq / Hkv);
    if (rows <= 32) return {1, decode_range(prefix_total, kSharedWaves * 32, 1, Hkv, 1, 1 << 20)};
    const int32_t cols = rows <= 64 ? 2 : rows <= 128 ? 4 : 8, step = 32 * (kWideWaves / cols);
    // One workgroup a CU.  Of the ranges that fill 1 .. 16 rounds of them the one whose rounds, each with a start, an end (its partial, written and
    // read) and its steps, take the least time.
    constexpr int64_t kResident = 256;
    const double start = 6 + 0.04 * 32 * cols, per_step = 0.63 * (kWideWaves / cols);
    const int64_t steps = ((int64_t)prefix_total + step - 1) / step, units = Hkv * ((rows + 32 * cols - 1) / (32 * cols));
    int64_t best = 1;
    double best_us = 0;
    for (int64_t rounds = 1; rounds <= 16; ++rounds) {
        const int64_t fit = rounds * kResident / units;
        int64_t take = fit > 0 ? (steps + fit - 1) / fit : steps;
        if (take > kWideMost / step) take = kWideMost / step;
        const int64_t wgs = (steps + take - 1) / take * units;
        const double us = (double)((wgs + kResident - 1) / kResident) * (start + per_step * (double)take);
        if (rounds == 1 || us < best_us) { best = take; best_us = us; }
    }
    return {cols, (int32_t)(best * step)};
}
static size_t shared_slots(int32_t n_groups, int32_t prefix_total, int32_t range) { return prefix_total > 0 ? (size_t)(prefix_total / range) + n_groups : 0; }
static size_t shared_prefix_bytes(int32_t n_groups, int32_t prefix_total, int32_t max_group, int32_t Hq, int32_t Hkv) {
    if (prefix_total <= 0) return 0;
    const size_t slots = shared_slots(n_groups, prefix_total, shared_plan(prefix_total, max_group, Hq, Hkv).range);
    return (slots * max_group * Hq * (kHeadDim + 2) * sizeof(float) + 255) / 256 * 256;
}
size_t decode_shared_workspace_bytes(int32_t B, int32_t n_groups, int32_t prefix_total, int32_t max_prefix, int32_t max_group, int32_t total_tokens,
                                     int32_t Hq, int32_t Hkv) {
    (void)max_prefix;
    return shared_prefix_bytes(n_groups, prefix_total, max_group, Hq, Hkv) + decode_workspace_bytes(B, total_tokens, Hq, Hkv);
}

esp_status launch_decode_shared(const SharedArgs& a, void* workspace, hipStream_t stream) {
    if ((int64_t)a.B * a.Hq > INT32_MAX) return fail(ESP_ERR_INVALID_ARG, "decode (shared): too many rows for one launch");
    const int32_t pairs = a.B * a.Hq, G = a.Hq / a.Hkv;
    SharedParts parts = {(float*)workspace, nullptr, 1};
    char* mine_at = (char*)workspace;
    int64_t most = 0;                                               // partials of a pair
    if (a.prefix_total > 0 && a.max_group > 0) {
        const SharedPlan plan = shared_plan(a.prefix_total, a.max_group, a.Hq, a.Hkv);
        parts.range = plan.range;
        const size_t slots = shared_slots(a.n_groups, a.prefix_total, parts.range);
        parts.ml = parts.acc + slots * a.max_group * a.Hq * kHeadDim;
        mine_at += shared_prefix_bytes(a.n_groups, a.prefix_total, a.max_group, a.Hq, a.Hkv);
        most = a.max_prefix / parts.range + 1;
        const int64_t tiles = ((int64_t)a.max_group * G + 31) / 32, blocks = (tiles + plan.cols - 1) / plan.cols, units = (int64_t)slots * a.Hkv;
        if (a.Hkv > 65535 || blocks * ((units + 7) / 8 * 8) > UINT32_MAX / (kWideWaves * 64))
            return fail(ESP_ERR_UNSUPPORTED, "decode (shared): too many heads, requests or groups for one launch");
        const float sl2 = a.softmax_scale * kLog2e;
#define ESP_WIDE_LAUNCH(COLS)                                                                                                               \
    hipLaunchKernelGGL(shared_wide_kernel<COLS>, dim3((unsigned)((units + 7) / 8 * 8 * blocks)), dim3(kWideWaves * 64), 0, stream, a, sl2, parts, \
                       (int32_t)units, (int32_t)blocks)
        if (plan.cols == 1) hipLaunchKernelGGL(shared_prefix_kernel, dim3((unsigned)slots, a.Hkv), dim3(kSharedWaves * 64), 0, stream, a, sl2, parts);
        else if (plan.cols == 2) ESP_WIDE_LAUNCH(2);
        else if (plan.cols == 4) ESP_WIDE_LAUNCH(4);
        else ESP_WIDE_LAUNCH(8);
#undef ESP_WIDE_LAUNCH
        const esp_status st = check_launch(plan.cols == 1 ? "shared_prefix_kernel" : "shared_wide_kernel");
        if (st != ESP_OK) return st;
    }
    DecodePartials mine;
    const esp_status st = launch_decode_partials(a.q, a.k_pool, a.v_pool, a.slot_idx, a.seq_offsets, a.B, a.total_tokens, a.max_len, a.Hq, a.Hkv,
                                                 a.softmax_scale, mine_at, decode_workspace_bytes(a.B, a.total_tokens, a.Hq, a.Hkv), stream, &mine);
    if (st != ESP_OK) return st;
    most += a.max_len / mine.range + 2;
#define ESP_COMBINE_LAUNCH(GROUPS)                                                                                                          \
    hipLaunchKernelGGL((shared_combine_kernel<GROUPS>), row_grid(((int64_t)pairs + 8 / GROUPS - 1) / (8 / GROUPS)), dim3(256), 0, stream, a, pairs, parts, mine)
    if (most <= 32) ESP_COMBINE_LAUNCH(2);
    else ESP_COMBINE_LAUNCH(8);
#undef ESP_COMBINE_LAUNCH
    return check_launch("shared_combine_kernel");
}

}  // namespace esp
