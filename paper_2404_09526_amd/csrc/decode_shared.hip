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
    const int32_t rho0 = blockIdx.z * 32, n_rows = min(32, n_req * G - rho0);
    if (t0 >= t1 || n_rows <= 0) return;
    const int32_t seg = t1 - t0;
    const int32_t rho = rho0 + min(qi, n_rows - 1), of = rho / G;
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

// ranges of the prefix lists, and the partials' slots
static int32_t shared_range(int32_t prefix_total, int32_t max_group, int32_t Hq, int32_t Hkv) {
    const int64_t blocks = ((int64_t)max_group * (Hq / Hkv) + 31) / 32;
    return decode_range(prefix_total, kSharedWaves * 32, 1, Hkv * blocks, 1, 1 << 20);
}
static size_t shared_slots(int32_t n_groups, int32_t prefix_total, int32_t range) { return prefix_total > 0 ? (size_t)(prefix_total / range) + n_groups : 0; }
static size_t shared_prefix_bytes(int32_t n_groups, int32_t prefix_total, int32_t max_group, int32_t Hq, int32_t Hkv) {
    if (prefix_total <= 0) return 0;
    const size_t slots = shared_slots(n_groups, prefix_total, shared_range(prefix_total, max_group, Hq, Hkv));
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
        parts.range = shared_range(a.prefix_total, a.max_group, a.Hq, a.Hkv);
        const size_t slots = shared_slots(a.n_groups, a.prefix_total, parts.range);
        parts.ml = parts.acc + slots * a.max_group * a.Hq * kHeadDim;
        mine_at += shared_prefix_bytes(a.n_groups, a.prefix_total, a.max_group, a.Hq, a.Hkv);
        most = a.max_prefix / parts.range + 1;
        const int64_t blocks = ((int64_t)a.max_group * G + 31) / 32;
        if (a.Hkv > 65535 || blocks > 65535 || slots > UINT32_MAX / (kSharedWaves * 64)) return fail(ESP_ERR_UNSUPPORTED, "decode (shared): too many heads, requests or groups for one launch");
        hipLaunchKernelGGL(shared_prefix_kernel, dim3((unsigned)slots, a.Hkv, (unsigned)blocks), dim3(kSharedWaves * 64), 0, stream, a, a.softmax_scale * kLog2e, parts);
        const esp_status st = check_launch("shared_prefix_kernel");
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
