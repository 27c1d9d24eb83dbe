// esp_partial_attn_decode_q4: one query token per request against rows of the pool in 4 bits.  Bound by the memory: a key-value head of a token is 136
// bytes, 256 CUs have 13 cycles for it.
//
// A wavefront has a KV head and tiles of 32 of its tokens; a workgroup has the heads of a whole row (up to eight; fewer heads: several wavefronts to a
// head, tiles in turn), so a random slot is one burst.  The query heads of the KV head are the columns of the products (16, or NC = 2 times 16):
//   S^T [32 keys x 16] = K [32 x 128] Q^T [128 x 16],   O^T [128 x 16] += V^T [128 x 32] P^T [32 x 16].
// Codes and scales go from memory to the LDS by themselves, a step ahead, and where rows are pieces of 16 bytes a row by neighbouring lanes: lanes that
// each load a row of their own, as the operands have them, kept the address unit busy all the time (97 cycles an instruction; 128 requests of 512 .. 1M
// tokens, 32 / 8 heads, 1570 us; four lanes to a head of a token 1310, whole rows 645: 3.94 GB of rows at 6.1 TB/s, in 4.19 GB of lines of 128 bytes,
// 6.6 TB/s.  A second step on its way: 658).  Codes become bf16 with their scales on the way from the LDS to the products, exactly.
//   K: a lane has four bytes of each block of a key, eight elements, which are a step of the contraction: operands without a turn.
//   V: its products need neighbouring keys in a register and codes are neighbours along a key.  A lane takes eight elements of each of eight keys, and
//   the halves of converted pairs are put together: element 8 c + d of column d of the lanes c makes up the rows of product d.  No turn through the LDS.
// Values in 4 bits are exact in bf16; the weights are rounded to bf16 for the second product, as in the other decode kernels, and the sum they are
// divided by is that of the rounded ones.
//
// What the weights are taken against follows the scores only when weights get large: any reference serves.  It is set to 2^11 times the largest weight
// so far, and again when a lane's eight weights pass 1 in sum, which leaves out the maximum of nearly every tile.  No weight is above 1, then, as if
// each tile's maximum were taken: a row that is much heavier than those before it does not pass the range of fp32, whatever finite values it has.
// (Against the largest weight itself, and up to 2048 times it, rows above 2^116 came out infinite.)  What the weights lose at the other end is far
// below what fp32 and bf16 hold.
#include <math.h>

#include "decode_merge.h"
#include "mfma_tile.h"
#include "q4.h"

namespace esp {

constexpr int kQ4Waves = 8;                        // wavefronts of a workgroup, at most
constexpr int kQ4Tile = 32;                        // tokens that a wavefront works on at a time
constexpr int kQ4MaxRanges = 1024;
constexpr float kQ4Above = 11.f;                   // the reference's logarithm over the largest score's, when it is set
constexpr float kQ4Most = 1.f;                     // of a lane's eight weights, before it is set again

struct Q4Geom {
    int32_t hw, nt;         // heads of a workgroup, wavefronts to each
    int32_t hgroups;        // workgroups to a row
    int32_t tiles, chunks;  // columns: tiles of 16 in a workgroup (1 or 2), workgroups to a KV head
    int32_t range, nwg, parts;
};

// What a wavefront keeps of its columns and does with a tile.
template <int NC>
struct Q4Columns {
    floatx4 oacc[NC][8];
    float m[NC], l[NC], l_r[NC];      // reference of this column's scaled scores; this lane's sums of the weights, as computed and as rounded to bf16
    bf16x8 qf[NC][4];
    union PFrag { uint32_t u[4]; bf16x8 v; };

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            m[c] = -INFINITY; l[c] = l_r[c] = 0.f;
#pragma unroll
            for (int d = 0; d < 8; ++d) oacc[c][d] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // Q^T: column l16 of a tile is row l16 of q (past ng: zeros), of each block of 32 elements the eight that a lane has of a key's
    __device__ __forceinline__ void load_queries(const uint16_t* q, int ng, int l16, int g) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = 16 * c + l16;
            const uint4* qp = (const uint4*)(q + (col < ng ? col : 0) * kHeadDim + 8 * g);
#pragma unroll
            for (int s = 0; s < 4; ++s) qf[c][s] = __builtin_bit_cast(bf16x8, col < ng ? qp[4 * s] : make_uint4(0u, 0u, 0u, 0u));
        }
    }
    __device__ __forceinline__ void queries_are_here() const {       // (waited for here, not among the transfers)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int s = 0; s < 4; ++s) asm volatile("" :: "v"(qf[c][s]));
    }
    // codes[u][s]: of block s of key l16 + 16 u, the lane's eight elements; scales[u]: that key's.  Register r of half u: key 4 g + r + 16 u.
    __device__ __forceinline__ void scores(const uint32_t (&codes)[2][4], const uint32_t (&scales)[2], floatx4 (&sc)[NC][2]) const {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int c = 0; c < NC; ++c) sc[c][u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const bf16x8 kf = __builtin_bit_cast(bf16x8, q4_to_bf16(codes[u][s], q4_scale(scales[u], s)));
#pragma unroll
                for (int c = 0; c < NC; ++c) sc[c][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c][s], sc[c][u], 0, 0, 0);
            }
        }
    }
    // Of a tile's keys the first `left` count; the ones past them are the last one again.  V's codes (vw as below) become zeros there, as 0 times an
    // infinity, of a scale of 2^126 or 2^127, is not 0.  (A NaN among its scales shows in the result by the last key itself.)
    static __device__ __forceinline__ void hide(uint32_t (&vw)[2][4], int left, int g) {
        if (left >= kQ4Tile) return;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * u + r >= left - 4 * g) vw[u][r] = 0;
    }
    // their scores to weights, in bf16
    __device__ __forceinline__ void weigh(floatx4 (&sc)[NC][2], int left, int g, float scale_log2, PFrag (&pf)[NC]) {
        if (left < kQ4Tile) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * u + r >= left - 4 * g)
#pragma unroll
                        for (int c = 0; c < NC; ++c) sc[c][u][r] = -INFINITY;
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float p[2][4], sum = weights(sc[c], scale_log2, m[c], p);
            if (__builtin_amdgcn_ballot_w64(!(sum <= kQ4Most)) != 0) {   // (none taken so far: m is -inf, and the sum infinite or NaN)
                float top = fmaxf(fmaxf(sc[c][0][0], sc[c][0][1]), fmaxf(sc[c][0][2], sc[c][0][3]));
                top = fmaxf(top, fmaxf(fmaxf(sc[c][1][0], sc[c][1][1]), fmaxf(sc[c][1][2], sc[c][1][3]))) * scale_log2;
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float m_new = fmaxf(m[c], top + kQ4Above);
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[c] - m_new);
                m[c] = m_new;
                l[c] *= alpha; l_r[c] *= alpha;
#pragma unroll
                for (int d = 0; d < 8; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) oacc[c][d][r] *= alpha;
                sum = weights(sc[c], scale_log2, finite_offset(m_new), p);
            }
            l[c] += sum;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t pk = pack_bf16(p[x >> 1][2 * (x & 1)], p[x >> 1][2 * (x & 1) + 1]);
                l_r[c] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), __builtin_bit_cast(bf16x2, 0x3f803f80u), l_r[c], false);
                pf[c].u[x] = pk;
            }
        }
    }
    static __device__ __forceinline__ float weights(const floatx4 (&sc)[2], float scale_log2, float from, float (&p)[2][4]) {
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[u][r] = __builtin_amdgcn_exp2f(fmaf(sc[u][r], scale_log2, -from));
                sum = u + r == 0 ? p[u][r] : sum + p[u][r];
            }
        return sum;
    }
    // vw[u][r]: codes of elements 8 l16 .. 8 l16 + 7 of key 4 g + r + 16 u, vs that key's scales, of which the lane's block is number `block`
    __device__ __forceinline__ void accumulate(const uint32_t (&vw)[2][4], const uint32_t (&vs)[2][4], int block, const PFrag (&pf)[NC]) {
        accumulate_pairs<0>(vw, vs, block, pf);
        accumulate_pairs<1>(vw, vs, block, pf);
        accumulate_pairs<2>(vw, vs, block, pf);
        accumulate_pairs<3>(vw, vs, block, pf);
    }
    template <int P>
    __device__ __forceinline__ void accumulate_pairs(const uint32_t (&vw)[2][4], const uint32_t (&vs)[2][4], int block, const PFrag (&pf)[NC]) {
        PFrag even, odd;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int u = x >> 1, r = 2 * (x & 1);
            const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vw[u][r], q4_scale(vs[u][r], block), P));
            const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vw[u][r + 1], q4_scale(vs[u][r + 1], block), P));
            even.u[x] = __builtin_amdgcn_perm(b, a, 0x05040100u);
            odd.u[x] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            oacc[c][2 * P] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even.v, pf[c].v, oacc[c][2 * P], 0, 0, 0);
            oacc[c][2 * P + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd.v, pf[c].v, oacc[c][2 * P + 1], 0, 0, 0);
        }
    }

    // The nt wavefronts of a head (this is number tsub; number u's block of 8 KiB is at blocks + (u - 1) * pitch, its row of s_ml u * apart on) combine
    // their results, a column tile at a time, and one partial leaves for each head, or the result where it is the only one.
    __device__ __forceinline__ void finish(int tsub, int nt, unsigned char* blocks, int pitch, float2 (*s_ml)[16], int apart, int ng, int l16, int g, int lane, bool whole,
                                           int64_t at, float* part_acc, float* part_ml, U32x2* O, float* LSE) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float lt = l[c] + __shfl_xor(l[c], 16), lr = l_r[c] + __shfl_xor(l_r[c], 16);
            lt += __shfl_xor(lt, 32);
            lr += __shfl_xor(lr, 32);
            const float fix = lr > 0.f ? lt / lr : 0.f;             // (a NaN among the weights is in oacc, too)
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) oacc[c][d][r] *= fix;
            float mx = m[c], lsum = lt;
            if (nt > 1) {
                if (tsub > 0) {
                    floatx4* mine = (floatx4*)(blocks + (tsub - 1) * pitch);
#pragma unroll
                    for (int d = 0; d < 8; ++d) mine[d * 64 + lane] = oacc[c][d];
                    if (g == 0) s_ml[tsub * apart][l16] = make_float2(mx, lt);
                }
                __syncthreads();
                if (tsub == 0) {
                    for (int u = 1; u < nt; ++u) mx = fmaxf(mx, s_ml[u * apart][l16].x);
                    const float ref = finite_offset(mx);
                    const float own = lt != 0.f ? __builtin_amdgcn_exp2f(m[c] - ref) : 0.f;   // no key seen (a sum of 0): nothing to add
                    lsum = lt * own;
#pragma unroll
                    for (int d = 0; d < 8; ++d)
#pragma unroll
                        for (int r = 0; r < 4; ++r) oacc[c][d][r] *= own;
                    for (int u = 1; u < nt; ++u) {
                        const float2 ml = s_ml[u * apart][l16];
                        const float share = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - ref) : 0.f;
                        lsum += ml.y * share;
                        const floatx4* from = (const floatx4*)(blocks + (u - 1) * pitch);
#pragma unroll
                        for (int d = 0; d < 8; ++d) {
                            const floatx4 x = from[d * 64 + lane];
#pragma unroll
                            for (int r = 0; r < 4; ++r) oacc[c][d][r] += x[r] * share;
                        }
                    }
                }
                __syncthreads();
            }
            const int col = 16 * c + l16;
            if (tsub != 0 || col >= ng) continue;
            const int64_t ph = at + col;
            // element 8 (4 g + r) + d of the column is register r of product d
            if (whole) {
                const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int d = 0; d < 8; d += 4)
                        O[ph * (kHeadDim / 4) + 2 * (4 * g + r) + (d >> 2)] = U32x2{pack_bf16(oacc[c][d][r] * inv, oacc[c][d + 1][r] * inv),
                                                                                   pack_bf16(oacc[c][d + 2][r] * inv, oacc[c][d + 3][r] * inv)};
                if (g == 0) LSE[ph] = lsum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(lsum)) * kLn2;
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int d = 0; d < 8; d += 4)
                        ((floatx4*)(part_acc + ph * kHeadDim))[2 * (4 * g + r) + (d >> 2)] = floatx4{oacc[c][d][r], oacc[c][d + 1][r], oacc[c][d + 2][r], oacc[c][d + 3][r]};
                if (g == 0) *(float2*)(part_ml + ph * 2) = make_float2(mx, lsum);
            }
        }
    }
};

// Range i of those that the requests have, counted from each one's first token on: the whole ones of all requests first, then what is left of each.  A
// lane looks at K consecutive requests, all at once, then the lanes at those of the lane that has it: two round trips for up to 4096 requests
// (request_range takes two for each 64, twice over: 64 requests of 1024 .. 131072, 32 / 1 heads, 55 us in ranges along the list, which cross up to four
// requests).
constexpr int32_t kQ4MostByRequest = 4096;
__device__ __forceinline__ int32_t wave_scan(int32_t x, int lane) {   // sum up to this lane's
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t below = __shfl_up(x, d);
        if (lane >= d) x += below;
    }
    return x;
}
__device__ __forceinline__ RequestRange q4_request_range(int32_t i, int32_t range, int32_t B, const int32_t* seq_offsets, int lane) {
    const int K = (B + 63) >> 6;
    int32_t whole = 0, rest = 0, s0 = seq_offsets[min(lane * K, B)];
#pragma unroll 4
    for (int k = 0; k < K; ++k) {
        const int32_t s1 = seq_offsets[min(lane * K + k + 1, B)], n = (s1 - s0) / range;
        whole += n;
        rest += s1 - s0 > n * range;
        s0 = s1;
    }
    int32_t upto_whole = wave_scan(whole, lane), upto_rest = wave_scan(rest, lane);
    const int32_t wholes = __builtin_amdgcn_readlane(upto_whole, 63);
    const bool of_rest = i >= wholes;
    if (of_rest) i -= wholes;
    uint64_t hit = __builtin_amdgcn_ballot_w64((of_rest ? upto_rest : upto_whole) > i);
    if (!hit) return {0, 0, 0, 0};                                  // the launch is an upper bound
    const int l = __builtin_ctzll(hit);
    i -= of_rest ? __builtin_amdgcn_readlane(upto_rest - rest, l) : __builtin_amdgcn_readlane(upto_whole - whole, l);
    const int first = l * K, b = min(first + lane, B - 1);
    const int32_t from = seq_offsets[b], to = seq_offsets[b + 1], n = (to - from) / range;
    const int32_t mine = lane >= K || first + lane >= B ? 0 : of_rest ? (to - from > n * range ? 1 : 0) : n, upto = wave_scan(mine, lane);
    hit = __builtin_amdgcn_ballot_w64(upto > i);
    const int at = hit ? __builtin_ctzll(hit) : 0;
    const int32_t start = __builtin_amdgcn_readlane(from, at), end = __builtin_amdgcn_readlane(to, at);
    const int32_t part = of_rest ? __builtin_amdgcn_readlane(n, at) : i - __builtin_amdgcn_readlane(upto - mine, at);
    const int32_t t0 = start + part * range;
    return {first + at, t0, t0 + min(range, end - t0), start / range + part};
}

// A workgroup's way along the token list: what it works on, request after request.  parts == 1: each request whole; > 1: so many ranges of each; < 0:
// as many as each has; 0: ranges along the list.
struct Q4Walk {
    int b;
    int32_t t0, t1, req_end, w;
    bool first;
    __device__ __forceinline__ bool start(int32_t range, int32_t parts, int32_t B, int32_t total_tokens, const int32_t* seq_offsets, int lane) {
        first = true;
        w = blockIdx.x;
        if (parts != 0) {
            const RequestRange at = parts > 0 ? request_part(w, parts, range, B, seq_offsets) : q4_request_range(w, range, B, seq_offsets, lane);
            b = at.b; t0 = at.t0; t1 = req_end = min(at.t1, total_tokens); w = at.w;
            return t0 < t1 || parts == 1;                           // (a request without tokens, in one part: its result is nothing)
        }
        t0 = w * range;
        t1 = t0 + min(range, total_tokens - t0);
        if (t0 >= t1) return false;
        const RequestAt at = request_of(t0, seq_offsets, B, lane);
        b = at.b; req_end = at.end;
        return true;
    }
    // the next request's tokens t0 .. t0 + seg - 1, or false
    __device__ __forceinline__ bool next(int32_t parts, int32_t B, const int32_t* seq_offsets, uint32_t& seg) {
        if (parts != 0) {
            if (!first) return false;
            first = false;
            seg = (uint32_t)max(t1 - t0, 0);
            return true;
        }
        while (t0 < t1 && b < B) {                                  // (tokens past the offsets' end belong to no request)
            if (!first) req_end = seq_offsets[b + 1];
            first = false;
            if (req_end > t0) { seg = (uint32_t)(min(t1, req_end) - t0); return true; }
            ++b;                                                    // empty request, or the last one where the range starts past its end
        }
        return false;
    }
    __device__ __forceinline__ void done(uint32_t seg) { t0 += (int32_t)seg; ++b; }
};

// Rows of four or eight heads (HW: the workgroup's), which are pieces of 16 bytes: every wavefront brings whole rows, K's and V's, for all of them, and
// reads what it needs of the others'.  Nothing is brought past the last step: 64 requests of 32 .. 4096 tokens, 32 / 8 heads, 3 or 4 steps to a
// workgroup, 22.5 against 23.0 us.  Loads go past the caches, but for PART: rows of four heads that are part of a slot's, of which neighbouring
// workgroups have a good deal of their lines of memory in common (82 requests of 4350 or so, 12 / 12 heads, 210 us, past the caches 220; of eight heads
// 667 and 662, 32 / 32 heads; whole rows of four 340 and 318, of eight 811 and 755).
template <int HW, int NC, bool PART>
__global__ __launch_bounds__(kQ4Waves * 64, NC == 1 ? 4 : 2) void decode_q4_rows_kernel(
    const uint16_t* __restrict__ q, const char* __restrict__ k_pool, const char* __restrict__ v_pool, const int32_t* __restrict__ slot_idx,
    const int32_t* __restrict__ seq_offsets, int32_t B, int32_t total_tokens, int32_t range, int32_t parts, uint32_t slot_bytes, int32_t Hq, int32_t Hkv,
    float scale_log2, float* __restrict__ part_acc, float* __restrict__ part_ml, U32x2* __restrict__ O, float* __restrict__ LSE) {
    constexpr int NT = kQ4Waves / HW, kStep = NT * kQ4Tile, kRow = HW * kQ4Head, kPieces = 34, kOwn = kStep / kQ4Waves;
    // a token's rows in the LDS, and 16 bytes that put 16 tokens' words into different banks
    constexpr int kPitch = 2 * kRow + 16, kStage = kStep * kPitch;
    static_assert(kPitch / 4 % 8 == 4, "");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kStage > (NT - 1) * HW * 8192 ? kStage : (NT - 1) * HW * 8192];
    __shared__ float2 s_ml[kQ4Waves][16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int tsub = wave / HW, hl = wave % HW;
    const int G = Hq / Hkv, g0 = blockIdx.z * (16 * NC), ng = min(16 * NC, G - g0);
    const int h0 = (blockIdx.y * HW + hl) * G + g0;
    const uint32_t lds = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem;
    const char* const kbase = k_pool + (int64_t)blockIdx.y * kRow;
    const char* const vbase = v_pool + (int64_t)blockIdx.y * kRow;
    // a lane's 16 bytes of the rows that the wavefront brings: eight transfers, of K's and V's row of four tokens, or of both rows (17 lanes each) of eight
    const char* const src = lane < 17 ? kbase + 16 * lane : vbase + 16 * (lane - 17);   // (HW = 4)
    const uint32_t dst = lds + wave * kOwn * kPitch;
    // what it reads: key l16 (and l16 + 16) for the first product, keys 4 g .. 4 g + 3 (and 16 more) for the second
    const uint32_t mine = lds + tsub * kQ4Tile * kPitch + hl * kQ4Head;
    const uint32_t k_rd = mine + l16 * kPitch + 4 * g, ks_rd = mine + l16 * kPitch + kQ4Codes, v_rd = mine + kRow + 4 * g * kPitch + 4 * l16,
                   vs_rd = mine + kRow + 4 * g * kPitch + kQ4Codes;

    Q4Walk at;
    if (!at.start(range, parts, B, total_tokens, seq_offsets, lane)) return;
    uint32_t seg;
    while (at.next(parts, B, seq_offsets, seg)) {
        Q4Columns<NC> cols;
        cols.clear();
        if (seg > 0) {
            const int32_t* const list = slot_idx + at.t0;
            const uint32_t steps = (seg + kStep - 1) / kStep;
            struct Slots { uint32_t s[kOwn]; };
            auto slots_of = [&](uint32_t j) {                       // past the last token: its slot again, hidden below
                Slots r;
#pragma unroll
                for (int i = 0; i < kOwn; ++i) r.s[i] = (uint32_t)list[min(j * kStep + wave * kOwn + i, seg - 1)];
                return r;
            };
            auto bring = [&](const Slots& sl) {
                if (lane < kPieces) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint64_t row = (uint64_t)sl.s[HW == 8 ? i >> 1 : i] * slot_bytes;
                        if (HW == 8) {                              // (addresses are scalars)
                            load_to_lds_b128_nt(dst + (i >> 1) * kPitch + (i & 1) * kRow, ((i & 1) ? vbase : kbase) + row, 16 * lane);
                        } else if (PART) {
                            load_to_lds_b128_at(dst + i * kPitch, src + row);
                        } else {
                            load_to_lds_b128_at_nt(dst + i * kPitch, src + row);
                        }
                    }
                }
            };
            cols.load_queries(q + ((int64_t)at.b * Hq + h0) * kHeadDim, ng, l16, g);
            bring(slots_of(0));
            Slots next = slots_of(1);
            for (uint32_t j = 0; j < steps; ++j) {
                wait_vm<0>();                                       // this wavefront's rows of the step have landed
                if (j == 0) cols.queries_are_here();
                wg_barrier();
                uint32_t kc[2][4], ks[2], vw[2][4], vs[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    ks[u] = *(const ESP_LDS uint32_t*)(uintptr_t)(ks_rd + u * 16 * kPitch);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        kc[u][r] = *(const ESP_LDS uint32_t*)(uintptr_t)(k_rd + u * 16 * kPitch + 16 * r);
                        vw[u][r] = *(const ESP_LDS uint32_t*)(uintptr_t)(v_rd + (r + 16 * u) * kPitch);
                        vs[u][r] = *(const ESP_LDS uint32_t*)(uintptr_t)(vs_rd + (r + 16 * u) * kPitch);
                    }
                }
                wg_barrier();                                       // the step is in registers: the next may come into its place
                const int left = (int)min(seg - j * kStep, (uint32_t)kStep) - tsub * kQ4Tile;
                cols.hide(vw, left, g);
                if (j + 1 < steps) {
                    bring(next);
                    next = slots_of(j + 2);
                }
                floatx4 sc[NC][2];
                typename Q4Columns<NC>::PFrag pf[NC];
                cols.scores(kc, ks, sc);
                cols.weigh(sc, left, g, scale_log2, pf);
                cols.accumulate(vw, vs, l16 >> 2, pf);
            }
            __syncthreads();
        }
        const int64_t row = (parts == 1 ? (int64_t)at.b : (int64_t)(at.w + at.b)) * Hq + h0;
        cols.finish(tsub, NT, smem + hl * 8192, HW * 8192, s_ml + hl, HW, ng, l16, g, lane, parts == 1, row, part_acc, part_ml, O, LSE);
        at.done(seg);
    }
}

// Any other number of heads, and short requests: every wavefront brings what it needs itself, its head of K and of V of a tile's tokens.  68 bytes are
// four pieces of 16 and one that ends with them, beside the fourth: five lanes, twelve tokens to a transfer.  A pool of one head that has V next to K
// (JOINT) has 136 bytes there: nine lanes.  (A line of memory asked for by one instruction and not by several: codes and scales apart were 160 requests
// a tile, the rate of which bounds such a kernel; these are 98, and 66.)  With NC = 2 there is one workgroup to a CU, and a second tile on its way.  64
// requests of 1024 .. 131072, 32 / 1 heads: 43 us, and 5 for the combination; 136 bytes at a random place are two lines of 128 and more, 230 MB, 5.1
// TB/s.  The heads' lines overlap, and stay in the caches: 161 requests of 8000 or so, 6 / 3 heads, 258 us, past the caches 332.
template <int NC, bool JOINT>
__global__ __launch_bounds__(kQ4Waves * 64, NC == 1 ? 4 : 2) void decode_q4_kernel(
    const uint16_t* __restrict__ q, const char* __restrict__ k_pool, const char* __restrict__ v_pool, const int32_t* __restrict__ slot_idx,
    const int32_t* __restrict__ seq_offsets, int32_t B, int32_t total_tokens, int32_t range, int32_t parts, int32_t hw, int32_t nt, uint32_t slot_bytes,
    int32_t Hq, int32_t Hkv, float scale_log2, float* __restrict__ part_acc, float* __restrict__ part_ml, U32x2* __restrict__ O, float* __restrict__ LSE) {
    constexpr int kStages = NC, kPieces = JOINT ? 9 : 5, kRows = JOINT ? 7 : 12, kPitch = 16 * kPieces, kBytes = JOINT ? 2 * kQ4Head : kQ4Head;
    constexpr int kTransfers = (kQ4Tile + kRows - 1) / kRows, kVRegion = JOINT ? 0 : kQ4Tile * kPitch, kStage = JOINT ? kQ4Tile * kPitch : 2 * kVRegion;
    constexpr int kSlots = kStages * kStage, kRing = 4, kWaveLds = kSlots + kRing * 128 > 8192 ? kSlots + kRing * 128 : 8192;
    static_assert(kPitch / 4 % 8 == 4, "16 tokens' words in different banks");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kQ4Waves * kWaveLds];
    __shared__ float2 s_ml[kQ4Waves][16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int tsub = wave / hw, hl = wave - tsub * hw;
    const int head = blockIdx.y * hw + hl;
    const bool active = head < Hkv;
    const int G = Hq / Hkv, g0 = blockIdx.z * (16 * NC), ng = active ? min(16 * NC, G - g0) : 0;
    const int h0 = head * G + g0;
    const uint32_t lds = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem + wave * kWaveLds;
    // on its way in: lane kPieces t + p has piece p of token t
    const int in_row = lane / kPieces, piece = lane - in_row * kPieces;
    const int64_t from = (int64_t)(active ? head : 0) * kQ4Head + (piece == kPieces - 1 ? kBytes - 16 : 16 * piece);
    const char* const k_src = k_pool + from;
    const char* const v_src = v_pool + from;
    // on its way out: key l16 (and l16 + 16) for the first product, keys 4 g .. 4 g + 3 (and 16 more) for the second.  The last piece's bytes lie 12
    // (JOINT: 8) further on.
    const uint32_t k_rd = lds + l16 * kPitch + 4 * g, ks_rd = lds + l16 * kPitch + (JOINT ? 64 : 76);
    const uint32_t v_rd = lds + kVRegion + 4 * g * kPitch + (!JOINT ? 4 * l16 : l16 < 15 ? kQ4Head + 4 * l16 : 136), vs_rd = lds + kVRegion + 4 * g * kPitch + (JOINT ? 140 : 76);

    Q4Walk at;
    if (!at.start(range, parts, B, total_tokens, seq_offsets, lane)) return;
    uint32_t seg;
    while (at.next(parts, B, seq_offsets, seg)) {
        // tiles of this wavefront: tsub, tsub + nt, ...
        const uint32_t tiles = (seg + kQ4Tile - 1) / kQ4Tile, n = active && tiles > (uint32_t)tsub ? (tiles - tsub + nt - 1) / nt : 0;
        Q4Columns<NC> cols;
        cols.clear();
        if (n > 0) {
            const int32_t* const list = slot_idx + at.t0;
            // slots of the wavefront's tile j; past the last token: its slot again, hidden below
            auto load_slots = [&](uint32_t j) {
                if (lane < 32) load_to_lds_b32_at(lds + kSlots + 128 * (j % kRing), list + min((tsub + j * nt) * kQ4Tile + lane, seg - 1));
            };
            // tile j, whose slots have landed
            auto load_tile = [&](uint32_t j) {
                const ESP_LDS uint32_t* slots = (const ESP_LDS uint32_t*)(uintptr_t)(lds + kSlots + 128 * (j % kRing));
                uint64_t row[kTransfers];
#pragma unroll
                for (int i = 0; i < kTransfers; ++i) row[i] = (uint64_t)slots[min(i * kRows + in_row, kQ4Tile - 1)] * slot_bytes;
                const uint32_t to = lds + kStage * (j % kStages);
                load_slots(j + 2);
#pragma unroll
                for (int i = 0; i < kTransfers; ++i) {
                    if (in_row < (i < kTransfers - 1 ? kRows : kQ4Tile - i * kRows)) {
                        load_to_lds_b128_at(to + i * kRows * kPitch, k_src + row[i]);
                        if (!JOINT) load_to_lds_b128_at(to + kVRegion + i * kRows * kPitch, v_src + row[i]);
                    }
                }
            };
            load_slots(0);
            load_slots(1);
            cols.load_queries(q + ((int64_t)at.b * Hq + h0) * kHeadDim, ng, l16, g);
            wait_vm<0>();
            cols.queries_are_here();
#pragma unroll
            for (int x = 0; x < kStages; ++x) load_tile(x);
            for (uint32_t j = 0; j < n; ++j) {
                const uint32_t stage = kStage * (j % kStages);
                wait_vm<(kStages - 1) * (kTransfers * (JOINT ? 1 : 2) + 1)>();   // this tile has landed, the next may be on its way
                uint32_t kc[2][4], ks[2], vw[2][4], vs[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    ks[u] = *(const ESP_LDS uint32_t*)(uintptr_t)(ks_rd + stage + u * 16 * kPitch);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        kc[u][r] = *(const ESP_LDS uint32_t*)(uintptr_t)(k_rd + stage + u * 16 * kPitch + 16 * r);
                        vw[u][r] = *(const ESP_LDS uint32_t*)(uintptr_t)(v_rd + stage + (r + 16 * u) * kPitch);
                        vs[u][r] = *(const ESP_LDS uint32_t*)(uintptr_t)(vs_rd + stage + (r + 16 * u) * kPitch);
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile is in registers: another may come into its place
                const int left = (int)min(seg - (tsub + j * nt) * kQ4Tile, (uint32_t)kQ4Tile);
                cols.hide(vw, left, g);
                if (kStages > 1 || j + 1 < n) load_tile(j + kStages);
                floatx4 sc[NC][2];
                typename Q4Columns<NC>::PFrag pf[NC];
                cols.scores(kc, ks, sc);
                cols.weigh(sc, left, g, scale_log2, pf);
                cols.accumulate(vw, vs, l16 >> 2, pf);
            }
            wait_vm<0>();                                           // (the tiles past the last: nothing may land in what follows)
        }
        const int64_t row = (parts == 1 ? (int64_t)at.b : (int64_t)(at.w + at.b)) * Hq + h0;
        cols.finish(tsub, nt, smem + (hl + hw) * kWaveLds, hw * kWaveLds, s_ml + hl, hw, ng, l16, g, lane, parts == 1, row, part_acc, part_ml, O, LSE);
        at.done(seg);
    }
}

static int64_t q4_partial_bytes(int32_t Hq) { return (int64_t)Hq * (kHeadDim + 2) * (int64_t)sizeof(float); }

// Rows of eight heads, or of four, where the heads come in such; otherwise as many as are alike in up to eight.
static bool q4_rows(int32_t Hkv) { return Hkv % 4 == 0; }
static void q4_heads(int32_t Hkv, int32_t& hw, int32_t& nt, int32_t& hgroups) {
    if (q4_rows(Hkv)) hw = Hkv % 8 == 0 ? 8 : 4;
    else hw = (Hkv + (Hkv + kQ4Waves - 1) / kQ4Waves - 1) / ((Hkv + kQ4Waves - 1) / kQ4Waves);
    hgroups = (Hkv + hw - 1) / hw;
    nt = kQ4Waves / hw;
}

// Ranges of the token list, along it or counted from each request's first token on: as many as fill 1 .. 8 rounds of the workgroups that are on the
// chip at once, none of less than two steps, whichever is estimated to take the least time.  A round is a start and an end, and the steps.  Along the
// list some workgroup has a start and an end more, 8 us, for a request that its range crosses into, which the others' longer work hides; by request
// there are some B / 2 ranges more, and the others longer (64 requests of 1024 .. 131072, 32 / 1 heads, 64 us along the list, 49 by request).  Where no
// request has more ranges than are on the chip at once for all, each gets so many without a search, and a request that is no longer than a range is one
// workgroup's, which writes the result itself.
static Q4Geom q4_geom(int32_t B, int32_t total_tokens, int32_t max_len, int32_t Hq, int32_t Hkv) {
    Q4Geom x;
    const int G = Hq / Hkv;
    q4_heads(Hkv, x.hw, x.nt, x.hgroups);
    x.tiles = G > 16 ? 2 : 1;
    x.chunks = (G + 16 * x.tiles - 1) / (16 * x.tiles);
    // Short requests, few enough that each KV head of each can have a workgroup of its own: a tile to each wavefront at a time, and no second launch
    // (32 / 8 heads: 4 of up to 1024 tokens 10.6 against 8.6 us, 64 of 512 19.1 against 12.9, 64 of 1024 24.1 against 20.9; one of 2048 is better in
    // ranges, 10.5 against 13.8).
    if (max_len <= 1024 && (int64_t)B * Hkv * x.chunks <= (x.tiles == 1 ? 512 : 256)) {
        x.hw = 1;
        x.nt = max_len > (kQ4Waves - 1) * kQ4Tile ? kQ4Waves : max_len > 0 ? (max_len + kQ4Tile - 1) / kQ4Tile : 1;
        x.hgroups = Hkv;
        x.range = x.nt * kQ4Tile;
        x.nwg = x.parts = 1;
        return x;
    }
    const int64_t rows = (int64_t)x.hgroups * x.chunks, step = (int64_t)x.nt * kQ4Tile, resident = x.tiles == 1 ? 512 : 256;
    const int64_t steps = ((int64_t)total_tokens + step - 1) / step;
    const double step_us = (double)resident * step * x.hw * (2 * kQ4Head) / 6.4e6;
    const int64_t finest = steps > 2 * kQ4MaxRanges ? (steps + kQ4MaxRanges - 1) / kQ4MaxRanges : 2;
    int64_t best = 0;
    double best_us = 0;
    bool by_request = false;
    for (int by = 0; by < (B > 1 && B <= kQ4MostByRequest ? 2 : 1); ++by)
        for (int64_t rounds = 1; rounds <= 8; ++rounds) {
            const int64_t more = by ? B / 2 : 0, fit = rounds * resident / rows - more;   // ranges in so many rounds
            if (fit < 1 && rounds < 8) continue;
            const int64_t s = fit > 0 ? (steps + fit - 1) / fit : steps, take = s > finest ? s : finest;
            const int64_t ranges = (steps + take - 1) / take + more, wgs = ranges * rows;
            const double us = (double)((wgs + resident - 1) / resident) * (6 + step_us * (double)take) + (by || B < 2 ? 0 : 8 * 16.0 / (16 + (double)take));
            if (best == 0 || us < best_us) { best = take; best_us = us; by_request = by; }
            if (take == finest) break;
        }
    x.range = (int32_t)(best * step > INT32_MAX ? INT32_MAX / step * step : best * step);
    x.nwg = (int32_t)(((int64_t)total_tokens + x.range - 1) / x.range);
    if (x.nwg < 1) x.nwg = 1;
    const int64_t each = ((int64_t)max_len + x.range - 1) / x.range;   // ranges of the longest request
    x.parts = total_tokens == 0 || each <= 1 ? 1 : B * each * rows <= resident ? (int32_t)each : by_request ? -1 : 0;
    if (x.parts == 1 && x.range < max_len) x.range = max_len;
    return x;
}

// Room for the shortest ranges that any number of KV heads is read in, so that it rises with every size (no range is shorter than two steps of one tile
// or more).
size_t decode_q4_workspace_bytes(int32_t B, int32_t total_tokens, int32_t Hq) {
    int64_t ranges = ((int64_t)total_tokens + kQ4Tile - 1) / kQ4Tile;
    if (ranges > kQ4MaxRanges) ranges = kQ4MaxRanges;
    return (size_t)((ranges + 1 + B) * q4_partial_bytes(Hq)) + 256;
}

esp_status launch_decode_q4(const void* q, const void* k_pool, const void* v_pool, int64_t slot_bytes, const int32_t* slot_idx, const int32_t* seq_offsets,
                            int32_t B, int32_t total_tokens, int32_t max_len, int32_t Hq, int32_t Hkv, float softmax_scale, void* O, float* LSE,
                            void* workspace, hipStream_t stream) {
    if ((int64_t)B * Hq > INT32_MAX) return fail(ESP_ERR_INVALID_ARG, "decode (4 bits): too many rows for one launch");
    const Q4Geom x = q4_geom(B, total_tokens, max_len, Hq, Hkv);
    if (x.hgroups > 65535 || x.chunks > 65535) return fail(ESP_ERR_UNSUPPORTED, "decode (4 bits): too many heads for one launch");
    const int64_t grid = x.parts > 0 ? (int64_t)B * x.parts : x.parts < 0 ? (int64_t)x.nwg + B : x.nwg;
    if (grid > (1 << 22)) return fail(ESP_ERR_INVALID_ARG, "decode (4 bits): too many requests for one launch");
    float* part_acc = (float*)workspace;
    float* part_ml = part_acc + (size_t)(x.nwg + B) * Hq * kHeadDim;
#define ESP_Q4_LAUNCH(NC, JOINT)                                                                                                                                 \
    hipLaunchKernelGGL((decode_q4_kernel<NC, JOINT>), dim3((unsigned)grid, x.hgroups, x.chunks), dim3(64 * x.hw * x.nt), 0, stream, (const uint16_t*)q,             \
                       (const char*)k_pool, (const char*)v_pool, slot_idx, seq_offsets, B, total_tokens, x.range, x.parts, x.hw, x.nt, (uint32_t)slot_bytes, Hq,     \
                       Hkv, score_factor(softmax_scale), part_acc, part_ml, (U32x2*)O, LSE)
#define ESP_Q4_ROWS_LAUNCH(HW, NC, PART)                                                                                                                  \
    hipLaunchKernelGGL((decode_q4_rows_kernel<HW, NC, PART>), dim3((unsigned)grid, x.hgroups, x.chunks), dim3(kQ4Waves * 64), 0, stream, (const uint16_t*)q,     \
                       (const char*)k_pool, (const char*)v_pool, slot_idx, seq_offsets, B, total_tokens, x.range, x.parts, (uint32_t)slot_bytes, Hq, Hkv,   \
                       score_factor(softmax_scale), part_acc, part_ml, (U32x2*)O, LSE)
    if (q4_rows(Hkv) && x.hw > 1) {
        if (x.hw == 8) {
            if (x.tiles == 1) ESP_Q4_ROWS_LAUNCH(8, 1, false);
            else ESP_Q4_ROWS_LAUNCH(8, 2, false);
        } else {
            const bool part = x.hgroups > 1;
            if (x.tiles == 1) { if (part) ESP_Q4_ROWS_LAUNCH(4, 1, true); else ESP_Q4_ROWS_LAUNCH(4, 1, false); }
            else { if (part) ESP_Q4_ROWS_LAUNCH(4, 2, true); else ESP_Q4_ROWS_LAUNCH(4, 2, false); }
        }
    } else if (Hkv == 1 && (const char*)v_pool == (const char*)k_pool + kQ4Head) {
        if (x.tiles == 1) ESP_Q4_LAUNCH(1, true); else ESP_Q4_LAUNCH(2, true);
    } else {
        if (x.tiles == 1) ESP_Q4_LAUNCH(1, false); else ESP_Q4_LAUNCH(2, false);
    }
#undef ESP_Q4_ROWS_LAUNCH
#undef ESP_Q4_LAUNCH
    const esp_status st = check_launch("decode_q4_kernel");
    if (st != ESP_OK || x.parts == 1) return st;
    return launch_decode_combine(seq_offsets, x.range, x.parts, max_len, B, Hq, part_acc, part_ml, nullptr, 0, O, LSE, stream);
}

}  // namespace esp
