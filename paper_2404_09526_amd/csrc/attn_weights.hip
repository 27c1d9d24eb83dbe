// esp_accumulate_attn_weights, ..._q4: for every key of the requests' lists, the attention weights that the requests' queries give it,
//   sum over queries t and heads h of exp(softmax_scale q_th . k_h/G - LSE_th),
// added up per pool slot.  One pass over K: a wavefront has a KV head and tiles of 32 tokens, the query heads of all of its queries are columns of
//   S^T [32 keys x 16] = K [32 x 128] Q^T [128 x 16],
// 16 at a time against the tile in registers, and the weights of a key are added over the columns a lane has, the lanes, the heads (of a workgroup, through the
// LDS; it has all heads of its tokens, so nothing is added by two workgroups and the order is always the same), in fp32.
// Bound by the memory for one query a request: 256 bytes of a head of a token, or 68; for many queries by the waits for their chunks of columns, of which
// each is little work (32 queries of 4 heads a KV head: vector ALU busy for 30 % of the cycles, matrix cores for 14 %).
#include "attn_weights.h"
#include "decode_merge.h"
#include "mfma_tile.h"
#include "q4.h"

#include <algorithm>

namespace esp {

constexpr int kAwWaves = 8, kAwTile = 32;
constexpr int kAwSums = 1792;                     // heads of a workgroup times tokens of its range, at most (two workgroups fit a CU)

// The same in all lanes, and to be kept in scalars (the compiler does not read what the kernel might write with scalar loads).
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// What a lane brings of a tile's K rows, and reads of them.  4 bits: lane 5 t + p has piece p of token t (twelve tokens a transfer), the last piece is
// that which ends with the head; bf16: lane 16 t + p has piece p ^ t % 16 of token t (four a transfer).  Either way the words that 16 tokens' lanes
// read lie in different banks.
template <bool Q4>
struct KTile {
    static constexpr int kPitch = Q4 ? 80 : 256, kTransfers = Q4 ? 3 : 8, kRows = Q4 ? 12 : 4, kBytes = kAwTile * kPitch;
    struct Slots { int32_t s[Q4 ? kTransfers : 1]; };
    int in_row, from, lane, l16;
    uint32_t lds, k_rd, ks_rd;
    __device__ __forceinline__ void place(uint32_t at, int lane_) {
        lane = lane_; l16 = lane & 15; lds = at;
        const int g = lane >> 4;
        in_row = Q4 ? lane / 5 : lane >> 4;
        const int piece = Q4 ? lane - in_row * 5 : 0;
        from = Q4 ? (piece == 4 ? kQ4Head - 16 : 16 * piece) : 0;
        k_rd = Q4 ? lds + l16 * kPitch + 4 * g : lds + l16 * kPitch + ((g ^ l16) << 4);
        ks_rd = lds + l16 * kPitch + 76;
    }
    // slots of the tile at `first` of a list of seg tokens; past the last: its slot again, left out later
    __device__ __forceinline__ Slots slots_of(const int32_t* list, uint32_t first, uint32_t seg) const {
        Slots r;
        if constexpr (Q4) {
#pragma unroll
            for (int i = 0; i < kTransfers; ++i) r.s[i] = list[min(first + min(i * kRows + in_row, kAwTile - 1), seg - 1)];
        } else {
            r.s[0] = list[min(first + (lane & 31), seg - 1)];
        }
        return r;
    }
    // src: the head in slot 0
    __device__ __forceinline__ void bring(const char* src, uint32_t slot_bytes, const Slots& sl) const {
        // (formed anew each time: held over a loop, eight addresses went to scratch memory, and each transfer waited for the one before with its reload)
        int within = Q4 ? from : (l16 ^ in_row) << 4;
        asm volatile("" : "+v"(within));
#pragma unroll
        for (int i = 0; i < kTransfers; ++i) {
            const int32_t slot = Q4 ? sl.s[Q4 ? i : 0] : __shfl(sl.s[0], i * kRows + in_row);
            const uint64_t at = (uint64_t)(uint32_t)slot * slot_bytes + (uint32_t)(Q4 ? within : within ^ ((i & 3) << 6));
            if (!Q4 || in_row < (i < kTransfers - 1 ? kRows : kAwTile - i * kRows)) {
                // (heads of 68 bytes have lines in common with their neighbours', which stay in the caches; 64 requests of 1024 .. 131072, 6 / 3 heads,
                // 95 us, past them 103)
                if (Q4) load_to_lds_b128_at(lds + i * kRows * kPitch, src + at);
                else load_to_lds_b128_at_nt(lds + i * kRows * kPitch, src + at);
            }
        }
    }
    // the operand of keys l16 and l16 + 16: step s has elements 32 s + 8 (lane / 16) ..
    __device__ __forceinline__ void read(bf16x8 (&kf)[2][4]) const {
        if constexpr (Q4) {
            uint32_t kc[2][4], ks[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                ks[u] = *(const ESP_LDS uint32_t*)(uintptr_t)(ks_rd + u * 16 * kPitch);
#pragma unroll
                for (int s = 0; s < 4; ++s) kc[u][s] = *(const ESP_LDS uint32_t*)(uintptr_t)(k_rd + u * 16 * kPitch + 16 * s);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int s = 0; s < 4; ++s) kf[u][s] = __builtin_bit_cast(bf16x8, q4_to_bf16(kc[u][s], q4_scale(ks[u], s)));
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int s = 0; s < 4; ++s) kf[u][s] = *(const ESP_LDS bf16x8*)(uintptr_t)((k_rd ^ (s << 6)) + u * 16 * kPitch);
        }
    }
};

// Sums over the 16 lanes of a key, added to the tokens' sums so far: lane 4 u + r of the 16 has key 16 u + 4 (lane / 16) + r.
__device__ __forceinline__ void add_to_tokens(const float (&sum)[2][4], float* tokens, uint32_t first, uint32_t seg, int l16, int g) {
    float out = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float x = row16_sum(sum[u][r]);
            if (l16 == 4 * u + r) out = x;
        }
    const uint32_t token = first + 16 * (l16 >> 2) + 4 * g + (l16 & 3);
    if (l16 < 8 && token < seg) tokens[token] += out;
}

// One query a request, the other way round: S = Q K^T, so that a lane has keys l16 and l16 + 16 and four of the 16 columns, and little is left to be
// added across lanes (with a key to 16 lanes half of the instructions of a tile were those).
template <bool MASK>
struct OneQuery {
    bf16x8 qf[4];
    float against[4];
    int32_t q_pos[MASK ? 4 : 1];
    bool used[4];
    // columns: queries q0 .. q0 + nq of G heads (at most 16 columns), heads from h0 on
    __device__ __forceinline__ void load(const WeightsArgs& a, int32_t q0, int nq, int h0, int G, int l16, int g) {
        auto row_of = [&](int c, bool& in) {
            const int ql = c / G, hd = c - ql * G;
            in = ql < nq;
            return (int64_t)(q0 + (in ? ql : 0)) * a.Hq + h0 + (in ? hd : 0);
        };
        bool in;
        const uint4* qp = (const uint4*)(a.q + row_of(l16, in) * kHeadDim + 8 * g);
#pragma unroll
        for (int s = 0; s < 4; ++s) qf[s] = __builtin_bit_cast(bf16x8, qp[4 * s]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            against[r] = a.LSE[row_of(4 * g + r, used[r])];
            if (MASK) q_pos[r] = a.q_pos[q0 + (used[r] ? (4 * g + r) / G : 0)];
        }
    }
    // Waited for here: in the loop that uses them the compiler would wait for them, and for all transfers with them, each time (16 requests of 32 ..
    // 4096, 8 / 8 heads in bf16, 11.2 against 10.9 us).
    __device__ __forceinline__ void is_here() {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            asm volatile("" : "+v"(qf[r]), "+v"(against[r]));
            if (MASK) asm volatile("" : "+v"(q_pos[r]));
            used[r] = used[r] & (against[r] != -INFINITY);          // a query that saw nothing gives nothing, whatever it holds
            against[r] *= kLog2e;
        }
    }
    __device__ __forceinline__ float weights(const bf16x8 (&kf)[4], int32_t kv_pos, float scale_log2) const {
        floatx4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[s], kf[s], sc, 0, 0, 0);
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const bool seen = used[r] & (!MASK || kv_pos <= q_pos[MASK ? r : 0]);
            x[r] = __builtin_amdgcn_exp2f(seen ? fmaf(sc[r], scale_log2, -against[r]) : -INFINITY);
        }
        return (x[0] + x[1]) + (x[2] + x[3]);
    }
};
// The weights of keys l16 (x) and l16 + 16 (y), each a sum over some columns in lanes 16 apart: the whole sums, of x in lanes 0 .. 31 and of y in 32 .. 63.
__device__ __forceinline__ float both_keys(float x, float y) {
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));       // lanes 0 .. 31: both halves of x, 32 .. 63: of y
    x += y;
    y = x;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(x), "+v"(y));       // and both rows of 16 of each half
    return x + y;
}

template <bool Q4, bool MANY, bool MASK>
__global__ __launch_bounds__(kAwWaves * 64, 4) void attn_weights_kernel(WeightsArgs a) {
    // MANY: a chunk of columns, 16 rows of queries, what they are taken against and their positions, goes through the same block
    constexpr int kChunkBytes = 17 * 256, kWaveLds = MANY && KTile<Q4>::kBytes < kChunkBytes ? kChunkBytes : KTile<Q4>::kBytes;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kAwWaves * kWaveLds];
    __shared__ __attribute__((aligned(16))) int32_t s_pos[MASK ? kAwWaves * kAwTile : 4];   // a tile's positions
    __shared__ float s_sum[kAwSums];              // [heads of the workgroup][tokens of the range]
    __shared__ float s_keep[kAwSums];             // what a token's sum so far is multiplied by; negative: it is no request's
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int tsub = wave / a.hw, hl = wave - tsub * a.hw;
    const int G = a.Hq / a.Hkv;
    const int64_t begin = wide_block() * a.range;
    if (begin >= a.total_tokens) return;
    const int32_t r0 = (int32_t)begin, r1 = r0 + min(a.range, a.total_tokens - r0);
    const uint32_t lds = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem + wave * kWaveLds;
    KTile<Q4> tile;
    tile.place(lds, lane);
    // columns: QB queries of G heads, or 16 heads of one query
    const int QB = G <= 16 ? 16 / G : 1, HB = (G + 15) / 16;
    const int ql = G <= 16 ? l16 / G : 0, hd = l16 - ql * G;
    int in_ql[4];                                 // MANY: the queries of the four columns that this lane brings a part of
#pragma unroll
    for (int i = 0; i < 4; ++i) in_ql[i] = MANY && G <= 16 ? (4 * i + g) / G : 0;

    for (int i = threadIdx.x; i < a.hw * a.range; i += blockDim.x) s_sum[i] = 0.f;
    for (int i = threadIdx.x; i < a.range; i += blockDim.x) s_keep[i] = -1.f;
    RequestAt at = request_of(r0, a.seq_offsets, a.B, lane);
    __syncthreads();
    int b = at.b;
    int32_t t0 = r0, req_end = at.end;
    while (t0 < r1 && b < a.B) {                                    // (tokens past the offsets' end belong to no request)
        if (t0 > r0) req_end = uniform(a.seq_offsets[b + 1]);
        if (req_end <= t0) { ++b; continue; }
        const int32_t pe = min(r1, req_end);
        const uint32_t seg = (uint32_t)(pe - t0);
        for (int32_t i = t0 - r0 + (int32_t)threadIdx.x; i < pe - r0; i += (int32_t)blockDim.x) s_keep[i] = (int64_t)req_end - r0 - i <= a.fresh ? 0.f : a.decay;
        const int32_t q0 = a.q_offsets ? uniform(a.q_offsets[b]) : b, nq = a.q_offsets ? min(uniform(a.q_offsets[b + 1]) - q0, a.max_q) : 1;
        const int32_t* const list = a.slot_idx + t0;
        const uint32_t tiles = (seg + kAwTile - 1) / kAwTile, n = nq > 0 && tiles > (uint32_t)tsub ? (tiles - tsub + a.nt - 1) / a.nt : 0;
        for (int h = hl; n > 0 && h < a.Hkv; h += a.hw) {
            const char* const src = a.k_pool + h * (Q4 ? kQ4Head : 256);
            float* const tokens = s_sum + hl * a.range + (t0 - r0);
            auto first_of = [&](uint32_t j) { return (tsub + j * a.nt) * kAwTile; };
            auto bring = [&](uint32_t j, const typename KTile<Q4>::Slots& sl) {
                if (MASK && lane < kAwTile)
                    load_to_lds_b32_at((uint32_t)(uintptr_t)(ESP_LDS int32_t*)s_pos + wave * (kAwTile * 4), a.kv_pos + t0 + (int32_t)min(first_of(j) + lane, seg - 1));
                tile.bring(src, a.slot_bytes, sl);
            };
            bf16x8 kf[2][4], qf[4];
            int32_t kv_pos[2][4];
            auto read_tile = [&] {
                tile.read(kf);
                if constexpr (MASK) {
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r) kv_pos[u][r] = s_pos[wave * kAwTile + 16 * u + 4 * g + r];
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // in registers: what comes next may take its place
            };
            float sum[2][4];
            auto add_columns = [&](float lse, bool used, int32_t q_pos) {
                const float against = lse * kLog2e;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    floatx4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < 4; ++s) sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u][s], qf[s], sc, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool seen = used & (!MASK | (kv_pos[u][r] <= q_pos));
                        sum[u][r] += __builtin_amdgcn_exp2f(seen ? fmaf(sc[r], a.scale_log2, -against) : -INFINITY);
                    }
                }
            };
            auto clear = [&] {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[u][r] = 0.f;
            };
            bring(0, tile.slots_of(list, first_of(0), seg));
            auto next = tile.slots_of(list, first_of(1), seg);
            if constexpr (!MANY) {
                OneQuery<MASK> one;
                one.load(a, q0, nq, h * G, G, l16, g);
                one.is_here();
                for (uint32_t j = 0; j < n; ++j) {
                    wait_vm<0>();                                   // the tile has landed (and what else was on its way)
                    tile.read(kf);
                    int32_t pos[2] = {0, 0};
                    if constexpr (MASK) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) pos[u] = s_pos[wave * kAwTile + 16 * u + l16];
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    if (j + 1 < n) {
                        bring(j + 1, next);
                        next = tile.slots_of(list, first_of(j + 2), seg);
                    }
                    const float x = one.weights(kf[0], pos[0], a.scale_log2), y = one.weights(kf[1], pos[1], a.scale_log2);
                    const float both = both_keys(x, y);
                    const uint32_t token = first_of(j) + 8 * g + l16;
                    if (g % 2 == 0 && token < seg) tokens[token] += both;
                }
            } else {
                // Chunks of columns through the LDS, four lanes' 1 KiB each of its 16 rows: operands read from memory by their own lanes kept the
                // address unit busy for most of the time (32 queries of 4 heads a KV head, 143000 keys, 198 us).
                const int blocks = (nq + QB - 1) / QB;
                const uint32_t query_bytes = (uint32_t)a.Hq * (2 * kHeadDim);
                // block qb of queries, hb of heads; columns past the last have its query, or head, again
                auto bring_chunk = [&](int qb, int hb) {
                    const int left = nq - 1 - qb * QB;
                    const int64_t row = ((int64_t)q0 + qb * QB) * a.Hq + h * G;
                    const uint16_t* const queries = a.q + row * kHeadDim;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {                   // rows 4 i + g, piece l16 ^ (4 i + g) of each
                        const int head = min(hb * 16 + 4 * i + g - in_ql[i] * G, G - 1);
                        load_to_lds_b128(lds + 1024 * i, queries, (uint32_t)min(in_ql[i], left) * query_bytes + (uint32_t)(head << 8) + (((l16 ^ g) << 4) ^ (i << 6)));
                    }
                    const uint32_t query = (uint32_t)min(ql, left);
                    if (lane < 16) load_to_lds_b32(lds + 4096, a.LSE + row, 4 * (query * (uint32_t)a.Hq + (uint32_t)min(hb * 16 + hd, G - 1)));
                    if (MASK && lane < 16) load_to_lds_b32(lds + 4160, a.q_pos + q0 + qb * QB, 4 * query);
                };
                for (uint32_t j = 0; j < n; ++j) {
                    wait_vm<0>();
                    read_tile();
                    bring_chunk(0, 0);
                    clear();
                    for (int qb = 0, hb = 0; qb < blocks;) {
                        wait_vm<0>();
                        const uint32_t q_rd = lds + l16 * 256 + ((g ^ l16) << 4);
#pragma unroll
                        for (int s = 0; s < 4; ++s) qf[s] = *(const ESP_LDS bf16x8*)(uintptr_t)(q_rd ^ (s << 6));
                        const float lse = *(const ESP_LDS float*)(uintptr_t)(lds + 4096 + 4 * l16);
                        const int32_t q_pos = MASK ? *(const ESP_LDS int32_t*)(uintptr_t)(lds + 4160 + 4 * l16) : 0;
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                        // (a query that saw nothing gives nothing)
                        const bool used = qb * QB + ql < nq && hb * 16 + hd < G && (G > 16 || l16 < QB * G) && lse != -INFINITY;
                        if (++hb == HB) { hb = 0; ++qb; }
                        if (qb < blocks) bring_chunk(qb, hb);
                        else if (j + 1 < n) bring(j + 1, next);
                        add_columns(lse, used, q_pos);
                    }
                    next = tile.slots_of(list, first_of(j + 2), seg);
                    add_to_tokens(sum, tokens, first_of(j), seg, l16, g);
                }
            }
        }
        t0 = pe;
        ++b;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < r1 - r0; i += blockDim.x) {
        const float keep = s_keep[i];
        const int32_t slot = a.slot_idx[r0 + i];
        if (keep < 0.f || slot < 0 || slot >= a.num_slots) continue;
        float x = 0.f;
        for (int u = 0; u < a.hw; ++u) x += s_sum[u * a.range + i];
        a.sums[slot] = keep > 0.f ? fmaf(keep, a.sums[slot], x) : x;
    }
}

// Many queries against long lists: the workgroup's wavefronts have a tile of 32 tokens each and take the heads one after another, so that a chunk of
// columns is brought once for all of them, and a key's sum stays in registers over all heads.  With a head to a wavefront each brought the queries of
// its head for every 32 tokens: 32 queries of 4 heads a KV head, 143000 keys, 1.6 GB from the L2, 153 us; so 108.  One wavefront more brings the
// chunks, three ahead: loads are waited for in their order, and a chunk asked for behind the next head's tile waited for that (156 us, with eight
// wavefronts at any length).  Meeting once for two chunks, the next two on their way: 125.  Bound by instructions and their latency between two
// meetings: without its sums 93 us, without memory 120 of then 140.
constexpr int kAwPlaces = 4;                      // of chunks
constexpr int kAwTiles = 7;                       // wavefronts with a tile, at most (two workgroups fit a CU)
template <bool Q4, bool MASK>
__global__ __launch_bounds__((kAwTiles + 1) * 64, 4) void attn_weights_span_kernel(WeightsArgs a) {
    constexpr int kChunk = 17 * 256;              // 16 rows of queries, what they are taken against, their positions
    constexpr int kChunkTransfers = MASK ? 6 : 5;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kAwTiles * KTile<Q4>::kBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char s_chunk[kAwPlaces * kChunk];
    __shared__ float s_sum[kAwTiles * kAwTile], s_keep[kAwTiles * kAwTile];
    __shared__ int32_t s_pos[MASK ? kAwTiles * kAwTile : 4];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int G = a.Hq / a.Hkv;
    const int64_t begin = wide_block() * a.range;
    if (begin >= a.total_tokens) return;
    const int32_t r0 = (int32_t)begin, r1 = r0 + min(a.range, a.total_tokens - r0);
    const uint32_t lds_chunk = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)s_chunk;
    const int QB = G <= 16 ? 16 / G : 1, HB = (G + 15) / 16;
    const int ql = G <= 16 ? l16 / G : 0, hd = l16 - ql * G;

    for (int i = threadIdx.x; i < a.range; i += blockDim.x) { s_sum[i] = 0.f; s_keep[i] = -1.f; }
    RequestAt at = request_of(r0, a.seq_offsets, a.B, lane);
    __syncthreads();
    int b = at.b;
    int32_t t0 = r0, req_end = at.end;
    while (t0 < r1 && b < a.B) {                                    // (tokens past the offsets' end belong to no request)
        if (t0 > r0) req_end = uniform(a.seq_offsets[b + 1]);
        if (req_end <= t0) { ++b; continue; }
        const int32_t pe = min(r1, req_end);
        const uint32_t seg = (uint32_t)(pe - t0);
        for (int32_t i = t0 - r0 + (int32_t)threadIdx.x; i < pe - r0; i += (int32_t)blockDim.x) s_keep[i] = (int64_t)req_end - r0 - i <= a.fresh ? 0.f : a.decay;
        const int32_t q0 = a.q_offsets ? uniform(a.q_offsets[b]) : b, nq = a.q_offsets ? min(uniform(a.q_offsets[b + 1]) - q0, a.max_q) : 1;
        const int blocks = nq > 0 ? (nq + QB - 1) / QB : 0;
        const int64_t chunks = (int64_t)a.Hkv * blocks * HB;        // head by head, of each all queries; every wavefront meets the others once a chunk
        if (wave == a.nt) {
            // columns past the last have its query, or head, again
            const uint32_t query_bytes = (uint32_t)a.Hq * (2 * kHeadDim);
            int h = 0, qb = 0, hb = 0, place = 0;                   // the next to be brought
            int in_ql[4];                                           // the queries of the four rows that this lane brings a part of
#pragma unroll
            for (int i = 0; i < 4; ++i) in_ql[i] = G <= 16 ? (4 * i + g) / G : 0;
            auto bring_chunk = [&] {
                const int left = nq - 1 - qb * QB;
                const int64_t row = ((int64_t)q0 + qb * QB) * a.Hq + h * G;
                const uint16_t* const queries = a.q + row * kHeadDim;
                const uint32_t to = lds_chunk + place * kChunk;
#pragma unroll
                for (int i = 0; i < 4; ++i) {                       // rows 4 i + g, piece l16 ^ (4 i + g) of each
                    const int head = min(hb * 16 + 4 * i + g - in_ql[i] * G, G - 1);
                    load_to_lds_b128(to + 1024 * i, queries, (uint32_t)min(in_ql[i], left) * query_bytes + (uint32_t)(head << 8) + (((l16 ^ g) << 4) ^ (i << 6)));
                }
                if (lane < 16) {
                    const uint32_t query = (uint32_t)min(ql, left);
                    load_to_lds_b32(to + 4096, a.LSE + row, 4 * (query * (uint32_t)a.Hq + (uint32_t)min(hb * 16 + hd, G - 1)));
                    if (MASK) load_to_lds_b32(to + 4160, a.q_pos + q0 + qb * QB, 4 * query);
                }
                if (++hb == HB) { hb = 0; if (++qb == blocks) { qb = 0; ++h; } }
                place = place == kAwPlaces - 1 ? 0 : place + 1;
            };
            for (int c = 0; c < kAwPlaces - 1 && c < chunks; ++c) bring_chunk();
            for (int64_t c = 0; c < chunks; ++c) {
                if (c + kAwPlaces - 1 <= chunks) wait_vm<(kAwPlaces - 2) * kChunkTransfers>();
                else wait_vm<0>();
                wg_barrier();                                       // chunk c has landed; and all have read the one before, whose place the next brought takes
                if (c + kAwPlaces - 1 < chunks) bring_chunk();
            }
        } else if (chunks > 0) {
            const uint32_t first = wave * kAwTile;
            if (first >= seg) {
                for (int64_t c = 0; c < chunks; ++c) wg_barrier();
            } else {
                KTile<Q4> tile;
                tile.place((uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem + wave * KTile<Q4>::kBytes, lane);
                const auto slots = tile.slots_of(a.slot_idx + t0, first, seg);
                int32_t last_pos = 0;                               // of the tile's keys
                if constexpr (MASK) {
                    last_pos = a.kv_pos[t0 + (int32_t)min(first + (lane & 31), seg - 1)];
                    if (lane < kAwTile) s_pos[wave * kAwTile + lane] = last_pos;
#pragma unroll
                    for (int x = 1; x < kAwTile; x *= 2) last_pos = max(last_pos, __shfl_xor(last_pos, x));
                    last_pos = uniform(last_pos);
                }
                auto bring = [&](int h) { tile.bring(a.k_pool + h * (Q4 ? kQ4Head : 256), a.slot_bytes, slots); };
                float sum[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[u][r] = 0.f;
                bring(0);
                uint32_t from = lds_chunk;
                for (int h = 0; h < a.Hkv; ++h) {
                    bf16x8 kf[2][4];
                    wait_vm<0>();
                    tile.read(kf);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // in registers: the next head's may take its place
                    if (h + 1 < a.Hkv) bring(h + 1);
                    for (int qb = 0, hb = 0; qb < blocks;) {
                        wg_barrier();
                        const uint32_t q_rd = from + l16 * 256 + ((g ^ l16) << 4);
                        bf16x8 qf[4];
#pragma unroll
                        for (int s = 0; s < 4; ++s) qf[s] = *(const ESP_LDS bf16x8*)(uintptr_t)(q_rd ^ (s << 6));
                        const float lse = *(const ESP_LDS float*)(uintptr_t)(from + 4096 + 4 * l16);
                        const int32_t q_pos = MASK ? *(const ESP_LDS int32_t*)(uintptr_t)(from + 4160 + 4 * l16) : 0;
                        from = from == lds_chunk + (kAwPlaces - 1) * kChunk ? lds_chunk : from + kChunk;
                        const float against = lse * kLog2e;
                        // (a query that saw nothing gives nothing)
                        const bool used = (qb * QB + ql < nq) & (hb * 16 + hd < G) & ((G > 16) | (l16 < QB * G)) & (lse != -INFINITY);
                        if (++hb == HB) { hb = 0; ++qb; }
                        floatx4 sc[2];
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            sc[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int s = 0; s < 4; ++s) sc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u][s], qf[s], sc[u], 0, 0, 0);
                        }
                        if (__all(used & (!MASK | (last_pos <= q_pos)))) {      // most chunks: nothing to be left out
#pragma unroll
                            for (int u = 0; u < 2; ++u)
#pragma unroll
                                for (int r = 0; r < 4; ++r) sum[u][r] += __builtin_amdgcn_exp2f(fmaf(sc[u][r], a.scale_log2, -against));
                        } else {
#pragma unroll
                            for (int u = 0; u < 2; ++u)
#pragma unroll
                                for (int r = 0; r < 4; ++r) {
                                    const bool seen = used & (!MASK || s_pos[wave * kAwTile + 16 * u + 4 * g + r] <= q_pos);
                                    sum[u][r] += __builtin_amdgcn_exp2f(seen ? fmaf(sc[u][r], a.scale_log2, -against) : -INFINITY);
                                }
                        }
                    }
                }
                add_to_tokens(sum, s_sum + (t0 - r0), first, seg, l16, g);
            }
        }
        wg_barrier();                                               // the last chunk is read
        t0 = pe;
        ++b;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < r1 - r0; i += blockDim.x) {
        const float keep = s_keep[i];
        const int32_t slot = a.slot_idx[r0 + i];
        if (keep < 0.f || slot < 0 || slot >= a.num_slots) continue;
        a.sums[slot] = keep > 0.f ? fmaf(keep, a.sums[slot], s_sum[i]) : s_sum[i];
    }
}

// One query a request against rows of four or eight heads in 4 bits (HW: the workgroup's at a time): K's rows whole, by all wavefronts, as decode reads
// them.  64 requests of 1024 .. 131072, 32 / 8 heads: 186 us with a line asked for by each head's wavefront, 153 with a key's columns over 16 lanes and
// the list read again by every step, 127 so.  Of these 26 are the sums' own lines, one of 128 bytes for 4; the rows' lines, 5.3 of 128 bytes for 544,
// come at 5.4 TB/s.  (Two steps on their way, or a workgroup for all tokens of a third of a CU, were no faster: 131.)
constexpr int kAwRowsSums = 4096;                 // heads of a workgroup times tokens of its range, at most (three workgroups fit a CU)
template <int HW>
__global__ __launch_bounds__(kAwWaves * 64, 6) void attn_weights_rows_kernel(WeightsArgs a) {
    constexpr int NT = kAwWaves / HW, kStep = NT * kAwTile, kRow = HW * kQ4Head, kPitch = HW == 8 ? kRow + 16 : kRow, kOwn = kStep / kAwWaves;
    static_assert(kPitch / 4 % 8 == 4, "16 tokens' words in different banks");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kStep * kPitch];
    __shared__ float s_sum[kAwRowsSums];
    __shared__ float s_keep[kAwRowsSums / HW];
    __shared__ int32_t s_slot[kAwRowsSums / HW];                    // the range's part of the list
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int tsub = wave / HW, hl = wave % HW;
    const int G = a.Hq / a.Hkv;
    const int64_t begin = wide_block() * a.range;
    if (begin >= a.total_tokens) return;
    const int32_t r0 = (int32_t)begin, r1 = r0 + min(a.range, a.total_tokens - r0);
    const uint32_t lds = (uint32_t)(uintptr_t)(ESP_LDS unsigned char*)smem;
    const uint32_t mine = lds + (tsub * kAwTile + l16) * kPitch + hl * kQ4Head, k_rd = mine + 4 * g, ks_rd = mine + kQ4Codes;

    for (int i = threadIdx.x; i < HW * a.range; i += kAwWaves * 64) s_sum[i] = 0.f;
    for (int i = threadIdx.x; i < a.range; i += kAwWaves * 64) {
        s_keep[i] = -1.f;
        s_slot[i] = i < r1 - r0 ? a.slot_idx[r0 + i] : -1;
    }
    RequestAt at = request_of(r0, a.seq_offsets, a.B, lane);
    __syncthreads();
    int b = at.b;
    int32_t t0 = r0, req_end = at.end;
    while (t0 < r1 && b < a.B) {                                    // (tokens past the offsets' end belong to no request)
        if (t0 > r0) req_end = uniform(a.seq_offsets[b + 1]);
        if (req_end <= t0) { ++b; continue; }
        const int32_t pe = min(r1, req_end);
        const uint32_t seg = (uint32_t)(pe - t0);
        for (int32_t i = t0 - r0 + (int32_t)threadIdx.x; i < pe - r0; i += kAwWaves * 64) s_keep[i] = (int64_t)req_end - r0 - i <= a.fresh ? 0.f : a.decay;
        const int32_t q0 = a.q_offsets ? uniform(a.q_offsets[b]) : b, nq = a.q_offsets ? min(uniform(a.q_offsets[b + 1]) - q0, a.max_q) : 1;
        const uint32_t steps = nq > 0 ? (seg + kStep - 1) / kStep : 0;
        for (int h = hl, base = 0; base < a.Hkv && steps > 0; base += HW, h += HW) {
            const char* const src = a.k_pool + base * kQ4Head;
            auto bring = [&](uint32_t j) {                          // past the last token: its slot again, left out below
                uint64_t slot[kOwn];
#pragma unroll
                for (int i = 0; i < kOwn; ++i) slot[i] = (uint32_t)uniform(s_slot[t0 - r0 + (int32_t)min(j * kStep + wave * kOwn + i, seg - 1)]);
                if (lane < kRow / 16) {
#pragma unroll
                    for (int i = 0; i < kOwn; ++i)                  // (the same slot in all lanes: addresses are scalars)
                        load_to_lds_b128_nt(lds + (wave * kOwn + i) * kPitch, src + slot[i] * a.slot_bytes, 16 * lane);
                }
            };
            OneQuery<false> one;                                    // (G <= 16)
            one.load(a, q0, nq, h * G, G, l16, g);
            bring(0);
            one.is_here();
            for (uint32_t j = 0; j < steps; ++j) {
                wait_vm<0>();
                wg_barrier();
                uint32_t kc[2][4], ks[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    ks[u] = *(const ESP_LDS uint32_t*)(uintptr_t)(ks_rd + u * 16 * kPitch);
#pragma unroll
                    for (int s = 0; s < 4; ++s) kc[u][s] = *(const ESP_LDS uint32_t*)(uintptr_t)(k_rd + u * 16 * kPitch + 16 * s);
                }
                wg_barrier();                                       // in registers: the next step may take its place
                if (j + 1 < steps) bring(j + 1);
                float x[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    bf16x8 kf[4];
#pragma unroll
                    for (int s = 0; s < 4; ++s) kf[s] = __builtin_bit_cast(bf16x8, q4_to_bf16(kc[u][s], q4_scale(ks[u], s)));
                    x[u] = one.weights(kf, 0, a.scale_log2);
                }
                const float both = both_keys(x[0], x[1]);
                const uint32_t token = j * kStep + tsub * kAwTile + 8 * g + l16;
                if (g % 2 == 0 && token < seg) s_sum[hl * a.range + (t0 - r0) + (int32_t)token] += both;
            }
            wg_barrier();
        }
        t0 = pe;
        ++b;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < r1 - r0; i += kAwWaves * 64) {
        const float keep = s_keep[i];
        const int32_t slot = s_slot[i];
        if (keep < 0.f || slot < 0 || slot >= a.num_slots) continue;
        float x = 0.f;
#pragma unroll
        for (int u = 0; u < HW; ++u) x += s_sum[u * a.range + i];
        a.sums[slot] = keep > 0.f ? fmaf(keep, a.sums[slot], x) : x;
    }
}

esp_status launch_attn_weights(WeightsArgs a, bool q4, hipStream_t stream) {
    const int G = a.Hq / a.Hkv, QB = G <= 16 ? 16 / G : 1;
    const bool many = a.max_q > QB || G > 16, mask = a.q_pos != nullptr;
    const int groups = (a.Hkv + kAwWaves - 1) / kAwWaves;
    a.hw = (a.Hkv + groups - 1) / groups;
    const int64_t tiles = ((int64_t)a.total_tokens + kAwTile - 1) / kAwTile;
    // few tiles: fewer a workgroup, which takes requests one after another (32 queries, 32 / 2 heads, 64 lists of 30 or so, 78 against 32 us)
    a.nt = (int)std::min<int64_t>(kAwWaves / a.hw, (tiles + 511) / 512);
    // (Whole rows are read where nothing is masked alone: 64 requests of 1024 .. 131072, 32 / 8 heads in 4 bits, 127 us, by positions 178; over other
    // layouts positions cost little: 6 / 3 heads 93 and 106, 32 / 8 in bf16 333 and 336.)
    const bool by_rows = q4 && !many && !mask && a.Hkv % 4 == 0;
    if (by_rows) { a.hw = a.Hkv % 8 == 0 ? 8 : 4; a.nt = kAwWaves / a.hw; }
    // as many tokens as 512 workgroups get, in steps of the workgroup, no more than there is room for
    const int64_t step = (int64_t)a.nt * kAwTile, most = (by_rows ? kAwRowsSums : kAwSums) / a.hw / step * step;
    int64_t range = ((int64_t)a.total_tokens + 511) / 512;
    range = (range + step - 1) / step * step;
    a.range = (int32_t)(range > most ? most : range);
    const int64_t blocks = ((int64_t)a.total_tokens + a.range - 1) / a.range;
    // Two workgroups to a CU, of up to seven wavefronts with a tile (and one that brings queries: two to a SIMD each; with eight and one a CU had room
    // for one: 164 us for 143000 keys, of five in two even rounds 113, of seven 108).  With fewer tiles a head to a wavefront has more of the chip at
    // work (32 queries, 32 / 8 heads: 8 lists of 4096 or so 38 against 60 us, 16 of them 63 against 73, 64 of 1024 or so 101 against 76, 8 of 16384 150
    // against 90; 57 queries, 32 / 4 heads, 147 lists of 282 or so, 136 against 170); lists that leave most of a workgroup's tiles empty would undo it.
    // With one KV head there is nothing to lose: 57 queries of 32 heads, 147 lists of 282, 253 against 169 us; 32 queries, 64 lists of 30, 167 against
    // 39; one query, 256 of 50, 23 against 12.
    const int64_t each = std::min<int64_t>(kAwTiles, (tiles + 511) / 512);
    if (many && (a.Hkv == 1 || (tiles >= 512 * 4 && tiles * a.Hkv >= 512 * 32 && a.total_tokens / a.B >= 2 * kAwTile * each))) {
        a.nt = (int)each;
        a.range = a.nt * kAwTile;
        const dim3 grid = wide_grid((tiles + a.nt - 1) / a.nt);
#define ESP_AW_SPAN_LAUNCH(Q4, MASK) hipLaunchKernelGGL((attn_weights_span_kernel<Q4, MASK>), grid, dim3(64 * (a.nt + 1)), 0, stream, a)
        if (q4) { if (mask) ESP_AW_SPAN_LAUNCH(true, true); else ESP_AW_SPAN_LAUNCH(true, false); }
        else { if (mask) ESP_AW_SPAN_LAUNCH(false, true); else ESP_AW_SPAN_LAUNCH(false, false); }
#undef ESP_AW_SPAN_LAUNCH
        return check_launch("attn_weights_span_kernel");
    }
    if (by_rows) {
        if (a.hw == 8) hipLaunchKernelGGL(attn_weights_rows_kernel<8>, wide_grid(blocks), dim3(kAwWaves * 64), 0, stream, a);
        else hipLaunchKernelGGL(attn_weights_rows_kernel<4>, wide_grid(blocks), dim3(kAwWaves * 64), 0, stream, a);
        return check_launch("attn_weights_rows_kernel");
    }
#define ESP_AW_LAUNCH(Q4, MANY, MASK) \
    hipLaunchKernelGGL((attn_weights_kernel<Q4, MANY, MASK>), wide_grid(blocks), dim3(64 * a.hw * a.nt), 0, stream, a)
    if (q4) {
        if (many) { if (mask) ESP_AW_LAUNCH(true, true, true); else ESP_AW_LAUNCH(true, true, false); }
        else { if (mask) ESP_AW_LAUNCH(true, false, true); else ESP_AW_LAUNCH(true, false, false); }
    } else {
        if (many) { if (mask) ESP_AW_LAUNCH(false, true, true); else ESP_AW_LAUNCH(false, true, false); }
        else { if (mask) ESP_AW_LAUNCH(false, false, true); else ESP_AW_LAUNCH(false, false, false); }
    }
#undef ESP_AW_LAUNCH
    return check_launch("attn_weights_kernel");
}

}  // namespace esp
