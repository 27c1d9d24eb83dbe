// esp_qk_norm_rope_append: what a layer's new queries and keys go through between their projection and attention, in one pass.  For each
// head's 128 elements, y = x / sqrt(mean(x^2) + eps) * w (where there are weights), then the rotation of the first `rot` of them by
// the angles pos * inv_freq: a pair (a, b) becomes (a cos - b sin, b cos + a sin), pairs being elements i and i + rot / 2, or neighbours.
// K and V leave for their pool slots (and as dense rows where asked).  A row is read and written once and rounded once, so the call is bound by
// the memory: 2 x 256 bytes a head.
// 16 lanes have a head's row, 16 bytes each, a wavefront four rows a load.  A wavefront works for one token: sine and cosine of a
// lane's elements are taken once for all of the token's heads.
// Measured: 32768 tokens, 32 / 8 heads, K and V as dense rows and a quarter of them into the pool, 839 MB, 173 us: 4.85 TB/s, what a copy of 2 GiB reaches on this card (4.80).
#include "decode_merge.h"
#include "rotate.h"

namespace esp {

constexpr int kRotThreads = 256;
constexpr int kRotWaves = 4096;                   // that a call asks for where it can: 16 a CU

// Sine and cosine of the angle pos * inv_freq.  In turns, and reduced to half a turn, in 64 bits: at position 2^20 an angle in 32 bits would be off by a
// tenth of a radian.
__device__ __forceinline__ void turn_of(int32_t pos, float inv_freq, float& s, float& c) {
    const double turns = (double)pos * ((double)inv_freq * 0.15915494309189533577);
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
}

template <bool NEIGHBOURS>
__global__ __launch_bounds__(kRotThreads) void rotate_kernel(RotateArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = row_block() * (kRotThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t token = unit / a.parts;
    if (token >= a.T) return;
    const int part = (int)(unit - token * a.parts);
    const int seg = lane & 15, sub = lane >> 4, e0 = 8 * seg;
    const int heads = a.Hq + 2 * a.Hkv, h_end = min(heads, (part + 1) * a.part_heads);
    const int half = a.rot >> 1;
    const int32_t slot = a.slot_idx ? a.slot_idx[token] : -1;
    const bool kept = slot >= 0 && slot < a.num_slots;

    float sn[8], cs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { sn[e] = 0.f; cs[e] = 1.f; }
    const int partner = e0 >= a.rot ? lane : e0 < half ? lane + (half >> 3) : lane - (half >> 3);   // (within the 16 lanes)
    if (a.rot > 0 && part * a.part_heads < a.Hq + a.Hkv) {
        const int32_t pos = a.pos[token];
        if constexpr (NEIGHBOURS) {
#pragma unroll
            for (int e = 0; e < 8; e += 2)
                if (e0 + e < a.rot) {
                    turn_of(pos, a.inv_freq[(e0 + e) >> 1], sn[e], cs[e]);
                    cs[e + 1] = cs[e]; sn[e + 1] = sn[e]; sn[e] = -sn[e];
                }
        } else if (e0 < a.rot) {
            const int f0 = e0 < half ? e0 : e0 - half;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                turn_of(pos, a.inv_freq[f0 + e], sn[e], cs[e]);
                if (e0 < half) sn[e] = -sn[e];
            }
        }
    }
    for (int h0 = part * a.part_heads; h0 < h_end; h0 += 4) {
        const int h = h0 + sub;
        if (h >= h_end) continue;
        const int kind = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2, at = kind == 0 ? h : kind == 1 ? h - a.Hq : h - a.Hq - a.Hkv;
        char* const dense = kind == 0 ? a.q_out + 2 * (token * a.q_out_stride + at * kHeadDim) :
                            (kind == 1 ? a.k_out : a.v_out) + 2 * ((token * a.Hkv + at) * kHeadDim);
        const bool to_dense = kind == 0 || (kind == 1 ? a.k_out : a.v_out) != nullptr, to_pool = kind != 0 && kept;
        if (!to_dense && !to_pool) continue;
        const char* const src = (kind == 0 ? a.q + 2 * token * a.q_stride : kind == 1 ? a.k + 2 * token * a.k_stride : a.v + 2 * token * a.v_stride) + at * (2 * kHeadDim);
        uint4 w = load_once((const uint4*)src + seg);
        if (kind != 2) {
            float x[8], y[8];
            unpack8(w, x);
            const char* const weight = kind == 0 ? a.q_weight : a.k_weight;
            if (weight) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
                const float r = 1.0f / sqrtf(row16_sum(sum) * (1.f / kHeadDim) + a.eps);
                float g[8];
                unpack8(((const uint4*)weight)[seg], g);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= r * g[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float other = NEIGHBOURS ? x[e ^ 1] : __shfl(x[e], partner);
                y[e] = e0 + (NEIGHBOURS ? e : 0) < a.rot ? fmaf(x[e], cs[e], other * sn[e]) : x[e];   // (past them nothing of another element, not even 0 times it)
            }
            w = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
        }
        if (to_dense) ((uint4*)dense)[seg] = w;
        if (to_pool) ((uint4*)((kind == 1 ? a.k_pool : a.v_pool) + 2 * (((int64_t)slot * a.Hkv + at) * kHeadDim)))[seg] = w;
    }
}

esp_status launch_rotate(RotateArgs a, int32_t neighbours, hipStream_t stream) {
    const int64_t heads = (int64_t)a.Hq + 2 * (int64_t)a.Hkv;
    if (heads > INT32_MAX / 2) return fail(ESP_ERR_UNSUPPORTED, "norm and rotation: too many heads");
    // A token's heads by one wavefront, four at a time, as long as there are tokens enough; by several, of which each takes sine and cosine for
    // itself, where it is a chain of loads: 64 tokens, 32 / 8 heads, 12.0 us with one, 4.5 with twelve.
    const int64_t fours = (heads + 3) / 4, parts = a.T > 0 ? kRotWaves / a.T : 1;
    a.parts = (int32_t)(parts < 1 ? 1 : parts > fours ? fours : parts);
    a.part_heads = (int32_t)((fours + a.parts - 1) / a.parts * 4);
    a.parts = (int32_t)((fours * 4 + a.part_heads - 1) / a.part_heads);
    const int64_t blocks = (a.T * (int64_t)a.parts + kRotThreads / 64 - 1) / (kRotThreads / 64);
    if (blocks > kGridMost) return fail(ESP_ERR_INVALID_ARG, "norm and rotation: too many rows for one launch");
    if (neighbours) hipLaunchKernelGGL(rotate_kernel<true>, row_grid(blocks), dim3(kRotThreads), 0, stream, a);
    else hipLaunchKernelGGL(rotate_kernel<false>, row_grid(blocks), dim3(kRotThreads), 0, stream, a);
    return check_launch("rotate_kernel");
}

}  // namespace esp
