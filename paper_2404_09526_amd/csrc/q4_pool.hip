// esp_kv_append_q4, esp_kv_gather_q4: rows on their way into and out of the pool in 4 bits.  Bound by the memory: a head is 256 bytes dense
// and 68 in the pool.  16 lanes have a head of K and of V, 8 elements each: a block of 32 is four neighbouring lanes.  32768 rows of 8 heads, a quarter
// of them kept, in 13 us, 65536 rows back in 49: 6.2 TB/s read and written (a copy of 4 GiB: 4.8).
#include "q4.h"

namespace esp {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t largest_of(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// 8 elements of a lane (with those of its three neighbours: a block) to codes, and the block's scale
__device__ __forceinline__ uint32_t q4_from_bf16(const uint4& w, uint32_t& scale_byte) {
    constexpr uint32_t kMagnitude = 0x7fff7fffu;
    uint32_t m = largest_of(largest_of(w.x & kMagnitude, w.y & kMagnitude), largest_of(w.z & kMagnitude, w.w & kMagnitude));
    m = max(m & 0xffffu, m >> 16);
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));   // lane ^ 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));   // lane ^ 2
    scale_byte = q4_scale_byte(m);
    if (scale_byte == 255u) return 0;
    const float scale = q4_scale(scale_byte, 0);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w.x), scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w.y), scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w.z), scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w.w), scale, 3);
    return codes;
}

__global__ __launch_bounds__(256) void q4_append_kernel(const char* __restrict__ k, const char* __restrict__ v, int64_t k_stride, int64_t v_stride,
                                                        const int32_t* __restrict__ slot_idx, uint32_t heads, uint32_t Hkv, char* __restrict__ k_pool,
                                                        char* __restrict__ v_pool, int64_t slot_bytes, int64_t num_slots) {
    const int64_t at = row_block() * 16 + (threadIdx.x >> 4);
    if (at >= heads) return;
    const uint32_t t = (uint32_t)at / Hkv, h = (uint32_t)at - t * Hkv;
    const int seg = threadIdx.x & 15;
    const int32_t slot = slot_idx[t];
    if (slot < 0 || slot >= num_slots) return;                      // (all 16 lanes of the head)
    const uint4 kw = load_once((const uint4*)(k + 2 * (t * k_stride + h * kHeadDim)) + seg);
    const uint4 vw = load_once((const uint4*)(v + 2 * (t * v_stride + h * kHeadDim)) + seg);
    const int64_t row = slot * slot_bytes + (int64_t)h * kQ4Head;
    uint32_t ks, vs;
    const uint32_t kc = q4_from_bf16(kw, ks), vc = q4_from_bf16(vw, vs);
    *(uint32_t*)(k_pool + row + 4 * seg) = kc;
    *(uint32_t*)(v_pool + row + 4 * seg) = vc;
    if ((seg & 3) == 0) {
        k_pool[row + kQ4Codes + (seg >> 2)] = (char)ks;
        v_pool[row + kQ4Codes + (seg >> 2)] = (char)vs;
    }
}

// the inverse view: rows of the pool in the order of a slot list, dense; a slot outside the pool gives a row of zeros
__global__ __launch_bounds__(256) void q4_gather_kernel(const char* __restrict__ k_pool, const char* __restrict__ v_pool, const int32_t* __restrict__ slot_idx,
                                                        uint32_t heads, uint32_t Hkv, int64_t slot_bytes, int64_t num_slots, uint4* __restrict__ k,
                                                        uint4* __restrict__ v) {
    const int64_t at = row_block() * 16 + (threadIdx.x >> 4);
    if (at >= heads) return;
    const uint32_t t = (uint32_t)at / Hkv, h = (uint32_t)at - t * Hkv;
    const int seg = threadIdx.x & 15;
    const int32_t slot = slot_idx[t];
    uint4 kk = make_uint4(0u, 0u, 0u, 0u), vv = kk;
    if (slot >= 0 && slot < num_slots) {
        const int64_t row = slot * slot_bytes + (int64_t)h * kQ4Head;
        const uint32_t kc = *(const uint32_t*)(k_pool + row + 4 * seg), vc = *(const uint32_t*)(v_pool + row + 4 * seg);
        const uint32_t ks = (uint8_t)k_pool[row + kQ4Codes + (seg >> 2)], vs = (uint8_t)v_pool[row + kQ4Codes + (seg >> 2)];
        kk = q4_to_bf16(kc, q4_scale(ks, 0));
        vv = q4_to_bf16(vc, q4_scale(vs, 0));
    }
    store_once(k + at * 16 + seg, kk);
    store_once(v + at * 16 + seg, vv);
}

esp_status launch_kv_append_q4(const void* k, const void* v, int64_t k_stride, int64_t v_stride, const int32_t* slot_idx, int32_t T, int32_t Hkv, void* k_pool,
                               void* v_pool, int64_t slot_bytes, int64_t num_slots, hipStream_t stream) {
    const int64_t heads = (int64_t)T * Hkv;
    if (heads > INT32_MAX) return fail(ESP_ERR_INVALID_ARG, "append (4 bits): too many rows for one launch");
    hipLaunchKernelGGL(q4_append_kernel, row_grid((heads + 15) / 16), dim3(256), 0, stream, (const char*)k, (const char*)v, k_stride, v_stride, slot_idx,
                       (uint32_t)heads, (uint32_t)Hkv, (char*)k_pool, (char*)v_pool, slot_bytes, num_slots);
    return check_launch("q4_append_kernel");
}

esp_status launch_kv_gather_q4(const void* k_pool, const void* v_pool, int64_t slot_bytes, const int32_t* slot_idx, int32_t T, int64_t num_slots, int32_t Hkv,
                               void* k, void* v, hipStream_t stream) {
    const int64_t heads = (int64_t)T * Hkv;
    if (heads > INT32_MAX) return fail(ESP_ERR_INVALID_ARG, "gather (4 bits): too many rows for one launch");
    hipLaunchKernelGGL(q4_gather_kernel, row_grid((heads + 15) / 16), dim3(256), 0, stream, (const char*)k_pool, (const char*)v_pool, slot_idx, (uint32_t)heads,
                       (uint32_t)Hkv, slot_bytes, num_slots, (uint4*)k, (uint4*)v);
    return check_launch("q4_gather_kernel");
}

}  // namespace esp
