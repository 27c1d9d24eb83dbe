// Arguments of the norm and rotation of new queries and keys (rotate.hip).
#pragma once
#include "esp_common.h"

namespace esp {

struct RotateArgs {
    const char* q; const char* k; const char* v;
    int64_t q_stride, k_stride, v_stride, q_out_stride;   // elements from a token's first head to the next token's
    const int32_t* pos; const float* inv_freq;
    const char* q_weight; const char* k_weight;           // null: no norm
    char* q_out; char* k_out; char* v_out;                // k_out, v_out: null where no dense rows are asked for
    const int32_t* slot_idx; char* k_pool; char* v_pool; int64_t num_slots;
    int64_t T;
    int32_t Hq, Hkv, rot;
    float eps;
    int32_t parts, part_heads;                            // a token's heads (q, then k, then v) in so many parts, a wavefront each
};
esp_status launch_rotate(RotateArgs a, int32_t neighbours, hipStream_t stream);

}  // namespace esp
