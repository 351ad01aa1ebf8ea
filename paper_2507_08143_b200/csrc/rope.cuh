// Arguments of the norm and rotation kernel.
#pragma once
#include "common.cuh"

namespace compactor {

struct RopeArgs {
    long long tokens;
    int q_heads, k_heads;
    int rotary, interleaved;                   // channels that are rotated
    float eps;
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* q_weight;             // [128] or null: no norm
    const __nv_bfloat16* k_weight;
    const int* positions;                      // [tokens]
    const float* inv_freq;                     // [rotary / 2]
    __nv_bfloat16* q_out;
    __nv_bfloat16* k_out;
    __nv_bfloat16* k_plain;                    // keys before the rotation, or null
    long long q_token, q_head, k_token, k_head, qo_token, qo_head, ko_token, ko_head, p_token, p_head;     // strides in elements
};
cudaError_t launch_rope(const RopeArgs& a, int sm_count, cudaStream_t stream);

}  // namespace compactor
