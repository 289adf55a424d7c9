// libmmvseg: the gated delta rule over the prompts of a ragged batch and for single tokens (include/mmvseg.h).
#include <hip/hip_runtime.h>
#include <stdint.h>


#include "mmvseg.h"

#include "values.h"
#include "call_checks.h"
#include "delta.h"
#include "delta_host.h"

extern "C" {

size_t mmv_delta_attention_workspace_bytes(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t dk, uint32_t dv) {
    if (!delta_sizes(n, tokens, heads, heads, dk, dv)) return 0;
    return delta_workspace(n, tokens, heads, dk, dv);
}

mmv_status mmv_delta_attention(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t k_heads, uint32_t dk, uint32_t dv,
                               const void *d_q, uint64_t q_stride, const void *d_k, uint64_t k_stride, const void *d_v, uint64_t v_stride,
                               mmv_type type, const int32_t *d_offsets, const float *d_log_decay, const float *d_beta, float scale,
                               const float *d_state_in, float *d_state_out, uint64_t states, const int32_t *d_state_index,
                               void *d_out, void *d_ws, size_t ws_bytes, void *hip_stream) {
    if (!delta_sizes(n, tokens, heads, k_heads, dk, dv)) return MMV_ERR_INVALID_ARG;
    DeltaParams P = {};
    if (const mmv_status st = delta_params(P, n, tokens, heads, k_heads, dk, dv, d_q, q_stride, d_k, k_stride, d_v, v_stride, type, d_log_decay, d_beta, scale,
                                           d_state_in, d_state_out, states, d_state_index, d_out))
        return st;
    if (n == 0) return MMV_OK;
    if (!d_offsets) return MMV_ERR_NULL;
    if (!aligned_to(d_offsets, 4)) return MMV_ERR_INVALID_ARG;
    if (const mmv_status st = check_workspace(d_ws, ws_bytes, delta_workspace(n, tokens, heads, dk, dv))) return st;
    P.offsets = d_offsets;
    return delta_call(P, type, d_ws, (hipStream_t)hip_stream);
}

mmv_status mmv_delta_step(uint64_t n, uint32_t heads, uint32_t k_heads, uint32_t dk, uint32_t dv,
                          const void *d_q, uint64_t q_stride, const void *d_k, uint64_t k_stride, const void *d_v, uint64_t v_stride,
                          mmv_type type, const float *d_log_decay, const float *d_beta, float scale,
                          const float *d_state_in, float *d_state_out, uint64_t states, const int32_t *d_state_index,
                          void *d_out, void *hip_stream) {
    if (!delta_sizes(n, n, heads, k_heads, dk, dv)) return MMV_ERR_INVALID_ARG;
    DeltaParams P = {};
    if (const mmv_status st = delta_params(P, n, n, heads, k_heads, dk, dv, d_q, q_stride, d_k, k_stride, d_v, v_stride, type, d_log_decay, d_beta, scale, d_state_in,
                                           d_state_out, states, d_state_index, d_out))
        return st;
    if (n == 0) return MMV_OK;
    return delta_step_call(P, type, (hipStream_t)hip_stream);
}

}  // extern "C"
