// Host-side launchers of the sequence operators' kernels (include/ucd_seq.h has the formulas).  Descriptors have been
// checked and their strides filled in; every launcher only enqueues on `s` and returns the launch status.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "ucd_seq.h"

namespace ucd {

size_t group_norm_ws_bytes(const ucd_group_norm_t &d, int dir);
hipError_t group_norm_fwd(const ucd_group_norm_t &d, const void *x, const float *gamma, const float *beta_w, void *y,
                          float *stats, void *ws, hipStream_t s);
hipError_t group_norm_bwd(const ucd_group_norm_t &d, const void *x, const float *gamma, const float *beta_w,
                          const float *stats, const void *dy, void *dx, float *dgamma, float *dbeta, bool add, void *ws,
                          hipStream_t s);

struct CausalConvArgs {
    const void *x, *w;
    const float *bias;
    const int32_t *lengths, *slots;
    const void *state_in;
    void *state_out, *y;
    // Backward
    const void *dy, *dstate_out;
    void *dx;
    float *dw, *dbias;
    void *dstate_in;
};
size_t causal_conv_ws_bytes(const ucd_causal_conv_t &d);
hipError_t causal_conv_fwd(const ucd_causal_conv_t &d, const CausalConvArgs &a, hipStream_t s);
hipError_t causal_conv_bwd(const ucd_causal_conv_t &d, const CausalConvArgs &a, bool add, void *ws, hipStream_t s);
hipError_t causal_conv_step(const ucd_causal_conv_t &d, const CausalConvArgs &a, hipStream_t s);

size_t scan_ws_bytes(const ucd_scan_t &d, int dir);
size_t scan_saved_bytes(const ucd_scan_t &d);
hipError_t scan_fwd(const ucd_scan_t &d, const ucd_scan_in_t &in, const float *state_in, float *state_out, void *y,
                    float *saved, void *ws, hipStream_t s);
hipError_t scan_bwd(const ucd_scan_t &d, const ucd_scan_in_t &in, const void *dy, const float *dstate_out,
                    const float *saved, const ucd_scan_grad_t &g, bool add, void *ws, hipStream_t s);
hipError_t scan_step(const ucd_scan_t &d, const ucd_scan_in_t &in, float *state, void *y, hipStream_t s);

}  // namespace ucd
