// Launchers of the kernels for normalised rows, 8-bit codes, their products, and clipped gradient steps. Arguments are
// checked by the entry points (varco_scaled.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "varco.h"

struct NormFwdArgs {
    int64_t n_rows;
    int32_t width;
    const void* x;
    int64_t ldx;
    const void* residual;
    int64_t ldr;
    const float* gain;
    float eps;
    void* total;
    int64_t ldt;
    void* y;
    int64_t ldy;
    uint8_t* codes;
    uint8_t* scales;
    float* inv_rms;
};
struct NormBwdArgs {
    int64_t n_rows;
    int32_t width;
    const void* dy;
    int64_t lddy;
    const void* u;
    int64_t ldu;
    const float* gain;
    const float* inv_rms;
    const void* dtotal;
    int64_t lddt;
    void* dx;
    int64_t lddx;
    float* dgain;
    int32_t accumulate;
    float* partial;            // varco_norm_blocks(..) x width floats where that is above 1
};
hipError_t varco_launch_rms_norm_fwd(int dtype, const NormFwdArgs& a, hipStream_t stream);
int32_t varco_norm_blocks(int dtype, int64_t n_rows, int32_t width);       // workgroups of the backward kernel
hipError_t varco_launch_rms_norm_bwd(int dtype, const NormBwdArgs& a, hipStream_t stream);

hipError_t varco_launch_quantize_rows(int dtype, int64_t n_rows, int32_t width, const void* x, int64_t ldx, const void* gate, int64_t ldg,
                                      uint8_t* codes, uint8_t* scales, hipStream_t stream);
hipError_t varco_launch_quantize_weights(int32_t n_in, int32_t n_out, const float* h, int64_t ldh, uint8_t* turned, uint8_t* turned_scales,
                                         uint8_t* codes, uint8_t* scales, hipStream_t stream);

struct ScaledArgs {
    int64_t n_rows;
    int32_t n_in, n_out;
    const uint8_t* x;
    const uint8_t* x_scales;
    const uint8_t* w;             // [n_out][code_ld(n_in)]
    const uint8_t* w_scales;      // [blocks of n_out][scale_ld(n_in)]
    void* c;
    int64_t ldc;
    int32_t accumulate, relu;
};
hipError_t varco_launch_scaled_transform(int dtype, const ScaledArgs& a, hipStream_t stream);

struct ScaledWeightArgs {
    int64_t n_rows;
    int32_t n_in, n_out;
    const uint8_t* y;
    const uint8_t* y_scales;
    const uint8_t* d;
    const uint8_t* d_scales;
    float* dh;
    int64_t ldh;
    int32_t accumulate;
    float* partial;               // varco_scaled_weight_floats(..)
};
int64_t varco_scaled_weight_floats(int64_t n_rows, int32_t n_in, int32_t n_out);
hipError_t varco_launch_scaled_bwd_weight(const ScaledWeightArgs& a, hipStream_t stream);

// Sum of the squares of all elements in fp64: `blocks` partial sums, then norm and factor in out[0], out[1] by whoever reads them.
int32_t varco_clip_partials(int32_t n_tensors, const int64_t* sizes);
hipError_t varco_launch_square_sums(int dtype, int32_t n_tensors, const void* const* grads, const int64_t* sizes, double* partial,
                                    hipStream_t stream);
hipError_t varco_launch_norm_out(const double* partial, int32_t n_partial, float max_norm, float* out, hipStream_t stream);
hipError_t varco_launch_clip(int dtype, int32_t n_tensors, const void* const* grads, void* const* into, const int64_t* sizes,
                             const double* partial, int32_t n_partial, float max_norm, float* out, hipStream_t stream);
hipError_t varco_launch_sgd_clipped(int32_t n_tensors, void* const* w, const void* const* dw, const int64_t* sizes, float lr,
                                    const double* partial, int32_t n_partial, float max_norm, float* out, hipStream_t stream);
