// Launch interfaces of the 8-bit operators (internal): rows in 8-bit integers, the
// RMS norm of a sum, products of 8-bit matrices.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fo_internal.h"
#include "int8_form.h"

namespace fo {

struct Rows8Args {
    const uint16_t* x;          // [M] rows, ldx apart
    const uint16_t* residual;   // norm: or null
    const uint16_t* gamma;      // norm: [N] or null
    uint16_t* h;                // norm: or null
    uint16_t* y;                // norm: or null
    float* rstd;                // norm: [M] or null
    int8_t* codes;              // [M] rows, ldc apart; norm: or null, with scales
    float* scales;              // [M]
    int64_t M, N, ldx, ldr, ldh, ldy, ldc;
    float eps;
    float scale;                // norm: the largest power of two with N * scale <= 1
};
hipError_t launch_quantize(int dtype, const Rows8Args& a, hipStream_t s);
hipError_t launch_norm_add_forward(int dtype, const Rows8Args& a, hipStream_t s);

struct NormAddArgs {
    const uint16_t* dy;
    const uint16_t* dh;         // or null
    const uint16_t* h;
    const uint16_t* gamma;      // [N] or null
    const float* rstd;          // [M]
    uint16_t* dx;               // or null
    float* partial;             // [blocks][2][norm_partial_cols(N)] sums of dy * h * rstd (the first of the two), or null
    float* dots;                // wide rows: [M]
    int64_t M, N, lddy, lddh, ldh, lddx;
};
// The sums over rows go to a.partial; then dgamma (or null) is their sum.
hipError_t launch_norm_add_backward(int dtype, const NormAddArgs& a, float* dgamma, hipStream_t s);

int64_t int8_workspace_bytes(int64_t M, int64_t N, int64_t K);
// Whether a launch takes the product (work-items are counted in 32 bits).
bool int8_launchable(const Int8Args& a, bool experts);
// `blocks` tiles of 256 x 256 (K > 0).
hipError_t launch_int8_tile(int dtype, bool experts, uint32_t blocks, const Int8Args& a, hipStream_t s);
hipError_t launch_int8_product(int dtype, const Int8Args& a, hipStream_t s);
hipError_t launch_int8_experts(int dtype, const Int8Args& a, hipStream_t s);

}  // namespace fo
