// Launch interfaces of the row operators (internal): layer norm / RMS norm with
// its backward pass, 8-bit checkpoints, tokens sorted by expert and combined.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fo_internal.h"

namespace fo {

// Launches a kernel by one call of the runtime, which also says whether it went well
// (the launch syntax is three calls, and its error a fourth that would report earlier
// ones too).
template <typename... Params, typename... Args>
hipError_t launch(void (*kernel)(Params...), dim3 grid, dim3 threads, hipStream_t s, const Args&... args) {
    return [&](Params... params) {
        void* at[] = {static_cast<void*>(&params)...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, threads, at, 0, s);
    }(args...);
}

// A checkpoint of a matrix with N columns: blocks of 32 along a row.
inline int64_t pack_blocks(int64_t N) { return (N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK; }

struct NormArgs {
    const uint16_t* x;          // [M] rows, ldx apart; backward: null with a checkpoint
    const uint16_t* gamma;      // [N] or null
    const uint16_t* beta;       // [N] or null (forward)
    uint16_t* y;                // forward
    const uint16_t* dy;         // backward
    uint16_t* dx;               // backward, or null
    float* mean;                // [M] (layer norm) or null
    float* rstd;                // [M]
    uint8_t* packed;            // checkpoint, or null
    uint8_t* scales;
    float* partial;             // backward: [blocks][2][norm_partial_cols(N)] sums of dy * h and dy, or null
    float* dots;                // backward, wide rows: [M][2] (norm_dots_bytes)
    int64_t M, N, ldx, ldy, lddx;
    float eps;
    float scale;                // forward: the largest power of two with N * scale <= 1
    int32_t layer;              // 1: layer norm, 0: RMS norm
    int32_t format;             // of the checkpoint
    int32_t with_beta;          // backward: the sums of dy are wanted
};

// The kernel form of a norm's launch: threads of a row, chunks of eight values
// per thread, rows in flight per workgroup.
struct NormForm {
    int32_t threads, chunks, rows;
    uint32_t blocks;
};
constexpr int64_t kMaxNormCols = 32768;
// Columns of the partial sums: whole chunks, so that every row of them is 16-byte aligned.
FO_HD inline int64_t norm_partial_cols(int64_t N) { return (N + 7) / 8 * 8; }
NormForm norm_forward_form(int64_t M, int64_t N);
NormForm norm_backward_form(int64_t M, int64_t N);
// Workspace of rows too wide to be held, behind the partial sums.
int64_t norm_dots_bytes(int64_t M, int64_t N);
hipError_t launch_norm_forward(int dtype, const NormArgs& a, hipStream_t s);
// The sums over rows go to a.partial; then dgamma and dbeta (each or null) are their sums.
hipError_t launch_norm_backward(int dtype, const NormArgs& a, float* dgamma, float* dbeta, hipStream_t s);

struct PackArgs {
    uint16_t* x;                // [M] rows, ldx apart
    uint8_t* packed;
    uint8_t* scales;
    int64_t M, N, ldx;
};
hipError_t launch_pack(int dtype, int format, const PackArgs& a, hipStream_t s);
hipError_t launch_unpack(int dtype, int format, const PackArgs& a, hipStream_t s);

constexpr int kMaxExperts = FO_ROUTE_MAX_EXPERTS;
struct SortArgs {
    const void* ids;            // [pairs], of id_bytes each
    int64_t pairs;
    int32_t experts, align, id_bytes;
    int32_t* offsets;           // [experts + 1]
    int32_t* counts;            // [experts]
    int32_t* slot_of;           // [pairs]
    int32_t* pair_of;           // [capacity] or null
    int32_t* hist;              // [blocks][experts], more than one block only
};
int64_t sort_blocks(int64_t pairs);
hipError_t launch_sort(const SortArgs& a, hipStream_t s);

struct RouteArgs {
    const uint16_t* x;          // permute: [T, H]; combine's backward: dout
    uint16_t* rows;             // permute: out; combine: in; backward: in, or null with a checkpoint
    uint16_t* out;              // combine: [T, H]; backward: drows, or null
    const int32_t* slot_of;     // [T, K]
    const float* weights;       // [T, K] or null
    float* dweights;            // [T, K] or null
    const int32_t* offsets;     // [E + 1], with counts: rows between an expert's last and the
    const int32_t* counts;      //   next one's first are zeroed; or null
    uint8_t* packed;            // checkpoint of rows, or null
    uint8_t* scales;
    int64_t H, ldx, ldr, ldo;
    int32_t T, K, E, capacity, format;
};
hipError_t launch_permute(const RouteArgs& a, hipStream_t s);
hipError_t launch_combine(int dtype, const RouteArgs& a, hipStream_t s);
hipError_t launch_combine_backward(int dtype, const RouteArgs& a, hipStream_t s);

}  // namespace fo
