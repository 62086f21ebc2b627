// 8-bit checkpoints: pack and unpack, one lane per chunk of eight values.
#include <hip/hip_runtime.h>

#include "rowops.h"
#include "rows.h"

namespace fo {
namespace {

constexpr int kThreads = 256;

// One wave per (row, slice of 64 chunks); a row has slices of its padded length.
template <int DT, int FMT>
__global__ __launch_bounds__(kThreads) void pack_kernel(const PackArgs a, uint32_t slices) {
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * (kThreads / 64) + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t i = unit / slices;
    if (i >= a.M) return;
    const uint32_t s = unit - (uint32_t)i * slices;
    const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK;
    const uint16_t* row = a.x + i * a.ldx;
    uint8_t* packed = a.packed + i * blocks * FO_PACK_BLOCK;
    uint8_t* scales = a.scales + i * blocks;
    const int c = (int)s * 64 + lane;
    if (c < a.N / FO_PACK_BLOCK * 4) {
        float f[8];
        widen<DT>(load8(row + 8 * (int64_t)c), f);
        pack_chunk<DT, FMT>(f, c, packed, scales);
    }
    if (s == slices - 1 && a.N % FO_PACK_BLOCK) pack_last<DT, FMT>(row, a.N, lane, packed, scales);
}

template <int DT, int FMT>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const PackArgs a, uint32_t slices) {
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * (kThreads / 64) + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t i = unit / slices;
    if (i >= a.M) return;
    const uint32_t s = unit - (uint32_t)i * slices;
    const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK;
    uint16_t* row = a.x + i * a.ldx;
    const uint8_t* packed = a.packed + i * blocks * FO_PACK_BLOCK;
    const uint8_t* scales = a.scales + i * blocks;
    const int c = (int)s * 64 + lane;
    const int full = (int)(a.N >> 3), tail = (int)(a.N & 7);
    if (c < full) {
        float f[8];
        decode8<FMT>(*reinterpret_cast<const u32x2_t*>(packed + 8 * (int64_t)c), scale_of(scales[c >> 2]), f);
        store8(row + 8 * (int64_t)c, narrow<DT>(f));
    }
    if (s == slices - 1 && lane < tail) {
        const int64_t n = a.N - tail + lane;
        row[n] = (uint16_t)from_f32<DT>(decode1<FMT>(packed[n], scale_of(scales[n / FO_PACK_BLOCK])));
    }
}

template <typename F>
hipError_t for_types(int dtype, int format, F f) {
    if (dtype == FO_FP16) {
        if (format == FO_PACK_INT8) f(std::integral_constant<int, FO_FP16>(), std::integral_constant<int, FO_PACK_INT8>());
        else f(std::integral_constant<int, FO_FP16>(), std::integral_constant<int, FO_PACK_E4M3>());
    } else {
        if (format == FO_PACK_INT8) f(std::integral_constant<int, FO_BF16>(), std::integral_constant<int, FO_PACK_INT8>());
        else f(std::integral_constant<int, FO_BF16>(), std::integral_constant<int, FO_PACK_E4M3>());
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_pack(int dtype, int format, const PackArgs& a, hipStream_t s) {
    const uint32_t slices = (uint32_t)((a.N / 8 + 63) / 64 ? (a.N / 8 + 63) / 64 : 1);
    const dim3 g((uint32_t)((a.M * slices + 3) / 4)), b(kThreads);
    return for_types(dtype, format, [&](auto dt, auto fmt) {
        hipLaunchKernelGGL((pack_kernel<decltype(dt)::value, decltype(fmt)::value>), g, b, 0, s, a, slices);
    });
}

hipError_t launch_unpack(int dtype, int format, const PackArgs& a, hipStream_t s) {
    const uint32_t slices = (uint32_t)((a.N / 8 + 63) / 64 ? (a.N / 8 + 63) / 64 : 1);
    const dim3 g((uint32_t)((a.M * slices + 3) / 4)), b(kThreads);
    return for_types(dtype, format, [&](auto dt, auto fmt) {
        hipLaunchKernelGGL((unpack_kernel<decltype(dt)::value, decltype(fmt)::value>), g, b, 0, s, a, slices);
    });
}

}  // namespace fo
