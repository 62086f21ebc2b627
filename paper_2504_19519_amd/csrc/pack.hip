// 8-bit checkpoints: pack and unpack, bound by memory.
//
// A wave takes kAhead times 64 chunks of eight values of one row, all of their loads
// in flight together; four lanes share a block's scale. The 16-bit side goes past the
// caches in both directions, so that the codes stay: 8192x14336 bf16 to int8 and back
// 59 + 51 us (6.0 and 6.9 TB/s; with cached loads 62 + 55, cached stores too 77 + 60,
// one chunk per lane and cached 71 + 59).
#include <hip/hip_runtime.h>

#include "rowops.h"
#include "rows.h"

namespace fo {
namespace {

constexpr int kThreads = 256;

constexpr int kAhead = 2, kSlice = 64 * kAhead;      // chunks of one wave

// This wave's row and first chunk. 32 bits: the host sees to the number of waves.
struct Slice {
    int64_t i;
    int c0;
    bool last;
};
__device__ __forceinline__ Slice slice_of(uint32_t slices) {
    const uint32_t unit = blockIdx.x * (kThreads / 64) + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t i = unit / slices, s = unit - i * slices;
    return {(int64_t)i, (int)(s * kSlice), s == slices - 1};
}

template <int DT, int FMT>
__global__ __launch_bounds__(kThreads) void pack_kernel(const PackArgs a, uint32_t slices) {
    const int lane = threadIdx.x & 63;
    const Slice s = slice_of(slices);
    if (s.i >= a.M) return;
    const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK;
    const int whole = (int)(a.N / FO_PACK_BLOCK) * 4;           // chunks of whole blocks
    const uint16_t* row = a.x + s.i * a.ldx;
    uint8_t* packed = a.packed + s.i * blocks * FO_PACK_BLOCK;
    uint8_t* scales = a.scales + s.i * blocks;
    u32x4_t v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int c = s.c0 + 64 * j + lane;
        if (c < whole) v[j] = stream_load8(row + 8 * (int64_t)c);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int c = s.c0 + 64 * j + lane;
        if (c < whole) {
            float f[8];
            widen<DT>(v[j], f);
            pack_chunk<DT, FMT>(f, c, packed, scales);
        }
    }
    if (s.last && a.N % FO_PACK_BLOCK) pack_last<DT, FMT>(row, a.N, lane, packed, scales);
}

template <int DT, int FMT>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const PackArgs a, uint32_t slices) {
    const int lane = threadIdx.x & 63;
    const Slice s = slice_of(slices);
    if (s.i >= a.M) return;
    const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK;
    const int full = (int)(a.N >> 3), tail = (int)(a.N & 7);
    uint16_t* row = a.x + s.i * a.ldx;
    const uint8_t* packed = a.packed + s.i * blocks * FO_PACK_BLOCK;
    const uint8_t* scales = a.scales + s.i * blocks;
    u32x2_t code[kAhead];
    uint32_t scale[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int c = s.c0 + 64 * j + lane;
        if (c < full) {
            code[j] = *reinterpret_cast<const u32x2_t*>(packed + 8 * (int64_t)c);
            scale[j] = scales[c >> 2];
        }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int c = s.c0 + 64 * j + lane;
        if (c < full) {
            float f[8];
            decode8<FMT>(code[j], scale_of(scale[j]), f);
            stream8(row + 8 * (int64_t)c, narrow<DT>(f));
        }
    }
    if (s.last && lane < tail) {
        const int64_t n = a.N - tail + lane;
        row[n] = (uint16_t)from_f32<DT>(decode1<FMT>(packed[n], scale_of(scales[n / FO_PACK_BLOCK])));
    }
}

uint32_t slices_of(int64_t N) { return (uint32_t)(N / 8 > kSlice ? (N / 8 + kSlice - 1) / kSlice : 1); }

uint32_t workgroups(const PackArgs& a) { return (uint32_t)((a.M * slices_of(a.N) + kThreads / 64 - 1) / (kThreads / 64)); }

}  // namespace

hipError_t launch_pack(int dtype, int format, const PackArgs& a, hipStream_t s) {
    const bool int8 = format == FO_PACK_INT8;
    return launch(dtype == FO_FP16 ? (int8 ? pack_kernel<FO_FP16, FO_PACK_INT8> : pack_kernel<FO_FP16, FO_PACK_E4M3>)
                                   : (int8 ? pack_kernel<FO_BF16, FO_PACK_INT8> : pack_kernel<FO_BF16, FO_PACK_E4M3>),
                  workgroups(a), kThreads, s, a, slices_of(a.N));
}

hipError_t launch_unpack(int dtype, int format, const PackArgs& a, hipStream_t s) {
    const bool int8 = format == FO_PACK_INT8;
    return launch(dtype == FO_FP16 ? (int8 ? unpack_kernel<FO_FP16, FO_PACK_INT8> : unpack_kernel<FO_FP16, FO_PACK_E4M3>)
                                   : (int8 ? unpack_kernel<FO_BF16, FO_PACK_INT8> : unpack_kernel<FO_BF16, FO_PACK_E4M3>),
                  workgroups(a), kThreads, s, a, slices_of(a.N));
}

}  // namespace fo
