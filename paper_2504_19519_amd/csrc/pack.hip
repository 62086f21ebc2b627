// 8-bit checkpoints: pack and unpack, bound by memory.
//
// Four lanes share a block of 32 values and its scale, a chunk of eight each; a
// thread takes kAhead chunks, a workgroup's width apart, with their loads in flight
// together. The chunks of all rows are numbered through, so that short rows fill
// waves as long ones do; rows without gaps between them are one row.
//
// The 16-bit side goes past the caches in both directions, so that the codes stay:
// 8192x14336 bf16 to int8 and back 59 + 51 us (6.0 and 6.9 TB/s; with cached loads
// 62 + 55, cached stores too 77 + 60, one chunk per lane and cached 71 + 59).
#include <hip/hip_runtime.h>

#include "rowops.h"
#include "rows.h"

namespace fo {
namespace {

constexpr int kThreads = 256;

constexpr int kAhead = 2;

// Chunk `at` of the matrix: its row and its place in it.
struct Chunk {
    int64_t i;
    uint32_t c;
};
__device__ __forceinline__ Chunk chunk_of(const PackArgs& a, uint32_t at, uint32_t per_row) {
    if (a.M == 1) return {0, at};
    const uint32_t i = at / per_row;
    return {(int64_t)i, at - i * per_row};
}

// `chunks` in all, `per_row` (a multiple of four) in a row's blocks.
template <int DT, int FMT>
__global__ __launch_bounds__(kThreads) void pack_kernel(const PackArgs a, uint32_t chunks, uint32_t per_row) {
    const uint32_t first = blockIdx.x * (kThreads * kAhead) + threadIdx.x;
    u32x4_t v[kAhead];
    Chunk at[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const uint32_t q = first + j * kThreads;
        if (q >= chunks) continue;
        at[j] = chunk_of(a, q, per_row);
        const int64_t n = 8 * (int64_t)at[j].c;
        v[j] = read_chunk<kStreamed>(a.x + at[j].i * a.ldx + n, a.N - n);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        if (first + j * kThreads >= chunks) continue;       // (four lanes of a block at once)
        float f[8];
        widen<DT>(v[j], f);
        pack_chunk<DT, FMT>(f, at[j].c, a.packed + at[j].i * per_row * 8, a.scales + at[j].i * (per_row / 4));
    }
}

template <int DT, int FMT>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const PackArgs a, uint32_t chunks, uint32_t per_row) {
    const uint32_t first = blockIdx.x * (kThreads * kAhead) + threadIdx.x;
    u32x2_t code[kAhead];
    uint32_t scale[kAhead];
    Chunk at[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const uint32_t q = first + j * kThreads;
        if (q >= chunks) continue;
        // (the codes' rows have no gaps)
        at[j] = chunk_of(a, q, per_row);
        code[j] = *reinterpret_cast<const u32x2_t*>(a.packed + 8 * (int64_t)q);
        scale[j] = a.scales[q >> 2];
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        if (first + j * kThreads >= chunks) continue;
        const int64_t n = 8 * (int64_t)at[j].c;
        float f[8];
        decode8<FMT>(code[j], scale_of(scale[j]), f);
        write_chunk(a.x + at[j].i * a.ldx + n, narrow<DT>(f), a.N - n);
    }
}

using Kernel = void (*)(PackArgs, uint32_t, uint32_t);
hipError_t launch_chunks(Kernel kernel, PackArgs a, hipStream_t s) {
    if (a.ldx == a.N && a.N % FO_PACK_BLOCK == 0) {
        a.N *= a.M;
        a.ldx = a.N;
        a.M = 1;
    }
    const int64_t per_row = 4 * pack_blocks(a.N), chunks = a.M * per_row;
    return launch(kernel, (uint32_t)((chunks + kThreads * kAhead - 1) / (kThreads * kAhead)), kThreads, s, a,
                  (uint32_t)chunks, (uint32_t)per_row);
}

}  // namespace

hipError_t launch_pack(int dtype, int format, const PackArgs& a, hipStream_t s) {
    const bool int8 = format == FO_PACK_INT8;
    return launch_chunks(dtype == FO_FP16
                             ? (int8 ? pack_kernel<FO_FP16, FO_PACK_INT8> : pack_kernel<FO_FP16, FO_PACK_E4M3>)
                             : (int8 ? pack_kernel<FO_BF16, FO_PACK_INT8> : pack_kernel<FO_BF16, FO_PACK_E4M3>), a, s);
}

hipError_t launch_unpack(int dtype, int format, const PackArgs& a, hipStream_t s) {
    const bool int8 = format == FO_PACK_INT8;
    return launch_chunks(dtype == FO_FP16
                             ? (int8 ? unpack_kernel<FO_FP16, FO_PACK_INT8> : unpack_kernel<FO_FP16, FO_PACK_E4M3>)
                             : (int8 ? unpack_kernel<FO_BF16, FO_PACK_INT8> : unpack_kernel<FO_BF16, FO_PACK_E4M3>), a, s);
}

}  // namespace fo
