// Device helpers of the row operators: rows of any length and stride in chunks of
// eight values, sums over a wave, and 8-bit checkpoint codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fo.h"
#include "fo_device.h"

namespace fo {

// Eight 16-bit values at any 2-byte aligned address: one 16-byte access (global
// memory takes unaligned ones), so rows of odd length or stride need no kernel
// of their own. The values behind a row's last whole chunk (fewer than eight)
// are taken one by a lane.
__device__ __forceinline__ u32x4_t load8(const uint16_t* p) {
    u32x4_t v;
    __builtin_memcpy(&v, p, sizeof(v));
    return v;
}
__device__ __forceinline__ void store8(uint16_t* p, u32x4_t v) { __builtin_memcpy(p, &v, sizeof(v)); }
// The same past the caches' keeping (nontemporal): large outputs that this kernel
// does not read again.
typedef uint32_t u32x4_near_t __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void stream8(uint16_t* p, u32x4_t v) {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_near_t*>(p));
}

template <int DT>
__device__ __forceinline__ void widen(u32x4_t v, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = to_f32<DT>(v[e] & 0xFFFFu);
        f[2 * e + 1] = to_f32<DT>(v[e] >> 16);
    }
}

template <int DT>
__device__ __forceinline__ u32x4_t narrow(const float* f) {
    u32x4_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack2<DT>(f[2 * e], f[2 * e + 1]);
    return v;
}

// Sum over the 64 lanes, the same in each: six adds on the vector unit with lanes
// moved within rows of 16 (row_shr 1, 2, 4, 8), then from row to row (row_bcast 15
// and 31), without the LDS that a shuffle goes through.
template <int CTRL, int ROWS>
__device__ __forceinline__ float add_moved(float v) {
    return v + bit_cast<float>(__builtin_amdgcn_update_dpp(0, bit_cast<int>(v), CTRL, ROWS, 0xF, true));
}
__device__ __forceinline__ float wave_sum(float v) {
    v = add_moved<0x111, 0xF>(v);
    v = add_moved<0x112, 0xF>(v);
    v = add_moved<0x114, 0xF>(v);
    v = add_moved<0x118, 0xF>(v);
    v = add_moved<0x142, 0xA>(v);
    v = add_moved<0x143, 0xC>(v);
    return bit_cast<float>(__builtin_amdgcn_readlane(bit_cast<int>(v), 63));
}

// ---- 8-bit checkpoints ------------------------------------------------------
// A block of 32 values shares a scale 2^s, stored as s + 127; value = code * 2^s.
// With 2^e the largest power of two <= the block's largest magnitude:
//   int8: s = e - 6, code = RNE(x / 2^s) in [-127, 127];
//   e4m3: s = e - 8, or e - 7 where the largest magnitude exceeds 1.75 * 2^e (448
//         = 1.75 * 2^8 is e4m3's largest value), code = RNE(x / 2^s).
// s >= -126, so that 2^s and 2^-s are normal fp32 numbers and the products exact: the
// only rounding is the code's. A block with an infinity or a NaN has scale byte 255
// (2^s reads as infinity) and codes 0, which read as NaN.
// Eight lanes' worth of a block: four lanes of one chunk each.

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

// Largest magnitude bits of eight values.
__device__ __forceinline__ uint32_t top_bits(u32x4_t v) {
    u16x2_t m = bit_cast<u16x2_t>(v[0] & 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, bit_cast<u16x2_t>(v[i] & 0x7FFF7FFFu));
    return m[0] > m[1] ? m[0] : m[1];
}

struct BlockScale {
    float inverse;              // 2^-s
    float limit;                // largest magnitude before rounding (e4m3)
    uint32_t byte;              // s + 127, or 255
};

// The scale of a block from the bits of its largest magnitude.
template <int DT, int FMT>
__device__ __forceinline__ BlockScale block_scale(uint32_t top) {
    const uint32_t bits = bit_cast<uint32_t>(to_f32<DT>(top));
    int s;
    BlockScale b;
    if constexpr (FMT == FO_PACK_INT8) {
        s = (int)(bits >> 23) - 127 - 6;
        b.limit = 127.0f;
    } else {
        const int e = (int)((bits + 0x1FFFFFu) >> 23) - 127;    // one more above 1.75 * 2^e
        s = e - 8;
        // a largest value that would round up past the type's range (to 256 * 2^s)
        b.limit = e > (DT == FO_FP16 ? 15 : 127) ? 240.0f : 448.0f;
    }
    s = s < -126 ? -126 : s;
    const bool finite = top < (DT == FO_FP16 ? 0x7C00u : 0x7F80u);
    b.byte = finite ? (uint32_t)(s + 127) : 255u;
    b.inverse = bit_cast<float>((uint32_t)(127 - s) << 23);
    return b;
}

// Four values' codes, little-endian.
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float* f, const BlockScale& b) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_fmed3f(f[i] * b.inverse, -b.limit, b.limit);
    uint32_t code;
    if constexpr (FMT == FO_PACK_INT8) {
        // v + 1.5 * 2^23 rounds v to a whole number (to nearest even), whose low byte
        // is the code
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = bit_cast<uint32_t>(v[i] + 12582912.0f) & 0xFFu;
        code = w[0] | (w[1] << 8) | (w[2] << 16) | (w[3] << 24);
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
        code = (uint32_t)w;
    }
    return b.byte == 255u ? 0u : code;
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return bit_cast<float>(byte << 23); }

// What four codes stand for.
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t code, float scale, float* f) {
    if constexpr (FMT == FO_PACK_INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(code >> (8 * i)) * scale;
    } else {
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)code, false);
        const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)code, true);
        f[0] = lo[0] * scale;
        f[1] = lo[1] * scale;
        f[2] = hi[0] * scale;
        f[3] = hi[1] * scale;
    }
}

template <int FMT>
__device__ __forceinline__ float decode1(uint32_t code, float scale) {
    float f[4];
    decode4<FMT>(code, scale, f);
    return f[0];
}

// Chunk c of a checkpoint's row (codes at `row`, scale bytes at `scale`).
template <int FMT>
__device__ __forceinline__ void decode8(u32x2_t code, float scale, float* f) {
    decode4<FMT>(code[0], scale, f);
    decode4<FMT>(code[1], scale, f + 4);
}

// A lane's chunk of a whole block, packed with the three neighbours' that share it
// (lanes 4 i .. 4 i + 3 hold chunks 4 j .. 4 j + 3; every lane of the four calls).
template <int DT, int FMT>
__device__ __forceinline__ void pack_chunk(u32x4_t v, int c, uint8_t* packed_row, uint8_t* scale_row) {
    uint32_t top = top_bits(v);
    // the other three lanes': quad_perm [1, 0, 3, 2], then [2, 3, 0, 1]
    uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true);
    top = top > other ? top : other;
    other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true);
    top = top > other ? top : other;
    const BlockScale b = block_scale<DT, FMT>(top);
    float f[8];
    widen<DT>(v, f);
    u32x2_t code;
    code[0] = encode4<FMT>(f, b);
    code[1] = encode4<FMT>(f + 4, b);
    *reinterpret_cast<u32x2_t*>(packed_row + 8 * (int64_t)c) = code;
    if ((c & 3) == 0) scale_row[c >> 2] = (uint8_t)b.byte;
}

// The row's last block where N is no multiple of 32: one value per lane of the
// first 32, codes behind the row's end 0.
template <int DT, int FMT>
__device__ __forceinline__ void pack_last(const uint16_t* row, int64_t N, int lane, uint8_t* packed_row,
                                          uint8_t* scale_row) {
    const int64_t block = N / FO_PACK_BLOCK, n = block * FO_PACK_BLOCK + lane;
    const uint32_t bits = lane < FO_PACK_BLOCK && n < N ? row[n] : 0u;
    uint32_t top = bits & 0x7FFFu;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const uint32_t other = __shfl_xor(top, off, 64);
        top = top > other ? top : other;
    }
    if (lane < FO_PACK_BLOCK) {
        const BlockScale b = block_scale<DT, FMT>(top);
        const float f[4] = {to_f32<DT>(bits), 0.0f, 0.0f, 0.0f};
        packed_row[n] = (uint8_t)encode4<FMT>(f, b);
        if (lane == 0) scale_row[block] = (uint8_t)b.byte;
    }
}

}  // namespace fo
