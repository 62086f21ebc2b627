// Device helpers of the row operators: rows of any length and stride in chunks of
// eight values, sums over a wave, and 8-bit checkpoint codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fo.h"
#include "fo_device.h"

namespace fo {

// Eight 16-bit values at any 2-byte aligned address: one 16-byte access (global
// memory takes unaligned ones), so that rows of odd length or stride need no kernel
// of their own.
__device__ __forceinline__ u32x4_t load8(const uint16_t* p) {
    u32x4_t v;
    __builtin_memcpy(&v, p, sizeof(v));
    return v;
}
// The same past the caches' keeping (nontemporal), for inputs that are read once and
// outputs that the kernel does not read again.
typedef uint32_t u32x4_near_t __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ u32x4_t stream_load8(const uint16_t* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_near_t*>(p));
}

__device__ __forceinline__ void stream8(uint16_t* p, u32x4_t v) {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_near_t*>(p));
}

// A row's chunk of which `left` values lie within the row: all eight; the row's last
// few, as four, two and one of them (the rest reads as zeros); or none.
enum Through { kCached, kStreamed };
template <Through T>
__device__ __forceinline__ u32x4_t read_chunk(const uint16_t* p, int64_t left) {
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (left >= 8) {
        v = T == kStreamed ? stream_load8(p) : load8(p);
    } else if (left > 0) {
        const int n = (int)left;
        u32x2_t four = {0u, 0u};
        uint32_t two = 0u, one = 0u;
        if (n & 4) __builtin_memcpy(&four, p, sizeof(four));
        if (n & 2) __builtin_memcpy(&two, p + (n & 4), sizeof(two));
        if (n & 1) one = p[n & 6];
        const uint32_t next = n & 2 ? two : one, last = n & 2 ? one : 0u;      // behind the four
        v[0] = n & 4 ? four[0] : next;
        v[1] = n & 4 ? four[1] : last;
        v[2] = n & 4 ? next : 0u;
        v[3] = n & 4 ? last : 0u;
    }
    return v;
}
// Written the same way, past the caches' keeping.
__device__ __forceinline__ void write_chunk(uint16_t* p, u32x4_t v, int64_t left) {
    if (left >= 8) {
        stream8(p, v);
    } else if (left > 0) {
        const int n = (int)left;
        const u32x2_t four = {v[0], v[1]};
        const uint32_t next = n & 4 ? v[2] : v[0], last = n & 4 ? v[3] : v[1];
        const uint16_t one = (uint16_t)(n & 2 ? last : next);
        if (n & 4) __builtin_memcpy(p, &four, sizeof(four));
        if (n & 2) __builtin_memcpy(p + (n & 4), &next, sizeof(next));
        if (n & 1) p[n & 6] = one;
    }
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

// Sum over TH neighbouring lanes (8, 16, 32 or all 64), the same in each of them. Lanes
// change places within four (quad_perm [1, 0, 3, 2], [2, 3, 0, 1]), eight and sixteen
// (row_half_mirror, row_mirror), and rows of sixteen by the swap of neighbouring ones.
template <int TH>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (TH == 64) {
        return wave_sum(v);
    } else {
        v = add_moved<0xB1, 0xF>(v);
        v = add_moved<0x4E, 0xF>(v);
        v = add_moved<0x141, 0xF>(v);
        if constexpr (TH > 8) v = add_moved<0x140, 0xF>(v);
        if constexpr (TH > 16) {
            const u32x2_t swapped = bit_cast<u32x2_t>(
                __builtin_amdgcn_permlane16_swap(bit_cast<uint32_t>(v), bit_cast<uint32_t>(v), false, false));
            v = bit_cast<float>(swapped[0]) + bit_cast<float>(swapped[1]);
        }
        return v;
    }
}

// Two sums over the 64 lanes for little more than one: the halves change places, so
// that the lower lanes go on with a's sum and the upper ones with b's.
__device__ __forceinline__ void wave_sums(float& a, float& b) {
    const u32x2_t swapped = bit_cast<u32x2_t>(
        __builtin_amdgcn_permlane32_swap(bit_cast<uint32_t>(a), bit_cast<uint32_t>(b), false, false));
    float v = bit_cast<float>(swapped[0]) + bit_cast<float>(swapped[1]);
    v = add_moved<0x111, 0xF>(v);
    v = add_moved<0x112, 0xF>(v);
    v = add_moved<0x114, 0xF>(v);
    v = add_moved<0x118, 0xF>(v);
    v = add_moved<0x142, 0xA>(v);
    a = bit_cast<float>(__builtin_amdgcn_readlane(bit_cast<int>(v), 31));
    b = bit_cast<float>(__builtin_amdgcn_readlane(bit_cast<int>(v), 63));
}
// Sum over the first W lanes (up to 16; the others up to 16 hold zeros), the same in each lane.
template <int W>
__device__ __forceinline__ float first_sum(float v) {
    if constexpr (W > 1) v = add_moved<0x111, 0xF>(v);
    if constexpr (W > 2) v = add_moved<0x112, 0xF>(v);
    if constexpr (W > 4) v = add_moved<0x114, 0xF>(v);
    if constexpr (W > 8) v = add_moved<0x118, 0xF>(v);
    return bit_cast<float>(__builtin_amdgcn_readlane(bit_cast<int>(v), W - 1));
}

// 1 / sqrt(v), within 1.5 steps of fp32: the hardware's, which takes values below the
// normal range as zero, for a scaled value where v may be one.
__device__ __forceinline__ float rsqrt_of(float v) {
    const bool small = v < 0x1p-96f;
    const float r = __builtin_amdgcn_rsqf(small ? v * 0x1p64f : v);
    return small ? r * 0x1p32f : r;
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

typedef int16_t i16x2_t __attribute__((ext_vector_type(2)));

// Largest magnitude of eight values, NaN if one is.
__device__ __forceinline__ float top_of(const float* f) {
    float m = __builtin_elementwise_maximum(__builtin_fabsf(f[0]), __builtin_fabsf(f[1]));
#pragma unroll
    for (int e = 2; e < 8; ++e) m = __builtin_elementwise_maximum(m, __builtin_fabsf(f[e]));
    return m;
}

struct BlockScale {
    float inverse;              // 2^-s
    float limit;                // largest magnitude before rounding (e4m3)
    uint32_t byte;              // s + 127, or 255
};

// The scale of a block from its largest magnitude.
template <int DT, int FMT>
__device__ __forceinline__ BlockScale block_scale(float top) {
    const uint32_t bits = bit_cast<uint32_t>(top) & 0x7FFFFFFFu;
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
    b.byte = bits < 0x7F800000u ? (uint32_t)(s + 127) : 255u;
    b.inverse = bit_cast<float>((uint32_t)(127 - s) << 23);
    return b;
}

// Four values' codes, little-endian.
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float* f, const BlockScale& b) {
    uint32_t code;
    if constexpr (FMT == FO_PACK_INT8) {
        // x / 2^s + 1.5 * 2^23 rounds x / 2^s to a whole number (to nearest even), which
        // its low 16 bits hold; two of them at a time are kept within [-127, 127]
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t lo = bit_cast<uint32_t>(__builtin_fmaf(f[2 * i], b.inverse, 12582912.0f));
            const uint32_t hi = bit_cast<uint32_t>(__builtin_fmaf(f[2 * i + 1], b.inverse, 12582912.0f));
            i16x2_t v = bit_cast<i16x2_t>(__builtin_amdgcn_perm(hi, lo, 0x05040100u));
            v = __builtin_elementwise_min(v, i16x2_t{127, 127});
            v = __builtin_elementwise_max(v, i16x2_t{-127, -127});
            w[i] = bit_cast<uint32_t>(v);
        }
        code = __builtin_amdgcn_perm(w[1], w[0], 0x06040200u);
    } else {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_fmed3f(f[i] * b.inverse, -b.limit, b.limit);
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

// What a chunk's eight codes stand for.
template <int FMT>
__device__ __forceinline__ void decode8(u32x2_t code, float scale, float* f) {
    decode4<FMT>(code[0], scale, f);
    decode4<FMT>(code[1], scale, f + 4);
}

// A lane's chunk f, packed with the three neighbours' that share its block (lanes
// 4 i .. 4 i + 3 hold chunks 4 j .. 4 j + 3; all four lanes call). Values behind the
// row's end are zeros.
template <int DT, int FMT>
__device__ __forceinline__ void pack_chunk(const float* f, uint32_t c, uint8_t* packed_row, uint8_t* scale_row) {
    float top = top_of(f);
    // the other three lanes': quad_perm [1, 0, 3, 2], then [2, 3, 0, 1]
    top = __builtin_elementwise_maximum(
        top, bit_cast<float>(__builtin_amdgcn_update_dpp(0, bit_cast<int>(top), 0xB1, 0xF, 0xF, true)));
    top = __builtin_elementwise_maximum(
        top, bit_cast<float>(__builtin_amdgcn_update_dpp(0, bit_cast<int>(top), 0x4E, 0xF, 0xF, true)));
    const BlockScale b = block_scale<DT, FMT>(top);
    u32x2_t code;
    code[0] = encode4<FMT>(f, b);
    code[1] = encode4<FMT>(f + 4, b);
    *reinterpret_cast<u32x2_t*>(packed_row + 8 * (int64_t)c) = code;
    if ((c & 3) == 0) scale_row[c >> 2] = (uint8_t)b.byte;
}

}  // namespace fo
