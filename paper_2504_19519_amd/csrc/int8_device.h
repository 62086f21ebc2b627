// Device helpers of the 8-bit products: which block of the result a workgroup computes,
// its rows of a, and a finished sum.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "fo_device.h"
#include "fo_internal.h"
#include "int8ops.h"

namespace fo {

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int wait_imm(int vm, int lgkm) {
    return (vm & 15) | (7 << 4) | ((lgkm & 15) << 8) | (((vm >> 4) & 3) << 14);
}
constexpr int kRsrcWord3 = 0x00020000;          // raw byte-addressed buffer accesses
constexpr uint32_t kSpan = 0x80000000u;         // bytes that a buffer resource covers
constexpr uint32_t kOutside = kSpan;            // an offset past it: reads zeros, no memory access

template <typename F, int... Is>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, Is...>) {
    (f(std::integral_constant<int, Is>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_impl(f, std::make_integer_sequence<int, N>{});
}

__device__ __forceinline__ i32x4_t mfma16(u32x4_t x, u32x4_t y, i32x4_t c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(bit_cast<i32x4_t>(x), bit_cast<i32x4_t>(y), c, 0, 0, 0);
}

// This wave waits until at most VM of its vector memory operations are in flight and all
// of its LDS reads have returned, then meets the others.
template <int VM>
__device__ __forceinline__ void wait_and_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(wait_imm(VM, 0));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Where a workgroup's block of the result lies.
struct Block {
    int64_t row0, col0;         // of c
    int rows;                   // that it has
    int expert;
};

// Sums over lanes 0 .. l, in lane l.
__device__ __forceinline__ int lanes_before(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, true);
    return v;
}

// An expert's rows of c: the first, and how many (those below the capacity).
struct ExpertRows {
    int first, count;
};
__device__ __forceinline__ ExpertRows expert_rows(const Int8Args& a, int e) {
    const int o = a.offsets[e], n = a.counts[e], most = o < 0 || o > a.capacity ? 0 : a.capacity - o;
    return {o, n < 0 ? 0 : n > most ? most : n};
}

// The experts' row blocks of BM: lane l adds up those of experts l run .. l run + run - 1,
// run = ceil(E / 64). rows_of(e): an expert's rows.
struct Survey {
    int mine, upto;             // of the lane's experts, and of all up to them
};
template <int BM, typename F>
__device__ __forceinline__ Survey survey(const Int8Args& a, F rows_of) {
    const int lane = threadIdx.x & 63, run = (a.E + 63) / 64;
    Survey s = {0, 0};
#pragma unroll 4
    for (int i = 0; i < run; ++i) {
        const int e = lane * run + i;
        if (e < a.E) s.mine += (rows_of(e).count + BM - 1) / BM;
    }
    s.mine = s.mine < 1 << 24 ? s.mine : 1 << 24;       // (more than any launch has: the sums stay in 31 bits)
    s.upto = lanes_before(s.mine);
    return s;
}

// The block at position `p` of those of BM rows and `width` columns of the experts; false: none.
template <int BM, typename F>
__device__ __forceinline__ bool locate(const Int8Args& a, const Survey& s, F rows_of, int p, int width, Block& b) {
    const int lane = threadIdx.x & 63, run = (a.E + 63) / 64, cols = (int)((a.N + width - 1) / width);
    // each chiplet takes a contiguous share of the blocks, an expert's after another's
    constexpr int kXcds = 8;
    const int64_t all = (int64_t)__builtin_amdgcn_readlane(s.upto, 63) * cols, per = (all + kXcds - 1) / kXcds;
    const int64_t l = p / kXcds, t = (int64_t)(p % kXcds) * per + l;
    if (l >= per || t >= all) return false;
    const int at = (int)(t / cols);             // among the experts' row blocks
    const int owner = __builtin_ctzll(__builtin_amdgcn_ballot_w64(s.upto > at));
    const int before = __builtin_amdgcn_readlane(s.upto, owner) - __builtin_amdgcn_readlane(s.mine, owner);
    // the owner's experts, one to a lane
    const int e = owner * run + lane;
    ExpertRows mine = {0, 0};
    if (lane < run && e < a.E) mine = rows_of(e);
    const int past = before + lanes_before((mine.count + BM - 1) / BM);
    const int w = __builtin_ctzll(__builtin_amdgcn_ballot_w64(past > at));
    const int n = __builtin_amdgcn_readlane(mine.count, w), high = (n + BM - 1) / BM;
    const int first = __builtin_amdgcn_readlane(past, w) - high;
    // (an expert's row blocks side by side: they share its weights)
    const int inside = (int)(t - (int64_t)first * cols), r = inside % high * BM;
    b.expert = owner * run + w;
    b.row0 = (int64_t)__builtin_amdgcn_readlane(mine.first, w) + r;
    b.col0 = (int64_t)(inside / high) * width;
    b.rows = n - r < BM ? n - r : BM;
    return true;
}

// The block of workgroup `p` of those of BM rows and `width` columns; false: none.
template <int BM, bool EXPERTS>
__device__ __forceinline__ bool find_block(const Int8Args& a, int p, int width, Block& b) {
    if constexpr (EXPERTS) {
        const auto rows_of = [&](int e) { return expert_rows(a, e); };
        return locate<BM>(a, survey<BM>(a, rows_of), rows_of, p, width, b);
    } else {
        constexpr int kXcds = 8;
        const int cols = (int)((a.N + width - 1) / width), rows = (int)((a.M + BM - 1) / BM), blocks = rows * cols;
        const int t = tile_of_position(p, rows, cols, FO_ORDER_XCD, rows < 4 ? rows : 4, blocks < kXcds ? blocks : kXcds);
        b.row0 = (int64_t)(t / cols) * BM;
        b.col0 = (int64_t)(t % cols) * width;
        b.rows = (int)(a.M - b.row0 < BM ? a.M - b.row0 : BM);
        b.expert = 0;
        return true;
    }
}

// The row of a that row r of the block is of; -1: none.
template <bool EXPERTS>
__device__ __forceinline__ int64_t source_row(const Int8Args& a, const Block& b, int r) {
    if (r >= b.rows) return -1;
    if constexpr (EXPERTS) {
        int64_t s = b.row0 + r;
        if (a.pair_of) {
            const int pair = a.pair_of[s];
            s = pair < 0 ? -1 : pair / a.choices;
        }
        return s < a.a_rows ? s : -1;
    } else {
        return b.row0 + r;
    }
}

// The scales (of K = 0: zeros) and bias of columns n .. n + 3 (not by experts).
struct Columns {
    f32x4_t scale, bias;
};
template <int DT>
__device__ __forceinline__ Columns columns_of(const Int8Args& a, int64_t n) {
    Columns c;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool there = n + e < a.N;
        c.scale[e] = there && a.K > 0 ? a.b_scales[n + e] : 0.0f;
        c.bias[e] = there && a.bias ? to_f32<DT>(a.bias[n + e]) : 0.0f;
    }
    return c;
}

// Four results of a row, in 16 bits.
template <int DT>
__device__ __forceinline__ u32x2_t finish(i32x4_t sum, float row, f32x4_t scale, f32x4_t bias) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)sum[e] * row * scale[e] + bias[e];
    return u32x2_t{pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
}

// The `left` first of four results, at any 2-byte aligned address.
__device__ __forceinline__ void write_four(uint16_t* p, u32x2_t v, int64_t left) {
    if (left >= 4) {
        __builtin_memcpy(p, &v, sizeof(v));
    } else if (left > 0) {
        p[0] = (uint16_t)v[0];
        if (left > 1) p[1] = (uint16_t)(v[0] >> 16);
        if (left > 2) p[2] = (uint16_t)v[1];
    }
}

// Columns of the sums of a part of k: whole groups of four, so that every row is 16-byte aligned.
FO_HD inline int64_t partial_cols(int64_t N) { return (N + 3) / 4 * 4; }

}  // namespace fo
