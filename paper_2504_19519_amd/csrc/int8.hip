// Products of 8-bit matrices, alone and by experts (gfx950).
//
//   c[m, n] = (sum over k of a[m, k] b[n, k]) sa[m] sb[n] + bias[n],
//
// a [M, K] and b [N, K] in 8-bit integers, both k-contiguous. The sums are exact (32-bit
// integers, v_mfma_i32_16x16x64_i8), so no order of them changes a result; a sum is
// rounded to fp32, and the result to 16 bits. By experts: b, its scales and bias are the
// row's expert's, and the rows of a are taken through the pairs that fo_route_sort has
// put in order.
//
// Codes behind a row's end, up to a multiple of 16, are zeros; chunks of 16 past that
// are not read.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>
#include <utility>

#include "int8ops.h"
#include "rows.h"
#include "rowops.h"

namespace fo {
namespace {

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

// The block of workgroup `p` of those of BM rows and BN columns; false: none. Experts:
// every wave adds up the experts' blocks (E <= 1024: up to 16 loads, all in flight).
template <int BM, int BN, bool EXPERTS>
__device__ __forceinline__ bool find_block(const Int8Args& a, int p, Block& b) {
    const int cols = (int)((a.N + BN - 1) / BN);
    constexpr int kXcds = 8;
    if constexpr (!EXPERTS) {
        const int rows = (int)((a.M + BM - 1) / BM), blocks = rows * cols;
        const int t = tile_of_position(p, rows, cols, FO_ORDER_XCD, rows < 4 ? rows : 4, blocks < kXcds ? blocks : kXcds);
        b.row0 = (int64_t)(t / cols) * BM;
        b.col0 = (int64_t)(t % cols) * BN;
        b.rows = (int)(a.M - b.row0 < BM ? a.M - b.row0 : BM);
        b.expert = 0;
        return true;
    } else {
        const int lane = threadIdx.x & 63;
        constexpr int kRounds = FO_ROUTE_MAX_EXPERTS / 64;
        int blocks[kRounds];
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            blocks[i] = 0;
            if (64 * i < a.E) {
                const int e = 64 * i + lane;
                int n = e < a.E ? a.counts[e] : 0;
                const int o = e < a.E ? a.offsets[e] : 0;
                const int most = o < 0 || o > a.capacity ? 0 : a.capacity - o;      // rows below the capacity
                n = n < 0 ? 0 : n > most ? most : n;
                blocks[i] = (n + BM - 1) / BM;
            }
        }
        int upto[kRounds];
        int64_t total = 0;
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            upto[i] = 0;
            if (64 * i < a.E) {
                upto[i] = lanes_before(blocks[i]);
                total += __builtin_amdgcn_readlane(upto[i], 63);
            }
        }
        // each chiplet takes a contiguous share of the blocks, an expert's after another's
        total *= cols;
        const int64_t per = (total + kXcds - 1) / kXcds, l = p / kXcds, t = (int64_t)(p % kXcds) * per + l;
        if (l >= per || t >= total) return false;
        const int64_t at = t / cols;                // among the experts' row blocks
        int64_t before = 0;
        int expert = -1, first = 0, count = 0;
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            if (64 * i < a.E && expert < 0) {
                const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto[i] > at);
                if (past) {
                    const int w = __builtin_ctzll(past);
                    expert = 64 * i + w;
                    count = __builtin_amdgcn_readlane(blocks[i], w);
                    first = (int)(before + __builtin_amdgcn_readlane(upto[i], w)) - count;
                }
                before += __builtin_amdgcn_readlane(upto[i], 63);
            }
        }
        // (an expert's row blocks side by side: they share its weights)
        const int inside = (int)(t - (int64_t)first * cols);
        const int offset = a.offsets[expert], n = a.counts[expert], r = inside % count * BM;
        const int left = (n < a.capacity - offset ? n : a.capacity - offset) - r;
        b.expert = expert;
        b.row0 = (int64_t)offset + r;
        b.col0 = (int64_t)(inside / count) * BN;
        b.rows = left < BM ? left : BM;
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

// A row's four results of the columns n .. n + 3.
struct Columns {
    float scale[4], bias[4];
};
template <int DT>
__device__ __forceinline__ Columns columns_of(const Int8Args& a, int64_t expert, int64_t n) {
    Columns c;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool there = n + e < a.N;
        const int64_t at = expert * a.N + n + e;
        c.scale[e] = there ? a.b_scales[at] : 0.0f;
        c.bias[e] = there && a.bias ? to_f32<DT>(a.bias[at]) : 0.0f;
    }
    return c;
}
template <int DT>
__device__ __forceinline__ u32x2_t finish(i32x4_t sum, float scale, const Columns& c) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)sum[e] * scale * c.scale[e] + c.bias[e];
    return u32x2_t{pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
}

// ---- blocks ---------------------------------------------------------------
// Four waves, 2 x 2, on a block of BM x BN. k steps of 128, moving from memory straight
// into an LDS ring of ST stages; the next substep's fragments are read while the MFMAs
// of the current one run, one barrier per step. An operand row of a step is 128 bytes,
// chunk c of row r at slot c ^ ((r / 2) % 8): 16 rows' chunks lie on different banks.
template <int DT, int BM, int BN, int ST, bool EXPERTS>
__global__ __launch_bounds__(256) void int8_block_kernel(const Int8Args a) {
    constexpr int kWaves = 4, WTM = BM / 2, WTN = BN / 2, MI = WTM / 16, NJ = WTN / 16;
    constexpr int kA = BM * 128, kStage = (BM + BN) * 128;
    constexpr int kAI = kA / 1024 / kWaves, kBI = BN * 128 / 1024 / kWaves, kLoads = kAI + kBI;
    static_assert(BM >= 32 && BN >= 32 && ST >= 2 && ST <= 4 && ST * kLoads <= 62, "blocks and stages");

    // the stages live in separate arrays, so that the compiler can tell the stage being
    // read from the stages being filled
    __shared__ __attribute__((aligned(1024))) char st0[kStage], st1[kStage];
    __shared__ __attribute__((aligned(ST > 2 ? 1024 : 16))) char st2[ST > 2 ? kStage : 16];
    __shared__ __attribute__((aligned(ST > 3 ? 1024 : 16))) char st3[ST > 3 ? kStage : 16];
    auto stage = [&](auto uc) __attribute__((always_inline)) -> char* {
        constexpr int u = decltype(uc)::value % ST;
        if constexpr (u == 0) return st0;
        else if constexpr (u == 1) return st1;
        else if constexpr (u == 2) return st2;
        else return st3;
    };
    constexpr int kOutRow = WTN * 2 + 16;
    __shared__ __attribute__((aligned(16))) char s_out[kWaves][16 * kOutRow];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    Block b;
    if (!find_block<BM, BN, EXPERTS>(a, blockIdx.x, b)) return;
    const int bytes = (int)int8_row_bytes(a.K), steps = (bytes + 127) / 128;

    const bool gather = EXPERTS && a.pair_of;
    const int8_t* const ablk = gather ? a.a : a.a + b.row0 * a.lda;
    const int8_t* const bblk = a.b + ((int64_t)b.expert * a.N + b.col0) * a.ldb;
    const int cols = (int)(a.N - b.col0 < BN ? a.N - b.col0 : BN);

    // A load instruction fills 1 KB: 8 operand rows of 128 bytes. A lane's offset from the
    // operand's base, or kOutside for a row that is not there; and its place in the row.
    uint32_t voff[kLoads], place[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const bool is_a = i < kAI;
        const int r = (is_a ? wave * kAI + i : wave * kBI + i - kAI) * 8 + lane / 8;
        place[i] = 16u * (uint32_t)((lane & 7) ^ ((r >> 1) & 7));
        if (is_a) {
            const int64_t s = source_row<EXPERTS>(a, b, r);
            voff[i] = s < 0 ? kOutside : (uint32_t)((gather ? s : r) * a.lda) + place[i];
        } else {
            voff[i] = r < cols ? (uint32_t)(r * a.ldb) + place[i] : kOutside;
        }
    }
    // Fragments: lane l feeds row l % 16 of a 16-row block with chunk 4 h + l / 16 of MFMA
    // substep h. The weights are the first operand: lane l then holds row l % 16 of c,
    // columns 4 (l / 16) .. + 3.
    const int a_row = (wm * WTM + (lane & 15)) * 128, b_row = kA + (wn * WTN + (lane & 15)) * 128;
    int cslot[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) cslot[h] = 16 * ((4 * h + (lane >> 4)) ^ ((lane >> 1) & 7));
    u32x4_t fa[2][MI], fb[2][NJ];
    i32x4_t acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};

    auto load_at = [&](auto ic, int t, char* st) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        constexpr bool is_a = i < kAI;
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc((void*)(is_a ? ablk : bblk), 0, (int)kSpan, kRsrcWord3);
        // (the step's offset is added here: an offset past the resource stays past it)
        const uint32_t at = 128u * (uint32_t)t;
        const uint32_t v = place[i] + at < (uint32_t)bytes && voff[i] != kOutside ? voff[i] + at : kOutside;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            r, (lds_void_t*)(st + (is_a ? 0 : kA) + (is_a ? wave * kAI + i : wave * kBI + i - kAI) * 1024), 16, v, 0, 0, 0);
    };
    auto read_one = [&](auto ic, auto hc, const char* st, u32x4_t (&xa)[MI], u32x4_t (&xb)[NJ])
                        __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value, h = decltype(hc)::value;
        if constexpr (i == 0) xa[0] = *reinterpret_cast<const u32x4_t*>(st + a_row + cslot[h]);
        else if constexpr (i <= NJ) xb[i - 1] = *reinterpret_cast<const u32x4_t*>(st + b_row + (i - 1) * 2048 + cslot[h]);
        else xa[i - NJ] = *reinterpret_cast<const u32x4_t*>(st + a_row + (i - NJ) * 2048 + cslot[h]);
    };
    // One substep: its MFMAs carry the reads of the next one and, with loads_c, step t's
    // loads into stage lst.
    auto substep = [&](u32x4_t (&xa)[MI], u32x4_t (&xb)[NJ], auto h_next, const char* rst, u32x4_t (&ya)[MI],
                       u32x4_t (&yb)[NJ], auto loads_c, int t, char* lst) __attribute__((always_inline)) {
        constexpr int kM = MI * NJ, kR = MI + NJ;
        constexpr int rper = (kR + kM - 1) / kM, lper = (kLoads + kM - 1) / kM;
        constexpr int gap = kM / kLoads > 1 ? kM / kLoads : 1;
        static_for<kM>([&](auto mc) __attribute__((always_inline)) {
            constexpr int m = decltype(mc)::value;
            static_for<rper>([&](auto xc) __attribute__((always_inline)) {
                constexpr int r = m * rper + decltype(xc)::value;
                if constexpr (r < kR) read_one(std::integral_constant<int, r>{}, h_next, rst, ya, yb);
            });
            static_for<lper>([&](auto xc) __attribute__((always_inline)) {
                constexpr int l = m / gap * lper + decltype(xc)::value;
                if constexpr (decltype(loads_c)::value && m % gap == 0 && l < kLoads)
                    load_at(std::integral_constant<int, l>{}, t, lst);
            });
            acc[m / NJ][m % NJ] = mfma16(xb[m % NJ], xa[m / NJ], acc[m / NJ][m % NJ]);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // Step t (in stage u): its first substep while the second one's fragments are read;
    // then, once step t + 1 has landed and every wave has read this stage, the second one
    // while the next step's first fragments are read and step t + ST is loaded here.
    auto step = [&](auto uc, int t) __attribute__((always_inline)) {
        constexpr int u = decltype(uc)::value;
        char* const cur = stage(uc);
        char* const nxt = stage(std::integral_constant<int, u + 1>{});
        substep(fa[0], fb[0], std::integral_constant<int, 1>{}, cur, fa[1], fb[1], std::false_type{}, 0, cur);
        wait_and_barrier<(ST - 2) * kLoads>();
        substep(fa[1], fb[1], std::integral_constant<int, 0>{}, nxt, fa[0], fb[0], std::true_type{}, t + ST, cur);
    };
    auto rest = [&](auto&& self, auto uc, int t) __attribute__((always_inline)) -> void {
        constexpr int u = decltype(uc)::value;
        if constexpr (u + 1 < ST) {
            if (t + u < steps) {
                step(uc, t + u);
                self(self, std::integral_constant<int, u + 1>{}, t);
            }
        }
    };

    static_for<ST>([&](auto uc) __attribute__((always_inline)) {
        static_for<kLoads>([&](auto ic) __attribute__((always_inline)) { load_at(ic, decltype(uc)::value, stage(uc)); });
    });
    wait_and_barrier<(ST - 1) * kLoads>();
    static_for<MI + NJ>([&](auto ic) __attribute__((always_inline)) {
        read_one(ic, std::integral_constant<int, 0>{}, st0, fa[0], fb[0]);
    });
    int t = 0;
    for (; t + ST <= steps; t += ST)
        static_for<ST>([&](auto uc) __attribute__((always_inline)) { step(uc, t + decltype(uc)::value); });
    rest(rest, std::integral_constant<int, 0>{}, t);
    // (no load may still be writing LDS when the workgroup ends)
    wait_and_barrier<0>();

    // A wave's part of the block, 16 rows at a time: through LDS into whole rows.
    const int64_t col = b.col0 + wn * WTN;
    Columns of[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) of[j] = columns_of<DT>(a, b.expert, col + 16 * j + 4 * (lane >> 4));
    char* const out = s_out[wave];
    static_for<MI>([&](auto ic) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        const int r0 = wm * WTM + 16 * i;
        const int64_t s = source_row<EXPERTS>(a, b, r0 + (lane & 15));
        const float scale = s < 0 ? 0.0f : a.a_scales[s];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            *reinterpret_cast<u32x2_t*>(out + (lane & 15) * kOutRow + 32 * j + 8 * (lane >> 4)) =
                finish<DT>(acc[i][j], scale, of[j]);
        constexpr int kChunks = WTN / 8;            // of a row
#pragma unroll
        for (int q = 0; q < 16 * kChunks / 64 + (16 * kChunks % 64 != 0); ++q) {
            const int at = 64 * q + lane, r = at / kChunks, ch = at % kChunks;
            if (r >= 16) continue;
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(out + r * kOutRow + 16 * ch);
            if (source_row<EXPERTS>(a, b, r0 + r) < 0) continue;
            write_chunk(a.c + (b.row0 + r0 + r) * a.ldc + col + 8 * ch, v, a.N - col - 8 * ch);
        }
    });
}

// ---- few rows ---------------------------------------------------------------
// Up to 16 MB rows: the weights are read once, from memory straight into the MFMA's
// registers. The W waves of a workgroup share its 16 NB columns and divide k.
template <int DT, int MB, int NB, int W, int U, bool EXPERTS>
__global__ __launch_bounds__(64 * W) void int8_few_kernel(const Int8Args a) {
    __shared__ i32x4_t s_sum[W][MB * NB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Block b;
    if (!find_block<16 * MB, 16 * NB, EXPERTS>(a, blockIdx.x, b)) return;
    const int bytes = (int)int8_row_bytes(a.K), whole = bytes / 64;

    // lane l reads chunk l / 16 of a step of 64; rows that are not there stand for one that is
    const int8_t* pa[MB];
    const int8_t* pb[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int64_t s = source_row<EXPERTS>(a, b, 16 * i + (lane & 15));
        pa[i] = a.a + (s < 0 ? 0 : s) * a.lda + 16 * (lane >> 4);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int64_t n = b.col0 + 16 * j + (lane & 15);
        pb[j] = a.b + ((int64_t)b.expert * a.N + (n < a.N ? n : a.N - 1)) * a.ldb + 16 * (lane >> 4);
    }
    i32x4_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
    auto at = [](const int8_t* p) { return *reinterpret_cast<const u32x4_t*>(p); };

    // a wave's steps, pairs of them together: whole 128-byte lines
    const int per = ((whole + 1) / 2 + W - 1) / W * 2;
    int s = wave * per;
    const int end = s + per < whole ? s + per : whole;
    for (; s + U <= end; s += U) {
        u32x4_t fa[U][MB], fb[U][NB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int j = 0; j < NB; ++j) fb[u][j] = at(pb[j] + 64 * (s + u));
#pragma unroll
            for (int i = 0; i < MB; ++i) fa[u][i] = at(pa[i] + 64 * (s + u));
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mfma16(fb[u][j], fa[u][i], acc[i][j]);
    }
    for (; s < end; ++s) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = mfma16(at(pb[j] + 64 * s), at(pa[i] + 64 * s), acc[i][j]);
    }
    if (wave == W - 1 && 64 * whole < bytes) {       // the chunks behind the last whole step
        const bool there = 64 * whole + 16 * (lane >> 4) < bytes;
        const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                acc[i][j] = mfma16(there ? at(pb[j] + 64 * whole) : zero, there ? at(pa[i] + 64 * whole) : zero, acc[i][j]);
    }

    if constexpr (W > 1) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) s_sum[wave][i * NB + j][lane] = acc[i][j];
        __syncthreads();
    }
    for (int f = wave; f < MB * NB; f += W) {
        i32x4_t sum = {0, 0, 0, 0};
        if constexpr (W > 1) {
#pragma unroll
            for (int w = 0; w < W; ++w) sum += s_sum[w][f][lane];
        } else {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (f == i * NB + j) sum = acc[i][j];
        }
        const int r = 16 * (f / NB) + (lane & 15);
        const int64_t src = source_row<EXPERTS>(a, b, r), n = b.col0 + 16 * (f % NB) + 4 * (lane >> 4);
        if (src < 0 || n >= a.N) continue;
        const u32x2_t v = finish<DT>(sum, a.a_scales[src], columns_of<DT>(a, b.expert, n));
        uint16_t* const out = a.c + (b.row0 + r) * a.ldc + n;
        if (n + 4 <= a.N) {
            __builtin_memcpy(out, &v, sizeof(v));
        } else {
            out[0] = (uint16_t)v[0];
            if (n + 1 < a.N) out[1] = (uint16_t)(v[0] >> 16);
            if (n + 2 < a.N) out[2] = (uint16_t)v[1];
        }
    }
}

// Workgroups of blocks of BM x BN: of M rows, or of `capacity` rows of E experts.
template <bool EXPERTS>
int64_t blocks_of(const Int8Args& a, int64_t BM, int64_t BN) {
    const int64_t cols = (a.N + BN - 1) / BN;
    if constexpr (EXPERTS) {
        // each expert's last block may be nearly empty; whole rounds over the chiplets
        return (cols * (a.capacity / BM + std::min<int64_t>(a.E, a.capacity)) + 7) / 8 * 8;
    } else {
        return cols * ((a.M + BM - 1) / BM);
    }
}

template <int N>
using Int = std::integral_constant<int, N>;

// The form of a launch whose blocks have `rows` rows (of an expert: on average), as
// few(MB, NB, W, U) or block(BM, BN, ST).
template <bool EXPERTS, typename Few, typename Wide>
auto for_form(const Int8Args& a, Few few, Wide block) {
    const int64_t rows = EXPERTS ? (a.capacity + a.E - 1) / a.E : a.M;
    if (rows <= 16) return few(Int<1>(), Int<1>(), Int<4>(), Int<8>());
    if (rows <= 32) return few(Int<2>(), Int<1>(), Int<4>(), Int<4>());
    if (rows <= 64) return few(Int<4>(), Int<1>(), Int<4>(), Int<4>());
    if (blocks_of<EXPERTS>(a, 128, 128) < 256) return block(Int<64>(), Int<64>(), Int<4>());
    return block(Int<128>(), Int<128>(), Int<2>());
}

template <bool EXPERTS>
hipError_t launch_any(int dtype, const Int8Args& a, hipStream_t s) {
    return for_form<EXPERTS>(
        a,
        [&](auto mb, auto nb, auto w, auto u) {
            constexpr int MB = decltype(mb)::value, NB = decltype(nb)::value, W = decltype(w)::value, U = decltype(u)::value;
            return launch(dtype == FO_FP16 ? int8_few_kernel<FO_FP16, MB, NB, W, U, EXPERTS>
                                           : int8_few_kernel<FO_BF16, MB, NB, W, U, EXPERTS>,
                          (uint32_t)blocks_of<EXPERTS>(a, 16 * MB, 16 * NB), 64 * W, s, a);
        },
        [&](auto bm, auto bn, auto st) {
            constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value, ST = decltype(st)::value;
            return launch(dtype == FO_FP16 ? int8_block_kernel<FO_FP16, BM, BN, ST, EXPERTS>
                                           : int8_block_kernel<FO_BF16, BM, BN, ST, EXPERTS>,
                          (uint32_t)blocks_of<EXPERTS>(a, BM, BN), 256, s, a);
        });
}

template <bool EXPERTS>
bool fits(const Int8Args& a) {
    const int64_t blocks = for_form<EXPERTS>(
        a, [&](auto mb, auto nb, auto, auto) { return blocks_of<EXPERTS>(a, 16 * decltype(mb)::value, 16 * decltype(nb)::value); },
        [&](auto bm, auto bn, auto) { return blocks_of<EXPERTS>(a, decltype(bm)::value, decltype(bn)::value); });
    return blocks <= (int64_t)UINT32_MAX / 256;
}

}  // namespace

int64_t int8_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

bool int8_launchable(const Int8Args& a, bool experts) { return experts ? fits<true>(a) : fits<false>(a); }

hipError_t launch_int8_product(int dtype, const Int8Args& a, hipStream_t s) { return launch_any<false>(dtype, a, s); }
hipError_t launch_int8_experts(int dtype, const Int8Args& a, hipStream_t s) { return launch_any<true>(dtype, a, s); }

}  // namespace fo
