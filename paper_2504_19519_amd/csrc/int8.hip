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

#include "int8_device.h"
#include "int8ops.h"
#include "rows.h"
#include "rowops.h"

namespace fo {
namespace {

// ---- blocks ---------------------------------------------------------------
// Four waves, 2 x 2, on a block of BM x BN. k steps of 128, moving from memory straight
// into an LDS ring of ST stages; the next substep's fragments are read while the MFMAs
// of the current one run, one barrier per step. An operand row of a step is 128 bytes,
// chunk c of row r at slot c ^ ((r / 2) % 8): 16 rows' chunks lie on different banks. ONCE:
// the weights' loads are past the caches' keeping.
// Bound by the weights' bytes where rows are few (16 tokens to 8 of 256 experts, 2048 x 7168:
// 157 us, 6.3 TB/s), else by waits for LDS and by MFMAs (1024 x 4096 x 4096 22 us, 1.55 POPS).
constexpr int kNontemporal = 2;         // cache policy of a buffer load
template <int DT, int BM, int BN, int ST, bool EXPERTS, bool ONCE>
__global__ __launch_bounds__(256, BM == 32 ? 4 : ST == 3 && BN == 128 ? 1 : 2) void int8_block_kernel(const Int8Args a) {
    constexpr int kWaves = 4, WTM = BM / 2, WTN = BN / 2, MI = WTM / 16, NJ = WTN / 16;
    constexpr int kA = BM * 128, kStage = (BM + BN) * 128;
    constexpr int kAI = kA / 1024 / kWaves, kBI = BN * 128 / 1024 / kWaves, kLoads = kAI + kBI;
    static_assert(BM >= 32 && BN >= 32 && ST >= 2 && ST <= 4 && ST * kLoads <= 64, "blocks and stages");

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
    if (!find_block<BM, EXPERTS>(a, blockIdx.x, BN * a.span, b)) return;
    const int bytes = (int)int8_row_bytes(a.K);
    // the steps of this part of k
    const int every = (bytes + 127) / 128, part = EXPERTS ? 0 : (int)blockIdx.y, parts = EXPERTS ? 1 : a.parts;
    const int first = every * part / parts, steps = every * (part + 1) / parts - first;

    const bool gather = EXPERTS && a.pair_of;
    const int8_t* const ablk = gather ? a.a : a.a + b.row0 * a.lda;

    // What the epilogue wants to know of the rows and columns, a row and a column to a thread:
    // looked up ahead of the operands' loads, in LDS by the first steps. (Of K = 0 the scales
    // count as 0: they may be anything, and the sums are 0.)
    __shared__ int s_from[EXPERTS ? BM : 1];             // row of a, or -1
    __shared__ __attribute__((aligned(16))) float s_row[BM], s_scale[BN], s_bias[BN];
    const int tid = threadIdx.x;
    float row_scale = 0.0f, col_scale = 0.0f, col_bias = 0.0f;
    if (tid < BM) {
        const int64_t from = source_row<EXPERTS>(a, b, tid);
        if constexpr (EXPERTS) s_from[tid] = (int)from;
        if (from >= 0 && a.K > 0) row_scale = a.a_scales[from];
    }
    auto look_up = [&]() {
        const int64_t n = b.col0 + tid, at = (int64_t)b.expert * a.N + n;
        if (tid < BN && n < a.N) {
            if (a.K > 0) col_scale = a.b_scales[at];
            if (a.bias) col_bias = to_f32<DT>(a.bias[at]);
        }
    };
    look_up();
    if constexpr (EXPERTS) wait_and_barrier<63>();

    // A load instruction fills 1 KB: 8 operand rows of 128 bytes. A lane's offset from the
    // operand's base, or kOutside for a row that is not there; and its place in the row.
    uint32_t voff[kLoads], place[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = (i < kAI ? wave * kAI + i : wave * kBI + i - kAI) * 8 + lane / 8;
        place[i] = 16u * (uint32_t)((lane & 7) ^ ((r >> 1) & 7));
        if (i < kAI) {
            const int from = EXPERTS ? s_from[EXPERTS ? r : 0] : r < b.rows ? r : -1;
            voff[i] = from < 0 ? kOutside : (uint32_t)((gather ? from : r) * a.lda) + place[i];
        }
    }
    // Fragments: lane l feeds row l % 16 of a 16-row block with chunk 4 h + l / 16 of MFMA
    // substep h. The weights are the first operand: lane l then holds row l % 16 of c,
    // columns 4 (l / 16) .. + 3.
    const int a_row = (wm * WTM + (lane & 15)) * 128, b_row = kA + (wn * WTN + (lane & 15)) * 128;
    int cslot[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) cslot[h] = 16 * ((4 * h + (lane >> 4)) ^ ((lane >> 1) & 7));
    const int64_t end = a.N - b.col0 < (int64_t)BN * a.span ? a.N : b.col0 + BN * a.span;
    const int8_t* bblk;
    auto load_at = [&](auto ic, int t, char* st) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        constexpr bool is_a = i < kAI;
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc((void*)(is_a ? ablk : bblk), 0, (int)kSpan, kRsrcWord3);
        // (the step's offset past kOutside stays outside)
        const uint32_t at = 128u * (uint32_t)(first + t);
        const uint32_t v = place[i] + at < (uint32_t)bytes ? voff[i] : kOutside;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            r, (lds_void_t*)(st + (is_a ? 0 : kA) + (is_a ? wave * kAI + i : wave * kBI + i - kAI) * 1024), 16, v, at, 0,
            ONCE && !is_a ? kNontemporal : 0);
    };
    // The first loads of the block at b.col0.
    auto begin = [&]() __attribute__((always_inline)) {
        bblk = a.b + ((int64_t)b.expert * a.N + b.col0) * a.ldb;
#pragma unroll
        for (int i = kAI; i < kLoads; ++i) {
            const int r = (wave * kBI + i - kAI) * 8 + lane / 8;
            voff[i] = r < a.N - b.col0 ? (uint32_t)(r * a.ldb) + place[i] : kOutside;
        }
        static_for<ST>([&](auto uc) __attribute__((always_inline)) {
            static_for<kLoads>([&](auto ic) __attribute__((always_inline)) { load_at(ic, decltype(uc)::value, stage(uc)); });
        });
    };
    begin();
    bool more;
    do {
        u32x4_t fa[2][MI], fb[2][NJ];
        i32x4_t acc[MI][NJ];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};

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

        wait_and_barrier<(ST - 1) * kLoads>();
        if (tid < BM) s_row[tid] = row_scale;
        if (tid < BN) {
            s_scale[tid] = col_scale;
            s_bias[tid] = col_bias;
        }
        static_for<MI + NJ>([&](auto ic) __attribute__((always_inline)) {
            read_one(ic, std::integral_constant<int, 0>{}, st0, fa[0], fb[0]);
        });
        int t = 0;
        for (; t + ST <= steps; t += ST)
            static_for<ST>([&](auto uc) __attribute__((always_inline)) { step(uc, t + decltype(uc)::value); });
        rest(rest, std::integral_constant<int, 0>{}, t);
        // every wave has read the stages, and no load is writing LDS
        wait_and_barrier<0>();

        const int64_t col = b.col0 + wn * WTN;
        if constexpr (!EXPERTS) {
            if (parts > 1) {            // sums of this part of k, for int8_join_kernel
                const int64_t ld = partial_cols(a.N);
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    const int r = wm * WTM + 16 * i + (lane & 15);
                    if (r >= b.rows) continue;
                    int32_t* const to = a.partial + ((int64_t)part * a.M + b.row0 + r) * ld;
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const int64_t n = col + 16 * j + 4 * (lane >> 4);
                        if (n < a.N) *reinterpret_cast<i32x4_t*>(to + n) = acc[i][j];
                    }
                }
                return;
            }
        }
        f32x4_t scale[NJ], bias[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            scale[j] = *reinterpret_cast<const f32x4_t*>(s_scale + wn * WTN + 16 * j + 4 * (lane >> 4));
            bias[j] = *reinterpret_cast<const f32x4_t*>(s_bias + wn * WTN + 16 * j + 4 * (lane >> 4));
        }
        more = EXPERTS && (b.col0 += BN) < end;
        if (more) {                     // the next block's first loads ahead of this one's results
            look_up();
            begin();
        }

        // A wave's part of the block, 16 rows at a time: through LDS into whole rows.
        char* const out = s_out[wave];
        static_for<MI>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            const int r0 = wm * WTM + 16 * i;
            const float row = s_row[r0 + (lane & 15)];
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                *reinterpret_cast<u32x2_t*>(out + (lane & 15) * kOutRow + 32 * j + 8 * (lane >> 4)) =
                    finish<DT>(acc[i][j], row, scale[j], bias[j]);
            constexpr int kChunks = WTN / 8;            // of a row
#pragma unroll
            for (int q = 0; q < 16 * kChunks / 64 + (16 * kChunks % 64 != 0); ++q) {
                const int at = 64 * q + lane, r = at / kChunks, ch = at % kChunks;
                if (r >= 16) continue;
                const u32x4_t v = *reinterpret_cast<const u32x4_t*>(out + r * kOutRow + 16 * ch);
                if (EXPERTS ? s_from[EXPERTS ? r0 + r : 0] < 0 : r0 + r >= b.rows) continue;
                write_chunk(a.c + (b.row0 + r0 + r) * a.ldc + col + 8 * ch, v, a.N - col - 8 * ch);
            }
        });
    } while (more);
}

// ---- few blocks -------------------------------------------------------------
// 16 rows and 16 columns to a workgroup, whose four waves divide k: no barriers until the
// waves' sums meet, for products of so few blocks that a ring's steps would be waited for one
// by one (1 x 4096 x 4096 5.5 us, in the ring's blocks of 32 x 32 7.3; 16 x 256 x 1024 3.4 and
// 3.7). Weights and rows come from memory straight into the MFMA's registers.
//
// A load takes whole lines of 128 bytes, eight lanes a row: lane l reads chunk l / 8 of row
// l % 8, and of row 8 + l % 8 with a second load. An MFMA wants 16 rows in the 16 lanes of a
// row of lanes; with the halves of those swapped between the two loads, the first MFMA gets
// the even chunks of all 16 rows, the second one the odd ones. (Which k an MFMA sums in which
// order does not matter, as long as a and b agree.)
struct Pair {
    u32x4_t even, odd;
};
__device__ __forceinline__ Pair lines(u32x4_t low, u32x4_t high) {
    Pair p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        // row_ror:8 into lanes 8 .. 15 (banks 2, 3) or 0 .. 7 of each row of 16
        p.even[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)low[e], (int)high[e], 0x128, 0xF, 0xC, false);
        p.odd[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)high[e], (int)low[e], 0x128, 0xF, 0x3, false);
    }
    return p;
}

template <int DT>
__global__ __launch_bounds__(256) void int8_few_kernel(const Int8Args a) {
    constexpr int W = 4, U = 2;
    __shared__ i32x4_t s_sum[W][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Block b;
    find_block<16, false>(a, blockIdx.x, 16, b);
    const int bytes = (int)int8_row_bytes(a.K), steps = (bytes + 127) / 128;

    // rows and columns that are not there stand for one that is
    const int8_t* pa[2];
    const int8_t* pb[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = 8 * h + (lane & 7);
        const int64_t n = b.col0 + r;
        pa[h] = a.a + (b.row0 + (r < b.rows ? r : 0)) * a.lda + 16 * (lane >> 3);
        pb[h] = a.b + (n < a.N ? n : a.N - 1) * a.ldb + 16 * (lane >> 3);
    }
    i32x4_t acc = {0, 0, 0, 0};
    auto at = [](const int8_t* p) { return *reinterpret_cast<const u32x4_t*>(p); };
    auto multiply = [&](const u32x4_t (&fa)[2], const u32x4_t (&fb)[2]) {
        const Pair x = lines(fa[0], fa[1]), y = lines(fb[0], fb[1]);
        acc = mfma16(y.even, x.even, acc);
        acc = mfma16(y.odd, x.odd, acc);
    };

    // a wave's steps of 128 bytes
    const int per = (steps + W - 1) / W;
    int s = wave * per;
    const int end = s + per < steps ? s + per : steps;
    for (; s + U <= end && 128 * (s + U) <= bytes; s += U) {
        u32x4_t fa[U][2], fb[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fb[u][h] = at(pb[h] + 128 * (s + u));
                fa[u][h] = at(pa[h] + 128 * (s + u));
            }
#pragma unroll
        for (int u = 0; u < U; ++u) multiply(fa[u], fb[u]);
    }
    for (; s < end; ++s) {          // one at a time; the last one ends with the row
        u32x4_t fa[2], fb[2];
        const bool there = 128 * s + 16 * (lane >> 3) < bytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            fa[h] = fb[h] = u32x4_t{0u, 0u, 0u, 0u};
            if (there) {
                fb[h] = at(pb[h] + 128 * s);
                fa[h] = at(pa[h] + 128 * s);
            }
        }
        multiply(fa, fb);
    }

    s_sum[wave][lane] = acc;
    __syncthreads();
    const int r = lane & 15;
    const int64_t n = b.col0 + 4 * (lane >> 4);
    if (wave != 0 || r >= b.rows || n >= a.N) return;
    const i32x4_t sum = (s_sum[0][lane] + s_sum[1][lane]) + (s_sum[2][lane] + s_sum[3][lane]);
    const Columns of = columns_of<DT>(a, n);
    const u32x2_t v = finish<DT>(sum, a.K > 0 ? a.a_scales[b.row0 + r] : 0.0f, of.scale, of.bias);
    write_four(a.c + (b.row0 + r) * a.ldc + n, v, a.N - n);
}

// The result from the sums of the parts of k: four columns of a row per thread. (Whole
// numbers: their order does not matter.)
constexpr int kJoinThreads = 256;
template <int DT>
__global__ __launch_bounds__(kJoinThreads) void int8_join_kernel(const Int8Args a) {
    const int64_t ld = partial_cols(a.N), at = ((int64_t)blockIdx.x * kJoinThreads + threadIdx.x) * 4;
    if (at >= a.M * ld) return;
    const int64_t m = at / ld, n = at % ld;
    i32x4_t sum = {0, 0, 0, 0};
    for (int p = 0; p < a.parts; ++p) sum += *reinterpret_cast<const i32x4_t*>(a.partial + (int64_t)p * a.M * ld + at);
    const Columns of = columns_of<DT>(a, n);
    const u32x2_t v = finish<DT>(sum, a.a_scales[m], of.scale, of.bias);
    write_four(a.c + m * a.ldc + n, v, a.N - n);
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

template <bool EXPERTS>
hipError_t launch_any(int dtype, const Int8Args& a, const Int8Form& f, hipStream_t s) {
    const dim3 grid((uint32_t)blocks_of<EXPERTS>(a, f.rows, f.cols * f.span), (uint32_t)f.parts);
    const auto block = [&](auto bm, auto bn, auto st) {
        constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value, ST = decltype(st)::value;
        if constexpr (BN <= 64) {
            if (weights_once(a, f, EXPERTS))
                return launch(dtype == FO_FP16 ? int8_block_kernel<FO_FP16, BM, BN, ST, EXPERTS, true>
                                               : int8_block_kernel<FO_BF16, BM, BN, ST, EXPERTS, true>, grid, 256, s, a);
        }
        return launch(dtype == FO_FP16 ? int8_block_kernel<FO_FP16, BM, BN, ST, EXPERTS, false>
                                       : int8_block_kernel<FO_BF16, BM, BN, ST, EXPERTS, false>, grid, 256, s, a);
    };
    if (f.rows == 256) return launch_int8_tile(dtype, EXPERTS, grid.x, a, s);
    if constexpr (!EXPERTS) {
        if (f.cols == 64 && f.rows == 128) return block(Int<128>(), Int<64>(), Int<3>());
        if (f.rows == 128 && f.stages == 3) return block(Int<128>(), Int<128>(), Int<3>());
    }
    if (f.rows == 128) return block(Int<128>(), Int<128>(), Int<2>());
    if (f.cols == 64) return block(Int<64>(), Int<64>(), Int<4>());
    if constexpr (!EXPERTS) {
        if (f.rows == 64) return block(Int<64>(), Int<32>(), Int<4>());
        if (f.rows == 16)
            return launch(dtype == FO_FP16 ? int8_few_kernel<FO_FP16> : int8_few_kernel<FO_BF16>, grid, 256, s, a);
    }
    return block(Int<32>(), Int<32>(), Int<4>());
}

}  // namespace

int64_t int8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    const Int8Form f = product_form(M, N, K);
    return M > 0 && N > 0 && f.parts > 1 ? f.parts * M * partial_cols(N) * 4 : 0;
}

bool int8_launchable(const Int8Args& a, bool experts) {
    const Int8Form f = experts ? experts_form(a) : product_form(a.M, a.N, a.K);
    const int64_t blocks = experts ? blocks_of<true>(a, f.rows, f.cols * f.span) : blocks_of<false>(a, f.rows, f.cols * f.span);
    return blocks <= (int64_t)UINT32_MAX / 256;
}

hipError_t launch_int8_product(int dtype, const Int8Args& args, hipStream_t s) {
    Int8Args a = args;
    const Int8Form f = product_form(a.M, a.N, a.K);
    a.parts = f.parts;
    a.span = f.span;
    const hipError_t e = launch_any<false>(dtype, a, f, s);
    if (e != hipSuccess || f.parts == 1) return e;
    const int64_t threads = a.M * partial_cols(a.N) / 4;
    return launch(dtype == FO_FP16 ? int8_join_kernel<FO_FP16> : int8_join_kernel<FO_BF16>,
                  (uint32_t)((threads + kJoinThreads - 1) / kJoinThreads), kJoinThreads, s, a);
}
hipError_t launch_int8_experts(int dtype, const Int8Args& args, hipStream_t s) {
    Int8Args a = args;
    const Int8Form f = experts_form(a);
    a.span = f.span;
    return launch_any<true>(dtype, a, f, s);
}

}  // namespace fo
