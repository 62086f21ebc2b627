// Products of 8-bit matrices in tiles of 256 x 256 (gfx950).
//
// Four waves, one per SIMD, each on 128 x 128 of the tile: an operand byte that is read
// from LDS feeds 64 products, twice as many as in a 128 x 128 tile's waves of 64 x 64, whose
// LDS reads bound them. k steps of 128 move from memory straight into an LDS ring of two
// stages; v_mfma_i32_16x16x64_i8 in inline asm with the accumulators tied in place, every
// LDS read and load issue in the shadow of an MFMA. The scales, the bias and the rows' places
// wait in LDS from the tile's start.
//
// Workgroups compute one tile after another, and a tile's first loads go ahead of the results
// of the one before it: tiles of one size end together, and memory would see 32 MB of results
// and then 32 MB of operands, with no compute unit at work (14 us a tile; 4 are left). Which
// tiles are a workgroup's is fixed by the counts: experts' tiles of unequal height leave some
// workgroups more to do, but each finds its next tile and rows during the one before (8192
// tokens to 8 of 128 experts, 2880x1440: 427 us; a workgroup per tile 476).
// 8192x8192x8192 403 us, 2.7 POPS. 8192x8192x3584: the matrix units are busy for 58 % of the cycles,
// 8192x14336x4096 63 %; the power limit leaves 1.85 to 2.0 of 2.4 GHz. A step's 128 MFMAs a wave take
// 2048 cycles of the about 2900 between its barriers, and the order of its reads and loads makes no
// difference. Experts of 512 rows each, 2048x7168: 2.2 POPS, of as many on average 1.9 (48 % busy), a
// tile's weights coming from memory, not from the caches; loads past the caches' keeping help where one tile reads an expert's weights (256 rows each 512 -> 451 us), and cost as
// much where three do (528 rows each 539 -> 567): not taken.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "int8_device.h"
#include "rows.h"
#include "rowops.h"

namespace fo {
namespace {

// The accumulator is tied in place (dst = srcC), in VGPRs with KEEP_V and in AGPRs without:
// with 256 accumulator registers the compiler's own MFMAs get copied between the register
// files. The compiler does not track the hazards of these instructions: accumulators are
// never written by VALU right before one (the first MFMA of a tile takes srcC = 0) and read
// only after the wait that ends the main loop.
template <bool FIRST, bool KEEP_V>
__device__ __forceinline__ void mfma_tied(i32x4_t& c, const u32x4_t& x, const u32x4_t& y) {
    if constexpr (FIRST && KEEP_V) asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, 0" : "=v"(c) : "v"(x), "v"(y));
    else if constexpr (FIRST) asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, 0" : "=a"(c) : "v"(x), "v"(y));
    else if constexpr (KEEP_V) asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+v"(c) : "v"(x), "v"(y));
    else asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(x), "v"(y));
}

constexpr int kStage = (256 + 256) * 128;
constexpr int kOutRow = 128 * 2 + 16;               // a wave's 128 columns of a row, on their way out

// A tile's waves are 2 x 2, of 128 x 128 each; or, where it is the rest of an expert's rows
// and has at most 128, side by side, of 128 x 64 (half the MFMAs; the same loads).
template <int DT, bool EXPERTS>
__global__ __launch_bounds__(256, 1) void int8_tile_kernel(const Int8Args a) {
    constexpr int BM = 256, BN = 256, MI = 8, kA = BM * 128;
    constexpr int kAI = BM / 32, kBI = BN / 32, kLoads = kAI + kBI;      // load instructions per wave and step
    constexpr int kVRows = 2;                            // accumulator block rows held in VGPRs
    constexpr int kStores = 32;                          // store instructions of 128 x 128 results
    // (the stages are separate arrays, so that the compiler can tell the stage being read
    // from the stage being filled)
    __shared__ __attribute__((aligned(1024))) char st0[kStage];
    __shared__ __attribute__((aligned(1024))) char st1[kStage];
    __shared__ __attribute__((aligned(16))) char s_out[4 * 16 * kOutRow];
    // of the tile's columns and rows, for its results; of the next tile's rows
    __shared__ __attribute__((aligned(16))) float s_scale[256], s_bias[256], s_row[256];
    __shared__ bool s_there[256];
    __shared__ int s_from[EXPERTS ? 256 : 1];            // row of a, or -1
    __shared__ ExpertRows s_experts[EXPERTS ? FO_ROUTE_MAX_EXPERTS : 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t bytes = (uint32_t)int8_row_bytes(a.K);
    const int steps = (int)((bytes + 127) / 128);
    const bool gather = EXPERTS && a.pair_of;

    Block b;
    int p = blockIdx.x;
    // The tile at position p; by experts from what LDS has of them.
    Survey experts = {0, 0};
    const auto rows_of = [&](int e) { return s_experts[EXPERTS ? e : 0]; };
    const auto find = [&](Block& at) __attribute__((always_inline)) {
        if constexpr (EXPERTS) return locate<BM>(a, experts, rows_of, p, BN, at);
        else return p < a.blocks && find_block<BM, false>(a, p, BN, at);
    };
    if constexpr (EXPERTS) {
        for (int e = tid; e < a.E; e += 256) s_experts[e] = expert_rows(a, e);
        __syncthreads();
        experts = survey<BM>(a, rows_of);
    }
    if (!find(b)) return;
    if constexpr (EXPERTS) {
        s_from[tid] = (int)source_row<true>(a, b, tid);
        __syncthreads();
    }

    // A load instruction fills 1 KB: 8 operand rows of 128 bytes, chunk c of row r at slot
    // c ^ ((r / 2) % 8). A lane's offset from the operand's base, or kOutside for a row that
    // is not there; its place in the row goes by whether the instruction's number is odd.
    uint32_t voff[kLoads], place[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) place[i] = 16u * (uint32_t)((lane & 7) ^ ((4 * i + lane / 16) & 7));
    const int8_t* ablk;
    const int8_t* bblk;
    int cols;
    // What the epilogue wants to know of column `tid` and row `tid`, looked up ahead of the
    // first loads and put into LDS at the first step's barrier.
    float col_scale = 0.0f, row_scale = 0.0f;
    uint16_t col_bias = 0;
    bool there = false;
    auto set_up = [&]() __attribute__((always_inline)) {
        int lane_s = lane;              // formed anew for each tile: kept across it, the offsets go to scratch memory
        asm volatile("" : "+v"(lane_s));
        ablk = gather ? a.a : a.a + b.row0 * a.lda;
        bblk = a.b + ((int64_t)b.expert * a.N + b.col0) * a.ldb;
        cols = (int)(a.N - b.col0 < BN ? a.N - b.col0 : BN);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = (i < kAI ? wave * kAI + i : wave * kBI + i - kAI) * 8 + lane_s / 8;
            if (i < kAI) {
                const int from = EXPERTS ? s_from[EXPERTS ? r : 0] : r < b.rows ? r : -1;
                voff[i] = from < 0 ? kOutside : (uint32_t)((gather ? from : r) * a.lda) + place[i & 1];
            } else {
                voff[i] = r < cols ? (uint32_t)(r * a.ldb) + place[i & 1] : kOutside;
            }
        }
        const int64_t from = EXPERTS ? s_from[EXPERTS ? tid : 0] : source_row<false>(a, b, tid);
        there = from >= 0;
        if (there) row_scale = a.a_scales[from];
        if (tid < cols) {
            const int64_t at = (int64_t)b.expert * a.N + b.col0 + tid;
            col_scale = a.b_scales[at];
            if (a.bias) col_bias = a.bias[at];
        }
    };
    // Load `i` of step t. Chunks past a row's end, and steps past the last, lie outside the
    // resource: zeros, no memory access (every step issues the same loads, and the wait
    // counts stay uniform). The step's offset past kOutside stays outside.
    auto load_one = [&](auto ic, int t, char* st) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc((void*)(i < kAI ? ablk : bblk), 0, (int)kSpan, kRsrcWord3);
        const uint32_t at = 128u * (uint32_t)t;
        const uint32_t v = place[i & 1] + at < bytes ? voff[i] : kOutside;
        char* const to = st + (i < kAI ? 0 : kA) + (i < kAI ? wave * kAI + i : wave * kBI + i - kAI) * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)to, 16, v, at, 0, 0);
    };
    auto begin = [&]() __attribute__((always_inline)) {
        static_for<kLoads>([&](auto ic) __attribute__((always_inline)) { load_one(ic, 0, st0); });
        static_for<kLoads>([&](auto ic) __attribute__((always_inline)) { load_one(ic, 1, st1); });
    };
    bool more;
    // Behind a tile's first loads there may be kStores of the tile before (`stores`), which
    // are not waited for.
    bool stores = false;

    // The tile b, whose first loads are on their way; and the next one's first loads.
    auto tile = [&](auto half) __attribute__((always_inline)) {
        constexpr bool HALF = decltype(half)::value;
        constexpr int NJ = HALF ? 4 : 8;
        constexpr int kGap = MI * NJ / kLoads;           // MFMAs to a load
        const int row_w = HALF ? 0 : wave / 2 * 128, col_w = HALF ? wave * 64 : wave % 2 * 128;     // the wave's part
        // Fragments: lane l feeds row l % 16 of a 16-row block with chunk 4 h + l / 16 of MFMA
        // substep h. The weights are the first operand: each lane holds four consecutive columns
        // of a row of c.
        const int a_row = (row_w + (lane & 15)) * 128, b_row = kA + (col_w + (lane & 15)) * 128;
        int cslot[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) cslot[h] = 16 * ((4 * h + (lane >> 4)) ^ ((lane >> 1) & 7));
        i32x4_t acc[MI][NJ];
        u32x4_t fa0[MI], fb0[NJ], fa1[MI], fb1[NJ];
        // MFMA m of a substep carries fragment read m of the next one (the order in which that
        // needs them) and, with `loads`, every kGap-th one a load of the stage just freed.
        auto substep = [&](const u32x4_t (&xa)[MI], const u32x4_t (&xb)[NJ], const char* rst, auto h_next, u32x4_t (&ya)[MI],
                           u32x4_t (&yb)[NJ], auto loads, int t, char* lst, auto first) __attribute__((always_inline)) {
            constexpr int h = decltype(h_next)::value;
            static_for<MI * NJ>([&](auto mc) __attribute__((always_inline)) {
                constexpr int m = decltype(mc)::value, i = m / NJ, j = m % NJ;
                if constexpr (m == 0) ya[0] = *reinterpret_cast<const u32x4_t*>(rst + a_row + cslot[h]);
                else if constexpr (m <= NJ) yb[m - 1] = *reinterpret_cast<const u32x4_t*>(rst + b_row + (m - 1) * 2048 + cslot[h]);
                else if constexpr (m < MI + NJ) ya[m - NJ] = *reinterpret_cast<const u32x4_t*>(rst + a_row + (m - NJ) * 2048 + cslot[h]);
                if constexpr (decltype(loads)::value && m % kGap == 0 && m / kGap < kLoads)
                    load_one(std::integral_constant<int, m / kGap>{}, t, lst);
                mfma_tied<decltype(first)::value, (i >= MI - kVRows)>(acc[i][j], xb[j], xa[i]);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        // Step t (its first fragments are there) in stage cur, step t + 1 in nxt: once that has
        // landed and every wave has read all of cur, step t + 2 goes there.
        constexpr std::true_type kYes{};
        constexpr std::false_type kNo{};
        constexpr std::integral_constant<int, 0> k0{};
        constexpr std::integral_constant<int, 1> k1{};
        auto step = [&](int t, char* cur, const char* nxt, auto first) __attribute__((always_inline)) {
            substep(fa0, fb0, cur, k1, fa1, fb1, kNo, 0, cur, first);
            if (decltype(first)::value && stores) wait_and_barrier<kStores>();
            else wait_and_barrier<0>();
            if constexpr (decltype(first)::value) {
                s_scale[tid] = col_scale;
                s_bias[tid] = to_f32<DT>(col_bias);
                s_row[tid] = row_scale;
                s_there[tid] = there;
            }
            substep(fa1, fb1, nxt, k0, fa0, fb0, kYes, t + 2, cur, kNo);
        };

        // (the newest kLoads operations, or kStores more where that many stores followed, may
        // be in flight: the first stage has landed)
        if (stores) wait_and_barrier<kLoads + kStores>();
        else wait_and_barrier<kLoads>();
        fa0[0] = *reinterpret_cast<const u32x4_t*>(st0 + a_row + cslot[0]);
#pragma unroll
        for (int j = 0; j < NJ; ++j) fb0[j] = *reinterpret_cast<const u32x4_t*>(st0 + b_row + j * 2048 + cslot[0]);
#pragma unroll
        for (int i = 1; i < MI; ++i) fa0[i] = *reinterpret_cast<const u32x4_t*>(st0 + a_row + i * 2048 + cslot[0]);
        step(0, st0, st1, kYes);
        // the next tile, and by experts its row `tid`, which the main loop gives time to arrive
        Block next = b;
        p += gridDim.x;
        more = find(next);
        int pair = -1;
        if (gather && more && tid < next.rows) pair = a.pair_of[next.row0 + tid];
        int t = 1;
        for (; t + 2 <= steps; t += 2) {
            step(t, st1, st0, kNo);
            step(t + 1, st0, st1, kNo);
        }
        if (t < steps) step(t, st1, st0, kNo);
        if constexpr (EXPERTS) {
            const int64_t row = next.row0 + tid, from = gather ? (pair < 0 ? -1 : pair / a.choices) : tid < next.rows ? row : -1;
            s_from[tid] = from < a.a_rows ? (int)from : -1;
        }
        // the accumulators are read only once the last MFMA's result is written
        asm volatile("s_nop 7\n s_nop 7\n s_nop 7\n s_nop 7" ::: "memory");
        wait_and_barrier<0>();          // every wave has read the stages, and no load is writing LDS

        uint16_t* const out = a.c + (b.row0 + row_w) * a.ldc + b.col0 + col_w;
        const int left = cols - col_w;
        stores = more && !HALF && cols == BN && __builtin_amdgcn_ballot_w64(s_there[row_w + lane] && s_there[row_w + 64 + lane]) == ~0ull;
        if (more) {                     // the next tile's first loads ahead of this one's results
            b = next;
            set_up();
            begin();
        }

        // A wave's part of the tile, 16 rows at a time: through LDS into whole rows.
        int lane_e = lane;
        asm volatile("" : "+v"(lane_e)); // the addresses are formed here, not ahead of the main loop
        char* const stage = s_out + wave * 16 * kOutRow;
        const float* const scale_w = s_scale + col_w + 4 * (lane_e >> 4);
        const float* const bias_w = s_bias + col_w + 4 * (lane_e >> 4);
        static_for<MI>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            const float row = s_row[row_w + 16 * i + (lane_e & 15)];
            static_for<NJ>([&](auto jc) __attribute__((always_inline)) {
                constexpr int j = decltype(jc)::value;
                *reinterpret_cast<u32x2_t*>(stage + (lane_e & 15) * kOutRow + 32 * j + 8 * (lane_e >> 4)) =
                    finish<DT>(acc[i][j], row, *reinterpret_cast<const f32x4_t*>(scale_w + 16 * j),
                               *reinterpret_cast<const f32x4_t*>(bias_w + 16 * j));
            });
            constexpr int kChunks = 2 * NJ;             // of 16 bytes, of a row
#pragma unroll
            for (int q = 0; q < 16 * kChunks / 64; ++q) {
                const int at = 64 * q + lane_e, r = at / kChunks, ch = at % kChunks;
                const u32x4_t v = *reinterpret_cast<const u32x4_t*>(stage + r * kOutRow + 16 * ch);
                uint16_t* const to = out + (int64_t)(16 * i + r) * a.ldc + 8 * ch;
                if (!HALF && stores) stream8(to, v);    // (a whole part of a tile: kStores instructions)
                else if (s_there[row_w + 16 * i + r]) write_chunk(to, v, left - 8 * ch);
            }
        });
    };

    set_up();
    begin();
    do {
        if (!EXPERTS || b.rows > 128) tile(std::false_type{});
        else tile(std::true_type{});
    } while (more);
}

}  // namespace

hipError_t launch_int8_tile(int dtype, bool experts, uint32_t blocks, const Int8Args& args, hipStream_t s) {
    Int8Args a = args;
    a.blocks = (int32_t)blocks;
    const uint32_t grid = std::min<uint32_t>(blocks, 256);      // one workgroup to a compute unit
    if (experts)
        return launch(dtype == FO_FP16 ? int8_tile_kernel<FO_FP16, true> : int8_tile_kernel<FO_BF16, true>, grid, 256, s, a);
    return launch(dtype == FO_FP16 ? int8_tile_kernel<FO_FP16, false> : int8_tile_kernel<FO_BF16, false>, grid, 256, s, a);
}

}  // namespace fo
