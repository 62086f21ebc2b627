// Tokens sorted by expert and back (the two sides of an All-to-All between a
// router and its experts).
//
// Sort: a stable counting sort of the pairs (token t, choice k), p = t K + k, by
// expert. A workgroup takes a run of pairs, each of its waves a part of the
// run: the parts' counts per expert (LDS) summed up in order give each part's
// first place with each expert, and within a wave the lanes of one expert find
// each other by ballots, so that a pair's place is a sum of counts and no
// atomic's order shows. Several workgroups: a first launch writes their counts,
// which every workgroup of the second one adds up.
//
// Permute, combine and the combine's backward pass move whole rows of H values
// and are bound by memory: each row is read once (a token's row stays in
// registers while it goes to its K places, a token's K rows are in flight
// together). They write past the caches (nontemporal), which leaves these to what
// is read: 16384 tokens to 8 of 128 experts, H 2048, 115 -> 103 us; 4096 tokens from
// 8 experts, H 7168, 104 -> 95; 4096 tokens, 2 experts, combine with a checkpoint and
// its backward pass in turn, 53 + 42 -> 43 + 44. With the combine's rows loaded past
// the caches too, four of a token's at a time: 90 us (5.9 TB/s), and 42 + 43.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "rowops.h"
#include "rows.h"

namespace fo {
namespace {

constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;
// Pairs that one workgroup sorts by itself: one launch and no workspace. The kernels'
// time would draw the line lower (us, 8 / 64 / 256 experts: alone 1024 pairs 4.2 / 5.4 / 8.6,
// 2048 5.6 / 7.2 / 10.7, 4096 8.4 / 10.6 / 14.9, 8192 14.1 / 17.9 / 23.1; 8200 in two launches
// 9.1 / 10.0 / 11.8, 131072 10.3 / 11.2 / 13.7), a second launch aside.
constexpr int64_t kSortAlone = 8192;
constexpr int64_t kSortRun = 2048;          // pairs of one workgroup among several, at least
constexpr int kSortBlocks = 256;            // workgroups, at most
constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kBatch = 4;                   // rows of a token in flight

template <typename ID>
__device__ __forceinline__ int expert_of(const ID* ids, int64_t p, int64_t end, int experts) {
    if (p >= end) return -1;
    const ID e = ids[p];
    return e >= 0 && e < (ID)experts ? (int)e : -1;
}

template <typename ID>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs a, int64_t run) {
    __shared__ int32_t s_count[kMaxExperts];
    for (int e = threadIdx.x; e < a.experts; e += kSortThreads) s_count[e] = 0;
    __syncthreads();
    const int64_t first = blockIdx.x * run, end = first + run < a.pairs ? first + run : a.pairs;
    for (int64_t p = first + threadIdx.x; p < end; p += kSortThreads) {
        const int e = expert_of(static_cast<const ID*>(a.ids), p, end, a.experts);
        if (e >= 0) atomicAdd(&s_count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kSortThreads) a.hist[(int64_t)blockIdx.x * a.experts + e] = s_count[e];
}

template <typename ID>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const SortArgs a, int64_t run) {
    __shared__ int32_t s_place[kSortWaves][kMaxExperts];
    __shared__ int32_t s_first[kMaxExperts + 1], s_total[kMaxExperts], s_before[kMaxExperts], s_wave[kSortWaves];
    const ID* ids = static_cast<const ID*>(a.ids);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, E = a.experts;
    const int64_t first = blockIdx.x * run, end = first + run < a.pairs ? first + run : a.pairs;
    const int64_t part = run / kSortWaves, begin = first + wave * part;
    const int64_t stop = begin + part < end ? begin + part : end;

    for (int i = threadIdx.x; i < kSortWaves * E; i += kSortThreads) s_place[i / E][i % E] = 0;
    __syncthreads();
    for (int64_t p = begin + lane; p < stop; p += 64) {
        const int e = expert_of(ids, p, stop, E);
        if (e >= 0) atomicAdd(&s_place[wave][e], 1);
    }
    __syncthreads();
    // all workgroups' counts and those ahead of this one: kSortThreads / E threads per
    // expert, each over its share of the workgroups
    for (int e = threadIdx.x; e < E; e += kSortThreads) s_total[e] = s_before[e] = 0;
    __syncthreads();
    if (gridDim.x > 1) {
        const int shares = E < kSortThreads ? kSortThreads / E : 1;
        const int share = E < kSortThreads ? (int)threadIdx.x / E : 0;
        for (int e = threadIdx.x - share * E; share < shares && e < E; e += kSortThreads) {
            int32_t before = 0, total = 0;
#pragma unroll 8
            for (int b = share; b < (int)gridDim.x; b += shares) {
                const int32_t n = a.hist[(int64_t)b * E + e];
                before += b < (int)blockIdx.x ? n : 0;
                total += n;
            }
            atomicAdd(&s_total[e], total);
            atomicAdd(&s_before[e], before);
        }
        __syncthreads();
    }
    // per expert: the parts' counts to their first places within the expert
    for (int e = threadIdx.x; e < E; e += kSortThreads) {
        const int32_t before = s_before[e];
        int32_t at = before;
        for (int w = 0; w < kSortWaves; ++w) {
            const int32_t n = s_place[w][e];
            s_place[w][e] = at;
            at += n;
        }
        if (gridDim.x == 1) s_total[e] = at;
    }
    __syncthreads();
    // the experts' first rows: two experts per thread, padded counts summed up
    {
        int32_t mine[2], sum = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int e = 2 * threadIdx.x + j;
            mine[j] = sum;
            if (e < E) sum += (int32_t)(((uint32_t)s_total[e] + (uint32_t)a.align - 1) / (uint32_t)a.align * (uint32_t)a.align);
        }
        int32_t scan = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int32_t up = __shfl_up(scan, off, 64);
            if (lane >= off) scan += up;
        }
        if (lane == 63) s_wave[wave] = scan;
        __syncthreads();
        int32_t base = scan - sum;
        for (int w = 0; w < wave; ++w) base += s_wave[w];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int e = 2 * threadIdx.x + j;
            if (e < E) s_first[e] = base + mine[j];
            if (e == E - 1) s_first[E] = base + sum;
            if (blockIdx.x == 0) {
                if (e < E) {
                    a.offsets[e] = base + mine[j];
                    a.counts[e] = s_total[e];
                }
                if (e == E - 1) a.offsets[E] = base + sum;
            }
        }
    }
    __syncthreads();
    // padding rows belong to no pair: a wave per expert
    if (a.pair_of && a.align > 1) {
        for (int e = blockIdx.x * kSortWaves + wave; e < E; e += gridDim.x * kSortWaves)
            for (int32_t r = s_first[e] + s_total[e] + lane; r < s_first[e + 1]; r += 64) a.pair_of[r] = -1;
    }
    int bits = 0;
    while ((1 << bits) < E) ++bits;
    volatile int32_t* place = s_place[wave];
    for (int64_t p0 = begin; p0 < stop; p0 += 64) {
        const int64_t p = p0 + lane;
        const int e = expert_of(ids, p, stop, E);
        uint64_t same = __ballot(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((e >> b) & 1);
            same &= ((e >> b) & 1) ? set : ~set;
        }
        if (e >= 0) {
            const int rank = __popcll(same & ((1ull << lane) - 1));
            const int32_t slot = s_first[e] + place[e] + rank;
            a.slot_of[p] = slot;
            if (a.pair_of) a.pair_of[slot] = (int32_t)p;
        } else if (p < stop) {
            a.slot_of[p] = -1;
        }
        __builtin_amdgcn_wave_barrier();
        // the last lane of each expert moves its part's place on
        if (e >= 0 && (same >> lane) == 1ull) place[e] = place[e] + __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
}

// A thread's token and chunk in a grid of T tokens of `slices` times L chunks: L
// lanes to a slice (64, or fewer where a row is shorter than a wave).
struct Unit {
    int32_t t, c;
};
template <int L>
__device__ __forceinline__ Unit unit_of(uint32_t slices) {
    const uint32_t group = threadIdx.x / L;
    const uint32_t u = blockIdx.x * (kThreads / L) + (L < 64 ? group : (uint32_t)__builtin_amdgcn_readfirstlane(group));
    Unit r;
    r.t = (int32_t)(u / slices);
    r.c = (int32_t)(u - (uint32_t)r.t * slices) * L + (int)(threadIdx.x % L);
    return r;
}

// Rows between an expert's last and the next expert's first are zeroed: `per`
// workgroups per expert, a wave per row at a time.
__device__ __forceinline__ void zero_padding(const RouteArgs& a, uint16_t* rows, int64_t ld, uint32_t block, int per) {
    const int e = (int)(block / (uint32_t)per), lane = threadIdx.x & 63;
    const int waves = blockDim.x >> 6;
    const int wave = (int)(block % (uint32_t)per) * waves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t from = a.offsets[e] + a.counts[e], to = a.offsets[e + 1];
    from = from < 0 ? 0 : from;
    to = to > a.capacity ? a.capacity : to;
    for (int64_t r = (int64_t)from + wave; r < to; r += per * waves) {
        uint16_t* row = rows + r * ld;
        for (int64_t h = 8 * lane; h < a.H; h += 512) write_chunk(row + h, u32x4_t{0u, 0u, 0u, 0u}, a.H - h);
    }
}

__device__ __forceinline__ bool is_row(const RouteArgs& a, int32_t slot) { return slot >= 0 && slot < a.capacity; }

template <int L>
__global__ __launch_bounds__(kThreads) void permute_kernel(const RouteArgs a, uint32_t slices, uint32_t blocks, int per) {
    if (blockIdx.x >= blocks) return zero_padding(a, a.rows, a.ldr, blockIdx.x - blocks, per);
    const Unit u = unit_of<L>(slices);
    if (u.t >= a.T) return;
    const int64_t h = 8 * (int64_t)u.c, left = a.H - h;
    const u32x4_t v = read_chunk<kCached>(a.x + u.t * a.ldx + h, left);
    for (int k = 0; k < a.K; ++k) {
        const int32_t slot = a.slot_of[(int64_t)u.t * a.K + k];
        if (is_row(a, slot)) write_chunk(a.rows + slot * a.ldr + h, v, left);
    }
}

// FMT: -1, or the format of the checkpoint that the rows are packed into. kBatch of
// a token's rows are in flight together.
template <int DT, int FMT, int L>
__global__ __launch_bounds__(kThreads) void combine_kernel(const RouteArgs a, uint32_t slices) {
    const Unit u = unit_of<L>(slices);
    if (u.t >= a.T) return;
    const int64_t h = 8 * (int64_t)u.c, left = a.H - h;
    const int64_t blocks = (a.H + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK, first = (int64_t)u.t * a.K;
    float sum[8] = {};
    for (int k0 = 0; k0 < a.K; k0 += kBatch) {
        int32_t slot[kBatch];
        float w[kBatch];
        u32x4_t v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            slot[j] = k0 + j < a.K ? a.slot_of[first + k0 + j] : -1;
            w[j] = k0 + j < a.K && a.weights ? a.weights[first + k0 + j] : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            v[j] = u32x4_t{0u, 0u, 0u, 0u};
            if (is_row(a, slot[j])) v[j] = read_chunk<kStreamed>(a.rows + slot[j] * a.ldr + h, left);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (!is_row(a, slot[j])) continue;
            float f[8];
            widen<DT>(v[j], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += w[j] * f[e];
            if constexpr (FMT >= 0) {
                if (u.c < 4 * blocks)
                    pack_chunk<DT, FMT>(f, u.c, a.packed + slot[j] * blocks * FO_PACK_BLOCK, a.scales + slot[j] * blocks);
            }
        }
    }
    write_chunk(a.out + u.t * a.ldo + h, narrow<DT>(sum), left);
}

// L lanes per pair along its row (fewer than a wave, a wave or the whole workgroup):
// drows[slot] = w dout[t] and dw = <dout[t], rows[slot]>. SRC: where the rows come
// from: 0 themselves, 1 + format a checkpoint of them.
template <int DT, int SRC, int L>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(const RouteArgs a, uint32_t blocks, int per) {
    static_assert(L <= 64 || L == kThreads, "a workgroup's pair meets once");
    __shared__ float s_dot[kWaves];
    if (blockIdx.x >= blocks) return zero_padding(a, a.out, a.ldo, blockIdx.x - blocks, per);
    const int group = threadIdx.x / L, lane = threadIdx.x % L;
    const int64_t p = (int64_t)blockIdx.x * (kThreads / L) + (L < 64 ? group : __builtin_amdgcn_readfirstlane(group));
    if (p >= (int64_t)a.T * a.K) return;
    const int32_t slot = a.slot_of[p];
    if (!is_row(a, slot)) {
        if (lane == 0 && a.dweights) a.dweights[p] = 0.0f;
        return;
    }
    const float w = a.weights ? a.weights[p] : 1.0f;
    const int64_t blocks32 = (a.H + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK;
    const uint16_t* grow = a.x + (uint32_t)p / (uint32_t)a.K * a.ldx;
    const uint16_t* row = SRC == 0 && a.dweights ? a.rows + slot * a.ldr : nullptr;
    const uint8_t* packed = SRC ? a.packed + slot * blocks32 * FO_PACK_BLOCK : nullptr;
    const uint8_t* scales = SRC ? a.scales + slot * blocks32 : nullptr;
    uint16_t* out = a.out ? a.out + slot * a.ldo : nullptr;
    float dot = 0.0f;
    for (int64_t h = 8 * lane; h < a.H; h += 8 * L) {
        const int64_t left = a.H - h;
        float g[8];
        widen<DT>(read_chunk<kCached>(grow + h, left), g);
        if (a.dweights) {
            float f[8];
            if constexpr (SRC == 0) widen<DT>(read_chunk<kStreamed>(row + h, left), f);
            else decode8<SRC - 1>(*reinterpret_cast<const u32x2_t*>(packed + h), scale_of(scales[h / FO_PACK_BLOCK]), f);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot += g[e] * f[e];
        }
        if (out) {
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] *= w;
            write_chunk(out + h, narrow<DT>(g), left);
        }
    }
    if (a.dweights) {
        dot = lanes_sum<(L < 64 ? L : 64)>(dot);
        if constexpr (L > 64) {
            if ((threadIdx.x & 63) == 0) s_dot[threadIdx.x >> 6] = dot;
            __syncthreads();
            dot = 0.0f;
#pragma unroll
            for (int v = 0; v < kWaves; ++v) dot += s_dot[v];
        }
        if (lane == 0) a.dweights[p] = dot;
    }
}

template <int N>
using Int = std::integral_constant<int, N>;
// Lanes to a slice of a row of H values: a wave, or the most whose last slice leaves at
// most an eighth of the row's lanes idle; calls go(lanes) with them. (262144 tokens of
// 64 values, eight choices, a wave -> 8 lanes: permute 158 -> 55 us, combine 175 -> 53,
// its backward pass 631 -> 133; 29127 tokens of 576, two slices of a wave -> nine of 8
// lanes: combine with a checkpoint 106 -> 81, backward 149 -> 116.)
template <typename F>
hipError_t for_lanes(int64_t H, F go) {
    auto fits = [&](int64_t lanes) { return (H + 8 * lanes - 1) / (8 * lanes) * (8 * lanes) <= H + H / 8; };
    if (fits(64)) return go(Int<64>());
    if (fits(32)) return go(Int<32>());
    if (fits(16)) return go(Int<16>());
    return go(Int<8>());
}
// Slices of a row, and workgroups of a launch, with L lanes to a slice.
template <int L>
uint32_t slices_of(int64_t H) {
    return (uint32_t)((H + 8 * L - 1) / (8 * L));
}
template <int L>
uint32_t workgroups(const RouteArgs& a) {
    return (uint32_t)(((int64_t)a.T * slices_of<L>(a.H) + kThreads / L - 1) / (kThreads / L));
}
// Workgroups per expert that zero padding rows.
int padding_blocks(const RouteArgs& a) { return a.offsets ? std::max(1, std::min(16, 256 / a.E)) : 0; }

}  // namespace

int64_t sort_blocks(int64_t pairs) {
    return pairs <= kSortAlone ? 1 : std::min<int64_t>((pairs + kSortRun - 1) / kSortRun, kSortBlocks);
}

hipError_t launch_sort(const SortArgs& a, hipStream_t s) {
    const int64_t blocks = sort_blocks(a.pairs);
    // whole steps of every wave
    const int64_t run = ((a.pairs + blocks - 1) / blocks + kSortThreads - 1) / kSortThreads * kSortThreads;
    const bool wide = a.id_bytes == 8;
    if (blocks > 1) {
        const hipError_t e = launch(wide ? sort_count_kernel<int64_t> : sort_count_kernel<int32_t>, (uint32_t)blocks,
                                    kSortThreads, s, a, run);
        if (e != hipSuccess) return e;
    }
    return launch(wide ? sort_place_kernel<int64_t> : sort_place_kernel<int32_t>, (uint32_t)blocks, kSortThreads, s, a, run);
}

hipError_t launch_permute(const RouteArgs& a, hipStream_t s) {
    const int per = padding_blocks(a);
    return for_lanes(a.H, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const uint32_t blocks = workgroups<L>(a);
        return launch(permute_kernel<L>, blocks + (uint32_t)(per * a.E), kThreads, s, a, slices_of<L>(a.H), blocks, per);
    });
}

hipError_t launch_combine(int dtype, const RouteArgs& a, hipStream_t s) {
    return for_lanes(a.H, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        auto from = [&](auto dt) {
            constexpr int DT = decltype(dt)::value;
            return launch(!a.packed                     ? combine_kernel<DT, -1, L>
                          : a.format == FO_PACK_INT8 ? combine_kernel<DT, FO_PACK_INT8, L>
                                                     : combine_kernel<DT, FO_PACK_E4M3, L>,
                          workgroups<L>(a), kThreads, s, a, slices_of<L>(a.H));
        };
        return dtype == FO_FP16 ? from(Int<FO_FP16>()) : from(Int<FO_BF16>());
    });
}

hipError_t launch_combine_backward(int dtype, const RouteArgs& a, hipStream_t s) {
    const int64_t pairs = (int64_t)a.T * a.K;
    const int per = a.out ? padding_blocks(a) : 0;
    auto go = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const uint32_t blocks = (uint32_t)((pairs + kThreads / L - 1) / (kThreads / L));
        auto from = [&](auto dt) {
            constexpr int DT = decltype(dt)::value;
            return launch(!a.packed                     ? combine_backward_kernel<DT, 0, L>
                          : a.format == FO_PACK_INT8 ? combine_backward_kernel<DT, 1 + FO_PACK_INT8, L>
                                                     : combine_backward_kernel<DT, 1 + FO_PACK_E4M3, L>,
                          blocks + (uint32_t)(per * a.E), kThreads, s, a, blocks, per);
        };
        return dtype == FO_FP16 ? from(Int<FO_FP16>()) : from(Int<FO_BF16>());
    };
    // Four waves per pair while the pairs are too few to fill the device with one each
    // (us, one wave -> four, H 7168 from an int8 checkpoint: 128 pairs 11.4 -> 5.1, 1024
    // 12.6 -> 7.7, 2048 14.1 -> 12.6, 4096 17.5 -> 22.6, 8192 32.9 -> 42.8). A workgroup
    // per token with all of its rows in flight read dout once but wrote in more places
    // at a time: 8192 pairs of two choices 43 -> 58 to 66.
    if (pairs <= 2048 && a.H > 512) return go(Int<kThreads>());
    return for_lanes(a.H, go);
}

}  // namespace fo
