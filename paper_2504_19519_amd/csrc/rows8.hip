// Rows in 8-bit integers, and the RMS norm of a sum with its backward pass.
//
//   quantize:  m = max |x|, s = m / 127, code = 127 x / m to nearest even;
//   norm_add:  h = x + residual in 16 bits, r = 1 / sqrt(sum(h^2) / N + eps),
//              y = h r gamma, in 16 bits or as the codes of its row;
//   backward:  with g = dy gamma: dx = dh + r g - h r^3 sum(g h) / N,
//              dgamma = sum over rows of dy h r.
//
// All are bound by memory: a row is read once and held in registers between its sums
// and its output. The codes of y need no r: with t = h gamma, 127 y / max|y| is 127 t /
// max|t|, and t, a product of two 16-bit values, is exact in fp32. So one meeting of
// the row's threads gives the sum of squares and the maximum, and the codes are those
// of exact arithmetic (codes_of).
//
// bf16: 8192x14336 to codes 62 us (5.7 TB/s); the norm of 16384x4096 to 16 bits 86 us and its
// backward pass 86 (6.2 and 6.3 TB/s), the norm of 8192x4096 to h and codes 41 (5.7). A copy of
// 1 GiB reaches 6.25 TB/s.
//
// Rows end anywhere: the thread with a row's last chunk of eight takes the row's last
// eight values instead, some of them a second time. It writes what their own thread
// writes, and leaves them out of its sums.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "int8ops.h"
#include "rows.h"
#include "rowops.h"

namespace fo {
namespace {

template <int TH>
__device__ __forceinline__ int row_group() {
    const int group = threadIdx.x / TH;
    return TH < 64 ? group : __builtin_amdgcn_readfirstlane(group);
}

// Largest of TH neighbouring lanes' values (none below 0; NaN if one is), the same in each.
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_moved(float v) {
    return __builtin_elementwise_maximum(
        v, bit_cast<float>(__builtin_amdgcn_update_dpp(0, bit_cast<int>(v), CTRL, ROWS, 0xF, true)));
}
template <int TH>
__device__ __forceinline__ float lanes_max(float v) {
    if constexpr (TH >= 64) {
        v = max_moved<0x111, 0xF>(v);
        v = max_moved<0x112, 0xF>(v);
        v = max_moved<0x114, 0xF>(v);
        v = max_moved<0x118, 0xF>(v);
        v = max_moved<0x142, 0xA>(v);
        v = max_moved<0x143, 0xC>(v);
        return bit_cast<float>(__builtin_amdgcn_readlane(bit_cast<int>(v), 63));
    } else {
        v = max_moved<0xB1, 0xF>(v);
        v = max_moved<0x4E, 0xF>(v);
        v = max_moved<0x141, 0xF>(v);
        if constexpr (TH > 8) v = max_moved<0x140, 0xF>(v);
        if constexpr (TH > 16) {
            const u32x2_t swapped = bit_cast<u32x2_t>(
                __builtin_amdgcn_permlane16_swap(bit_cast<uint32_t>(v), bit_cast<uint32_t>(v), false, false));
            v = __builtin_elementwise_maximum(bit_cast<float>(swapped[0]), bit_cast<float>(swapped[1]));
        }
        return v;
    }
}
template <int W>
__device__ __forceinline__ float first_max(float v) {
    if constexpr (W > 1) v = max_moved<0x111, 0xF>(v);
    if constexpr (W > 2) v = max_moved<0x112, 0xF>(v);
    if constexpr (W > 4) v = max_moved<0x114, 0xF>(v);
    if constexpr (W > 8) v = max_moved<0x118, 0xF>(v);
    return bit_cast<float>(__builtin_amdgcn_readlane(bit_cast<int>(v), W - 1));
}

// The chunks of eight of a row of n values: chunk c starts at column 8 c, the last one at
// n - 8 (so that `twice` of its values are the chunk's before it as well). SMALL: rows of
// fewer than eight values, which have one, read and written in parts (of none: no chunk).
template <bool SMALL>
struct RowChunks {
    int n, last, twice;
    __device__ __forceinline__ explicit RowChunks(int64_t N)
        : n((int)N), last(((int)N - 1) >> 3), twice(SMALL ? 0 : 8 * (last + 1) - (int)N) {}
    // (unsigned, so that an access takes a row's address from scalar registers)
    __device__ __forceinline__ uint32_t column(int c) const { return (uint32_t)(8 * c - (c == last ? twice : 0)); }
    template <bool STREAMED = false>
    __device__ __forceinline__ u32x4_t read(const uint16_t* row, int c) const {
        if (c > last) return u32x4_t{0u, 0u, 0u, 0u};
        if constexpr (SMALL) return read_chunk<kCached>(row, n);
        else if constexpr (STREAMED) return stream_load8(row + column(c));
        else return load8(row + column(c));
    }
    __device__ __forceinline__ void write(uint16_t* row, int c, u32x4_t v) const {
        if (c > last) return;
        if constexpr (SMALL) write_chunk(row, v, n);
        else stream8(row + column(c), v);
    }
    // The sum over a chunk's values of their own, of term(e).
    template <typename F>
    __device__ __forceinline__ float sum(int c, F term) const {
        float s = 0.0f;
        if (SMALL || twice == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s += term(e);
        } else {
            const int from = c == last ? twice : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) s += e < from ? 0.0f : term(e);
        }
        return s;
    }
};

// What turns a row's values into codes. m: the row's largest magnitude.
struct RowCodes {
    float inverse, m;           // 127 / m, within 2^-22 of it; of values and m times `by`
    float by;                   // 1, but for an m whose reciprocal is not a normal number (or nearly so)
    bool finite;
    __device__ __forceinline__ explicit RowCodes(float m_) : m(m_) {
        by = m < 0x1p-100f ? 0x1p64f : m > 0x1p100f ? 0x1p-64f : 1.0f;
        finite = m < __builtin_inff();
        inverse = m > 0.0f && finite ? 127.0f * __builtin_amdgcn_rcpf(m * by) : 0.0f;
    }
};

// v / 127, rounded once: the error of the product with 1 / 127 taken back.
__device__ __forceinline__ float over_127(float v) {
    constexpr float kInverse = 1.0f / 127.0f;
    if (v < 0x1p-100f) return v / 127.0f;
    const float q = v * kInverse;
    return __builtin_fmaf(__builtin_fmaf(-q, 127.0f, v), kInverse, q);
}

// 127 t / m to the nearest whole number, ties to even, in eight codes' low bytes. The
// product with the reciprocal is off by less than 2^-15: where it comes so near to a tie
// that this could decide, 127 t is compared with the tie in 64 bits, in which both are
// exact (t has at most 22 bits, m as many).
__device__ __forceinline__ u32x2_t codes_of(const float* t, const RowCodes& r) {
    constexpr float kWhole = 12582912.0f;          // 1.5 * 2^23: adding it rounds to a whole number
    constexpr float kNear = 0.5f - 0x1p-15f;
    float v[8], w[8], most = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = t[e];
    if (r.by != 1.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= r.by;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = __builtin_fmaf(v[e], r.inverse, kWhole);
        most = __builtin_fmaxf(most, __builtin_fabsf(__builtin_fmaf(v[e], r.inverse, kWhole - w[e])));
    }
    if (most > kNear) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float c = w[e] - kWhole, off = __builtin_fmaf(v[e], r.inverse, -c);
            if (__builtin_fabsf(off) > kNear) {
                const float low = off > 0.0f ? c : c - 1.0f;        // the tie is low + 1/2
                const double d = 127.0 * (double)t[e] - ((double)low + 0.5) * (double)r.m;
                const bool odd = ((int)low & 1) != 0;
                w[e] = kWhole + (d > 0.0 || (d == 0.0 && odd) ? low + 1.0f : low);
            }
        }
    }
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        b[i] = __builtin_amdgcn_perm(bit_cast<uint32_t>(w[2 * i + 1]), bit_cast<uint32_t>(w[2 * i]), 0x0C0C0400u);
    u32x2_t code;
    code[0] = r.finite ? b[0] | b[1] << 16 : 0u;
    code[1] = r.finite ? b[2] | b[3] << 16 : 0u;
    return code;
}

// A chunk's codes to their places; the last chunk also clears what is behind the row's
// end, up to a multiple of 16.
template <bool SMALL>
__device__ __forceinline__ void write_codes(int8_t* row, int c, const RowChunks<SMALL>& k, u32x2_t code) {
    if (c > k.last) return;
    if (c == k.last) {
        uint64_t v = (uint64_t)code[1] << 32 | code[0];
        v >>= 8 * k.twice;                         // the chunk's own values first, zeros behind them
        code[0] = (uint32_t)v;
        code[1] = (uint32_t)(v >> 32);
        if ((c & 1) == 0) *reinterpret_cast<u32x2_t*>(row + 8 * (uint32_t)c + 8) = u32x2_t{0u, 0u};
    }
    *reinterpret_cast<u32x2_t*>(row + 8 * (uint32_t)c) = code;
}

constexpr int group_rows(int threads) { return threads < 64 ? 64 / threads : 1; }

// TH threads to a row, CH chunks each, a wave on several rows where they are short. The
// next row's loads are issued ahead of this row's sums. NORM: the sum's norm; else the
// codes of x.
template <int DT, int CH, int TH, bool NORM, bool SMALL, bool STREAMED>
__global__ __launch_bounds__(TH < 64 ? 64 : TH, 4) void rows8_kernel(const Rows8Args a) {
    constexpr int ROWS = group_rows(TH), kRowWaves = TH / 64;
    __shared__ float s_join[2][2][kRowWaves > 1 ? kRowWaves : 1];
    const int lane = threadIdx.x % TH, group = row_group<TH>();
    const RowChunks<SMALL> k(a.N);
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const float inv_n = 1.0f / ((float)a.N * a.scale);

    u32x4_t gamma[NORM ? CH : 1];
    if constexpr (NORM) {
#pragma unroll
        for (int t = 0; t < CH; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) gamma[t][e] = pack2<DT>(1.0f, 1.0f);
            if (a.gamma) gamma[t] = k.read(a.gamma, lane + TH * t);
        }
    }

    u32x4_t next[CH], next_r[NORM ? CH : 1];
    auto load = [&](int64_t i) {
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = i < a.M ? lane + TH * t : k.last + 1;
            next[t] = k.template read<STREAMED>(a.x + i * a.ldx, c);
            if constexpr (NORM) {
                if (a.residual) next_r[t] = k.template read<STREAMED>(a.residual + i * a.ldr, c);
            }
        }
    };
    int64_t i = (int64_t)blockIdx.x * ROWS + group;
    const int64_t rounds = (a.M - (int64_t)blockIdx.x * ROWS + step - 1) / step;   // the same for every row group
    load(i);
    for (int64_t round = 0; round < rounds; ++round, i += step) {
        u32x4_t v[CH];              // x, or h
        // x, or h gamma: kept for the output where the registers suffice, else formed again
        constexpr bool kKeep = !NORM || CH <= 3;
        float kept[kKeep ? CH : 1][8];
        auto scaled = [&](int t, float* x) {
            float g[8];
            asm volatile("" : "+v"(gamma[NORM ? t : 0]));      // widened anew for each row: half the registers
            widen<DT>(gamma[NORM ? t : 0], g);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= g[e];
        };
        float square = 0.0f, m = 0.0f;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            v[t] = next[t];
            float* const x = kept[kKeep ? t : 0];
            if constexpr (NORM) {
                if (a.residual) {
                    float r[8];
                    widen<DT>(next[t], x);
                    widen<DT>(next_r[t], r);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] += r[e];
                    v[t] = narrow<DT>(x);
                }
            }
            widen<DT>(v[t], x);
            if constexpr (NORM) {
                square += k.sum(lane + TH * t, [&](int e) { return x[e] * x[e]; });
                scaled(t, x);
            }
            if (!NORM || a.codes) m = __builtin_elementwise_maximum(m, top_of(x));
        }
        if (round + 1 < rounds) load(i + step);
        if constexpr (NORM) square = lanes_sum<(TH < 64 ? TH : 64)>(square * a.scale);
        m = lanes_max<TH>(m);
        if constexpr (kRowWaves > 1) {
            // (two sets of words, so that one barrier per row is enough)
            const int set = (int)(round & 1), w = threadIdx.x & 63;
            if (w == 0) {
                s_join[set][0][threadIdx.x >> 6] = square;
                s_join[set][1][threadIdx.x >> 6] = m;
            }
            __syncthreads();
            const bool there = w < kRowWaves;
            square = first_sum<kRowWaves>(there ? s_join[set][0][w] : 0.0f);
            m = first_max<kRowWaves>(there ? s_join[set][1][w] : 0.0f);
        }
        if (i >= a.M) continue;
        float rstd = 1.0f;
        if constexpr (NORM) rstd = rsqrt_of(square * inv_n + a.eps);
        const RowCodes codes(m);
        if (lane == 0) {
            if constexpr (NORM) {
                if (a.rstd) a.rstd[i] = rstd;
            }
            if (!NORM || a.codes) a.scales[i] = codes.finite ? over_127(m * rstd) : __builtin_nanf("");
        }
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = lane + TH * t;
            float* const x = kept[kKeep ? t : 0];
            if constexpr (!kKeep) {
                asm volatile("" : "+v"(v[t]));
                widen<DT>(v[t], x);
                if constexpr (NORM) scaled(t, x);
            }
            if constexpr (NORM) {
                if (a.h) k.write(a.h + i * a.ldh, c, v[t]);
                if (a.y) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = x[e] * rstd;
                    k.write(a.y + i * a.ldy, c, narrow<DT>(y));
                }
            }
            if (!NORM || a.codes) write_codes(a.codes + i * a.ldc, c, k, codes_of(x, codes));
        }
    }
}

// Rows of more values than a workgroup's registers hold: a workgroup per row, which it
// reads twice.
constexpr int kLongThreads = 1024;
template <int DT>
__global__ __launch_bounds__(kLongThreads) void quantize_long_kernel(const Rows8Args a) {
    __shared__ float s_max[kLongThreads / 64];
    const RowChunks<false> k(a.N);
    for (int64_t i = blockIdx.x; i < a.M; i += gridDim.x) {
        const uint16_t* row = a.x + i * a.ldx;
        float m = 0.0f;
        for (int c = threadIdx.x; c <= k.last; c += kLongThreads) {
            float x[8];
            widen<DT>(k.read(row, c), x);
            m = __builtin_elementwise_maximum(m, top_of(x));
        }
        m = lanes_max<64>(m);
        if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
        __syncthreads();
        m = first_max<16>((threadIdx.x & 63) < 16 ? s_max[threadIdx.x & 63] : 0.0f);
        const RowCodes codes(m);
        if (threadIdx.x == 0) a.scales[i] = codes.finite ? over_127(m) : __builtin_nanf("");
        for (int c = threadIdx.x; c <= k.last; c += kLongThreads) {
            float x[8];
            widen<DT>(k.read(row, c), x);
            write_codes(a.codes + i * a.ldc, c, k, codes_of(x, codes));
        }
        __syncthreads();
    }
}

// ---- backward ---------------------------------------------------------------

template <int CH>
struct GradPart {
    u32x4_t g[CH], h[CH], d[CH];
    float rstd;
};

// ROWS rows at a time, TH threads each; every thread keeps its columns' sums of
// dy h r over all of its rows, and the next row's loads are in flight.
template <int DT, int CH, int TH, int ROWS, bool SMALL, bool STREAMED>
__global__ __launch_bounds__(TH * ROWS) void norm_add_backward_kernel(const NormAddArgs a) {
    constexpr int kWaves = TH * ROWS / 64, kRowWaves = TH / 64;
    __shared__ float s_sum[2][kWaves];
    __shared__ float s_cols[ROWS > 1 ? ROWS / 2 : 1][ROWS > 1 ? 8 * CH : 1][ROWS > 1 ? TH : 1];
    const int lane = threadIdx.x % TH, group = row_group<TH>();
    const RowChunks<SMALL> k(a.N);
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const float inv_n = 1.0f / (float)a.N;

    u32x4_t gamma[CH];
    float dgamma[CH][8];
#pragma unroll
    for (int t = 0; t < CH; ++t) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dgamma[t][e] = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) gamma[t][e] = pack2<DT>(1.0f, 1.0f);
        if (a.gamma) gamma[t] = k.read(a.gamma, lane + TH * t);
    }
    // Chunks past the row's end, and rows past the last, read as zeros: they add nothing.
    auto load = [&](int64_t i, GradPart<CH>& p) {
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = i < a.M ? lane + TH * t : k.last + 1;
            p.g[t] = k.template read<STREAMED>(a.dy + i * a.lddy, c);
            p.h[t] = k.template read<STREAMED>(a.h + i * a.ldh, c);
            p.d[t] = u32x4_t{0u, 0u, 0u, 0u};
            if (a.dh && a.dx) p.d[t] = k.template read<STREAMED>(a.dh + i * a.lddh, c);
        }
        p.rstd = i < a.M ? a.rstd[i] : 0.0f;
    };
    int64_t i = (int64_t)blockIdx.x * ROWS + group;
    const int64_t rounds = (a.M - (int64_t)blockIdx.x * ROWS + step - 1) / step;   // the same for every row group
    GradPart<CH> next;
    load(i, next);
    for (int64_t n = 0; n < rounds; ++n, i += step) {
        const float rstd = next.rstd;
        float hv[CH][8], gv[CH][8], s = 0.0f;
        u32x4_t dv[CH];
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            float d[8], gamma_f[8];
            asm volatile("" : "+v"(gamma[t]));      // widened anew for each row: half the registers
            widen<DT>(gamma[t], gamma_f);
            widen<DT>(next.g[t], d);
            widen<DT>(next.h[t], hv[t]);
            dv[t] = next.d[t];
            asm volatile("" : "+v"(dv[t]));         // here before the barrier: dx may be dh
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dgamma[t][e] += (d[e] * rstd) * hv[t][e];
                gv[t][e] = d[e] * gamma_f[e];
            }
            s += k.sum(lane + TH * t, [&](int e) { return gv[t][e] * hv[t][e]; });
        }
        load(i + step, next);
        s = lanes_sum<(TH < 64 ? TH : 64)>(s);
        if constexpr (kRowWaves > 1) {
            // (two sets of words, so that one barrier per row is enough)
            const int set = (int)(n & 1), w = threadIdx.x & 63;
            if (w == 0) s_sum[set][threadIdx.x >> 6] = s;
            __syncthreads();
            s = first_sum<kRowWaves>(w < kRowWaves ? s_sum[set][group * kRowWaves + w] : 0.0f);
        }
        if (a.dx && i < a.M) {
            const float c2 = rstd * rstd * (rstd * s * inv_n);
#pragma unroll
            for (int t = 0; t < CH; ++t) {
                float d[8];
                widen<DT>(dv[t], d);
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] += rstd * gv[t][e] - hv[t][e] * c2;
                k.write(a.dx + i * a.lddx, lane + TH * t, narrow<DT>(d));
            }
        }
    }

    if (!a.partial) return;
    // the row groups' sums, the upper half of them added to the lower one until one is left
    if constexpr (ROWS > 1) {
#pragma unroll
        for (int half = ROWS / 2; half > 0; half >>= 1) {
            __syncthreads();
            if (group >= half && group < 2 * half) {
#pragma unroll
                for (int j = 0; j < 8 * CH; ++j) s_cols[group - half][j][lane] = dgamma[j / 8][j % 8];
            }
            __syncthreads();
            if (group < half) {
#pragma unroll
                for (int j = 0; j < 8 * CH; ++j) dgamma[j / 8][j % 8] += s_cols[group][j][lane];
            }
        }
    }
    if (group != 0) return;
    float* out = a.partial + (int64_t)blockIdx.x * 2 * norm_partial_cols(a.N);
#pragma unroll
    for (int t = 0; t < CH; ++t) {
        const int c = lane + TH * t;
        if (c < k.last || (c == k.last && k.twice == 0)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) out[8 * c + e] = dgamma[t][e];
        } else if (c == k.last) {
            // its own columns, and nothing behind the row's end
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= k.twice) out[k.column(c) + e] = dgamma[t][e];
        }
    }
}

// Rows of more than 16384 values: the rows' sums first, sum(g h) r^3 / N, then down the
// columns.
constexpr int kWideThreads = 256;
template <int DT>
__global__ __launch_bounds__(1024) void norm_add_wide_dots_kernel(const NormAddArgs a) {
    __shared__ float s_sum[2][16];
    const RowChunks<false> k(a.N);
    int set = 0;
    for (int64_t i = blockIdx.x; i < a.M; i += gridDim.x, set ^= 1) {
        float s = 0.0f;
        for (int c = threadIdx.x; c <= k.last; c += 1024) {
            float d[8], h[8], g[8];
            widen<DT>(k.read(a.dy + i * a.lddy, c), d);
            widen<DT>(k.read(a.h + i * a.ldh, c), h);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = 1.0f;
            if (a.gamma) widen<DT>(k.read(a.gamma, c), g);
            s += k.sum(c, [&](int e) { return (d[e] * g[e]) * h[e]; });
        }
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) s_sum[set][threadIdx.x >> 6] = s;
        __syncthreads();
        s = first_sum<16>((threadIdx.x & 63) < 16 ? s_sum[set][threadIdx.x & 63] : 0.0f);
        const float rstd = a.rstd[i];
        if (threadIdx.x == 0) a.dots[i] = rstd * rstd * (rstd * s * (1.0f / (float)a.N));
    }
}

// (A row's end is read and written in parts here: dx may be one of the inputs, and no
// barrier stands between a thread's reads and another one's writes.)
template <int DT>
__global__ __launch_bounds__(kWideThreads) void norm_add_wide_columns_kernel(const NormAddArgs a) {
    const int c = blockIdx.x * kWideThreads + threadIdx.x;
    const int64_t left = a.N - 8 * (int64_t)c, groups = gridDim.y;
    if (left <= 0) return;
    float gamma[8], dgamma[8] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) gamma[e] = 1.0f;
    if (a.gamma) widen<DT>(read_chunk<kCached>(a.gamma + 8 * c, left), gamma);
    constexpr int kAhead = 4;           // rows whose loads are in flight together
    for (int64_t i0 = blockIdx.y; i0 < a.M; i0 += kAhead * groups) {
        u32x4_t g[kAhead], h[kAhead], d[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t i = i0 + j * groups < a.M ? i0 + j * groups : i0;
            g[j] = read_chunk<kCached>(a.dy + i * a.lddy + 8 * c, left);
            h[j] = read_chunk<kCached>(a.h + i * a.ldh + 8 * c, left);
            d[j] = u32x4_t{0u, 0u, 0u, 0u};
            if (a.dh && a.dx) d[j] = read_chunk<kCached>(a.dh + i * a.lddh + 8 * c, left);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t i = i0 + j * groups;
            if (i >= a.M) break;
            const float rstd = a.rstd[i];
            float gf[8], hf[8], df[8];
            widen<DT>(g[j], gf);
            widen<DT>(h[j], hf);
            widen<DT>(d[j], df);
#pragma unroll
            for (int e = 0; e < 8; ++e) dgamma[e] += (gf[e] * rstd) * hf[e];
            if (a.dx) {
                const float c2 = a.dots[i];
#pragma unroll
                for (int e = 0; e < 8; ++e) df[e] += rstd * (gf[e] * gamma[e]) - hf[e] * c2;
                write_chunk(a.dx + i * a.lddx + 8 * c, narrow<DT>(df), left);
            }
        }
    }
    if (!a.partial) return;
    float* out = a.partial + (int64_t)blockIdx.y * 2 * norm_partial_cols(a.N) + 8 * c;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = dgamma[e];
}

template <int N>
using Int = std::integral_constant<int, N>;

// A kernel's threads per row and chunks per thread, as go(threads, chunks).
template <bool NORM, typename F>
hipError_t for_form(int64_t N, F go) {
    if (N <= 64) return go(Int<8>(), Int<1>());
    if (N <= 128) return go(Int<8>(), Int<2>());
    if (N <= 256) return go(Int<16>(), Int<2>());
    if (N <= 512) return go(Int<32>(), Int<2>());
    if (N <= 1024) return go(Int<64>(), Int<2>());
    if (N <= 2048) return go(Int<128>(), Int<2>());
    if (N <= 4096) return go(Int<256>(), Int<2>());
    if (N <= 6144) return go(Int<256>(), Int<3>());
    if (N <= 8192) return go(Int<512>(), Int<2>());
    if (N <= 12288) return go(Int<512>(), Int<3>());
    if (N <= 16384) return NORM ? go(Int<512>(), Int<4>()) : go(Int<1024>(), Int<2>());
    if (N <= 24576) return go(Int<1024>(), Int<3>());
    return go(Int<1024>(), Int<4>());
}

template <int CH, int TH, int MAX, int MIN, typename F>
hipError_t for_rows(int rows, F go) {
    if constexpr (MAX > MIN) {
        constexpr int kLess = MAX / 4 > MIN ? MAX / 4 : MIN;
        if (rows < MAX) return for_rows<CH, TH, kLess, MIN>(rows, go);
    }
    return go(Int<CH>(), Int<TH>(), Int<MAX>());
}
// As norm_backward_form has it, or fewer rows at a time (of which every workgroup then has
// some): half as many kernels.
template <typename F>
hipError_t for_backward(const NormForm& f, F go) {
    switch (f.threads) {
        case 8: return for_rows<1, 8, 128, 32>(f.rows, go);
        case 16: return for_rows<1, 16, 64, 16>(f.rows, go);
        case 32: return for_rows<1, 32, 32, 8>(f.rows, go);
        case 64: return for_rows<1, 64, 16, 1>(f.rows, go);
        case 128: return for_rows<1, 128, 8, 1>(f.rows, go);
        case 256: return for_rows<1, 256, 4, 1>(f.rows, go);
        case 512: return for_rows<1, 512, 2, 1>(f.rows, go);
        case 768: return for_rows<2, 768, 1, 1>(f.rows, go);
        default: return f.chunks == 1 ? for_rows<1, 1024, 1, 1>(f.rows, go) : for_rows<2, 1024, 1, 1>(f.rows, go);
    }
}

}  // namespace

// Whether a call's matrices are too large for the caches to keep any of them until they are
// read again; their loads then leave the caches to what is written (nontemporal). us, loads
// kept and not: norm_add and its backward pass 1217x2880 17.7 and 18.9, 8192x1024 27.6 and
// 31.1, 4096x4096 54.4 and 52.7, 16384x4096 188 and 180; quantize 16384x4096 41.7 and 36.5.
static bool streams(int64_t M, int64_t N) { return M * N > (int64_t)1 << 24; }

template <bool NORM>
static hipError_t launch_rows8(int dtype, const Rows8Args& a, hipStream_t s) {
    return for_form<NORM>(a.N, [&](auto th, auto ch) {
        constexpr int TH = decltype(th)::value, CH = decltype(ch)::value, kThreads = TH < 64 ? 64 : TH;
        // Waves over all compute units (256): the more of a row they have in flight each, the
        // fewer. (us: 8192x8192 bf16 to codes with 2048, 4096 and 8192 waves 66, 44, 41; its
        // norm and the backward pass 189, 193, 193; 4096x4096 to codes by the norm 29.3, 27.6,
        // 28.2.)
        const int64_t rows = group_rows(TH), groups = (a.M + rows - 1) / rows;
        const int64_t waves = !NORM ? 8192 : groups * kThreads / 64 >= 16 * 2048 ? 2048 : 4096;
        const uint32_t blocks = (uint32_t)std::min<int64_t>(groups, waves * 64 / kThreads);
        auto go = [&](auto small, auto streamed) {
            constexpr bool SMALL = decltype(small)::value, STREAMED = decltype(streamed)::value;
            return launch(dtype == FO_FP16 ? rows8_kernel<FO_FP16, CH, TH, NORM, SMALL, STREAMED>
                                           : rows8_kernel<FO_BF16, CH, TH, NORM, SMALL, STREAMED>, blocks, kThreads, s, a);
        };
        if constexpr (TH == 8 && CH == 1) {
            if (a.N < 8) return go(std::true_type(), std::false_type());
        }
        return streams(a.M, a.N) ? go(std::false_type(), std::true_type()) : go(std::false_type(), std::false_type());
    });
}

hipError_t launch_quantize(int dtype, const Rows8Args& a, hipStream_t s) {
    if (a.N > kMaxNormCols)
        return launch(dtype == FO_FP16 ? quantize_long_kernel<FO_FP16> : quantize_long_kernel<FO_BF16>,
                      (uint32_t)std::min<int64_t>(a.M, 4096), kLongThreads, s, a);
    return launch_rows8<false>(dtype, a, s);
}

hipError_t launch_norm_add_forward(int dtype, const Rows8Args& a, hipStream_t s) { return launch_rows8<true>(dtype, a, s); }

hipError_t launch_norm_add_backward(int dtype, const NormAddArgs& a, float* dgamma, hipStream_t s) {
    const NormForm f = norm_backward_form(a.M, a.N);
    hipError_t e = hipSuccess;
    int64_t blocks = a.M > 0 ? f.blocks : 0;
    if (a.M > 0 && norm_dots_bytes(a.M, a.N) > 0) {
        if (a.dx)
            e = launch(dtype == FO_FP16 ? norm_add_wide_dots_kernel<FO_FP16> : norm_add_wide_dots_kernel<FO_BF16>,
                       (uint32_t)std::min<int64_t>(a.M, 1024), 1024, s, a);
        const uint32_t slabs = (uint32_t)((a.N + 8 * kWideThreads - 1) / (8 * kWideThreads));
        if (e == hipSuccess)
            e = launch(dtype == FO_FP16 ? norm_add_wide_columns_kernel<FO_FP16> : norm_add_wide_columns_kernel<FO_BF16>,
                       dim3(slabs, (uint32_t)blocks), kWideThreads, s, a);
    } else if (a.M > 0) {
        e = for_backward(f, [&](auto ch, auto th, auto rows) {
            constexpr int CH = decltype(ch)::value, TH = decltype(th)::value, ROWS = decltype(rows)::value;
            blocks = std::min<int64_t>((a.M + ROWS - 1) / ROWS, f.blocks);      // (whose sums the workspace holds)
            auto go = [&](auto small, auto streamed) {
                constexpr bool SMALL = decltype(small)::value, STREAMED = decltype(streamed)::value;
                return launch(dtype == FO_FP16 ? norm_add_backward_kernel<FO_FP16, CH, TH, ROWS, SMALL, STREAMED>
                                               : norm_add_backward_kernel<FO_BF16, CH, TH, ROWS, SMALL, STREAMED>,
                              (uint32_t)blocks, TH * ROWS, s, a);
            };
            if constexpr (TH == 8) {
                if (a.N < 8) return go(std::true_type(), std::false_type());
            }
            if constexpr (TH * ROWS >= 768) {       // (as many rows at a time as there are threads for, then)
                if (streams(a.M, a.N)) return go(std::false_type(), std::true_type());
            }
            return go(std::false_type(), std::false_type());
        });
    }
    if (e == hipSuccess && dgamma) e = launch_norm_reduce(a.partial, (int)blocks, a.N, dgamma, nullptr, s);
    return e;
}

}  // namespace fo
