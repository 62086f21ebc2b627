// Layer norm and RMS norm, forward and backward.
//
//   mu = sum(x) / N (RMS norm: 0), r = 1 / sqrt(sum((x - mu)^2) / N + eps),
//   y = (x - mu) r gamma + beta;
//   with h = (x - mu) r and g = dy gamma:
//   dx = r (g - mean(g) - h mean(g h))   (RMS norm: without mean(g)),
//   dgamma = sum over rows of dy h, dbeta = sum over rows of dy.
//
// Both are bound by memory. A row is read once and held in registers between its
// statistics and its output: by a few lanes, a wave or a workgroup, as its length
// asks. All sums are in fp32; the variance is the mean square of the differences from
// the mean, so that a large mean costs it no digits.
//
// Backward: a workgroup takes rows blocks apart and keeps its columns' sums of
// dy h and dy in registers over all of them; the workgroups' sums are added in
// a second launch, in one order, so that equal calls give equal bits. 16384x4096
// bf16 from an int8 checkpoint 57 us (6.0 TB/s of the 6.25 that a copy reaches), with
// 5 us for the second launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "rowops.h"
#include "rows.h"

namespace fo {
namespace {

// Which of the workgroup's rows a thread works on. A wave that lies within one row
// has its number in a scalar register, and the row's addresses too.
template <int TH>
__device__ __forceinline__ int row_group() {
    const int group = threadIdx.x / TH;
    return TH < 64 ? group : __builtin_amdgcn_readfirstlane(group);
}

// ROWS rows at a time, TH threads each. Every thread keeps its columns of gamma and
// beta, and the next row's loads are issued ahead of this row's sums. Where a row
// has several waves each takes the mean of its own values and the sum of their
// squared differences from it, and one meeting joins them:
//   mu = mu_0 + sum over waves of n_w (mu_w - mu_0) / N,
//   sum of (x - mu)^2 = sum over waves of (their sum + n_w (mu_w - mu)^2).
// (The sum of the waves' n_w mu_w itself is rounded past 24 bits: rows of one fp16 value and more
// than 8192 columns then had a mean one step off, 0.89 in y for values of 2^14 and an eps of 1e-6.)
// Rows of up to half a wave share waves.
template <int DT, int CH, int TH, int ROWS>
__global__ __launch_bounds__(TH * ROWS) void norm_forward_kernel(const NormArgs a) {
    constexpr int kRowWaves = TH / 64;              // 0: several rows in a wave
    __shared__ float s_sum[2][2][TH * ROWS / 64];
    const int lane = threadIdx.x % TH, group = row_group<TH>();
    const int full = (int)(a.N >> 3), tail = (int)(a.N & 7);
    // The values behind the row's last whole chunk, fewer than eight: one to a lane, in
    // the wave that packs them.
    const int end_lane = TH <= 64 ? lane : lane - full % TH / 64 * 64;
    const bool has_tail = end_lane >= 0 && end_lane < tail;
    const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK, step = (int64_t)gridDim.x * ROWS;
    // A lane's sum is scaled by the power of two that makes N at most 1, so that the
    // row's sums (of squares: up to 2^120 on average) stay in fp32's range.
    const float scale = a.scale, n = (float)a.N * scale, inv_n = 1.0f / n;
    // A sum's quotient by a count, the error of the product with its reciprocal taken back:
    // a wave's sum of one 16-bit value, up to 2055 times, is exact, and so is that value as
    // its mean.
    auto quotient = [](float sum, float count, float inverse) {
        const float q = sum * inverse;
        return __builtin_fmaf(__builtin_fmaf(-q, count, sum), inverse, q);
    };

    u32x4_t gamma[CH], beta[CH];
    float gamma_t = 1.0f, beta_t = 0.0f, count = has_tail ? 1.0f : 0.0f;
#pragma unroll
    for (int t = 0; t < CH; ++t) {
        const int c = lane + TH * t;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            gamma[t][e] = pack2<DT>(1.0f, 1.0f);
            beta[t][e] = 0u;
        }
        if (c < full) {
            if (a.gamma) gamma[t] = load8(a.gamma + 8 * c);
            if (a.beta) beta[t] = load8(a.beta + 8 * c);
            count += 8.0f;
        }
    }
    if (a.gamma && has_tail) gamma_t = to_f32<DT>(a.gamma[8 * full + end_lane]);
    if (a.beta && has_tail) beta_t = to_f32<DT>(a.beta[8 * full + end_lane]);
    count = wave_sum(count * scale);                // of this wave, scaled like the sums (kRowWaves > 1)
    const float inv_count = count > 0.0f ? 1.0f / count : 0.0f;
    float wave_count = 0.0f;                        // lane w: of the row's wave w
    if constexpr (kRowWaves > 1) {
        if ((threadIdx.x & 63) == 0) s_sum[0][0][threadIdx.x >> 6] = count;
        __syncthreads();
        if ((threadIdx.x & 63) < kRowWaves) wave_count = s_sum[0][0][group * kRowWaves + (threadIdx.x & 63)];
        __syncthreads();
    }

    auto load = [&](int64_t i, u32x4_t* v, uint32_t& vt) {
        const uint16_t* row = a.x + i * a.ldx;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = lane + TH * t;
            v[t] = u32x4_t{0u, 0u, 0u, 0u};
            if (i < a.M && c < full) v[t] = load8(row + 8 * c);
        }
        vt = i < a.M && has_tail ? row[8 * full + end_lane] : 0u;
    };

    int64_t i = (int64_t)blockIdx.x * ROWS + group;
    const int64_t rounds = (a.M - (int64_t)blockIdx.x * ROWS + step - 1) / step;   // the same for every row group
    u32x4_t next[CH];
    uint32_t next_t;
    load(i, next, next_t);
    for (int64_t round = 0; round < rounds; ++round, i += step) {
        float x[CH][8];
#pragma unroll
        for (int t = 0; t < CH; ++t) widen<DT>(next[t], x[t]);
        const float xt = to_f32<DT>(next_t);
        if (round + 1 < rounds) load(i + step, next, next_t);

        if (a.packed && i < a.M) {
            uint8_t* packed = a.packed + i * blocks * FO_PACK_BLOCK;
            uint8_t* scales = a.scales + i * blocks;
            // the values behind the last whole chunk, to the thread that packs them
            float end[8] = {};
            if (tail) {
                const int from = TH < 64 ? (threadIdx.x & 63) - lane : 0;
#pragma unroll
                for (int e = 0; e < 7; ++e) {
                    const float v = __shfl(xt, from + e, 64);
                    end[e] = e < tail ? v : 0.0f;
                }
            }
#pragma unroll
            for (int t = 0; t < CH; ++t) {
                const int c = lane + TH * t;
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = x[t][e];
                if (tail && c == full) {
#pragma unroll
                    for (int e = 0; e < 7; ++e) f[e] = end[e];
                }
                if (c < 4 * (int)blocks) {
                    if (a.format == FO_PACK_INT8) pack_chunk<DT, FO_PACK_INT8>(f, c, packed, scales);
                    else pack_chunk<DT, FO_PACK_E4M3>(f, c, packed, scales);
                }
            }
        }

        float mean = 0.0f, square = 0.0f;
        if (a.layer) {          // (an RMS norm: differences from zero)
            float sum = xt;
#pragma unroll
            for (int t = 0; t < CH; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += x[t][e];
            sum = lanes_sum<(TH < 64 ? TH : 64)>(sum * scale);
            mean = kRowWaves > 1 ? quotient(sum, count, inv_count) : quotient(sum, n, inv_n);
        }
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            float q = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) q += (x[t][e] - mean) * (x[t][e] - mean);
            if (lane + TH * t < full) square += q;
        }
        if (has_tail) square += (xt - mean) * (xt - mean);
        square = lanes_sum<(TH < 64 ? TH : 64)>(square * scale);
        if constexpr (kRowWaves > 1) {
            // (two sets of words, so that one barrier per row is enough)
            const int set = (int)(round & 1), wave = threadIdx.x >> 6, w = threadIdx.x & 63;
            if (w == 0) {
                s_sum[set][0][wave] = mean;
                s_sum[set][1][wave] = square;
            }
            __syncthreads();
            const bool there = w < kRowWaves;
            const float mw = there ? s_sum[set][0][group * kRowWaves + w] : 0.0f;
            const float qw = there ? s_sum[set][1][group * kRowWaves + w] : 0.0f;
            const float m0 = bit_cast<float>(__builtin_amdgcn_readfirstlane(bit_cast<int>(mw)));
            mean = a.layer ? __builtin_fmaf(first_sum<kRowWaves>(wave_count * (mw - m0)), inv_n, m0) : 0.0f;
            square = first_sum<kRowWaves>(qw + wave_count * ((mw - mean) * (mw - mean)));
        }
        const float rstd = rsqrt_of(square * inv_n + a.eps);
        if (i >= a.M) continue;
        if (lane == 0) {
            if (a.mean) a.mean[i] = mean;
            if (a.rstd) a.rstd[i] = rstd;
        }
        uint16_t* out = a.y + i * a.ldy;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = lane + TH * t;
            float g[8], b[8];
            asm volatile("" : "+v"(gamma[t]), "+v"(beta[t]));      // widened anew for each row: half the registers
            widen<DT>(gamma[t], g);
            widen<DT>(beta[t], b);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = (x[t][e] - mean) * rstd * g[e] + b[e];
            if (c < full) stream8(out + 8 * c, narrow<DT>(g));
        }
        if (has_tail) out[8 * full + end_lane] = (uint16_t)from_f32<DT>((xt - mean) * rstd * gamma_t + beta_t);
    }
}

// The part of a row that one thread reads: CH chunks of dy and of x (or of x's
// checkpoint) and, from the first lanes, a value behind the last whole chunk.
template <int SRC, int CH>
struct RowPart {
    u32x4_t g[CH];
    u32x4_t x[SRC ? 1 : CH];
    u32x2_t code[SRC ? CH : 1];
    uint32_t scale[SRC ? CH : 1];
    uint32_t gt, xt, st;
    float mean, rstd;
};

// SRC: where x comes from: 0 the input itself, 1 + format a checkpoint of it.
// ROWS rows at a time, TH threads each. Every thread keeps its columns of gamma
// and of the two sums over rows; with the next AHEAD rows' loads issued ahead of this
// row's sums, one workgroup of 16 waves per compute unit keeps memory busy, and
// there are few workgroups' sums to add.
template <int DT, int SRC, int CH, int TH, int ROWS, int AHEAD>
__global__ __launch_bounds__(TH * ROWS) void norm_backward_kernel(const NormArgs a) {
    constexpr int kWaves = TH * ROWS / 64, kRowWaves = TH / 64;     // (0: several rows in a wave)
    __shared__ float s_sum[2][2][kWaves];
    __shared__ float s_cols[ROWS > 1 ? ROWS / 2 : 1][ROWS > 1 ? 8 * CH + 1 : 1][ROWS > 1 ? TH : 1];
    const int lane = threadIdx.x % TH, group = row_group<TH>();
    const int full = (int)(a.N >> 3), tail = (int)(a.N & 7);
    const float inv_n = 1.0f / (float)a.N;
    const bool has_tail = lane < tail;
    const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK, step = (int64_t)gridDim.x * ROWS;

    u32x4_t gamma[CH];
    float gamma_t = 1.0f;
    float dgamma[CH][8], dbeta[CH][8], dgamma_t = 0.0f, dbeta_t = 0.0f;
#pragma unroll
    for (int t = 0; t < CH; ++t) {
        const int c = lane + TH * t;
#pragma unroll
        for (int e = 0; e < 8; ++e) dgamma[t][e] = dbeta[t][e] = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) gamma[t][e] = pack2<DT>(1.0f, 1.0f);
        if (a.gamma && c < full) gamma[t] = load8(a.gamma + 8 * c);
    }
    if (a.gamma && has_tail) gamma_t = to_f32<DT>(a.gamma[8 * full + lane]);

    // Chunks past the row's end, and rows past the last, read as zeros: they add nothing.
    auto load = [&](int64_t i, RowPart<SRC, CH>& p) {
        const bool row = i < a.M;
        const uint16_t* grow = a.dy + i * a.ldy;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = lane + TH * t;
            p.g[t] = u32x4_t{0u, 0u, 0u, 0u};
            if constexpr (SRC == 0) {
                p.x[t] = p.g[t];
            } else {
                p.code[t] = u32x2_t{0u, 0u};
                p.scale[t] = 0u;
            }
            if (row && c < full) {
                p.g[t] = load8(grow + 8 * c);
                if constexpr (SRC == 0) {
                    p.x[t] = load8(a.x + i * a.ldx + 8 * c);
                } else {
                    p.code[t] = *reinterpret_cast<const u32x2_t*>(a.packed + i * blocks * FO_PACK_BLOCK + 8 * c);
                    p.scale[t] = a.scales[i * blocks + (c >> 2)];
                }
            }
        }
        p.gt = p.xt = p.st = 0u;
        if (row && has_tail) {
            const int c = 8 * full + lane;
            p.gt = grow[c];
            if constexpr (SRC == 0) {
                p.xt = a.x[i * a.ldx + c];
            } else {
                p.xt = a.packed[i * blocks * FO_PACK_BLOCK + c];
                p.st = a.scales[i * blocks + c / FO_PACK_BLOCK];
            }
        }
        p.mean = row && a.layer ? a.mean[i] : 0.0f;
        p.rstd = row ? a.rstd[i] : 0.0f;
    };

    int64_t i = (int64_t)blockIdx.x * ROWS + group;
    const int64_t rounds = (a.M - (int64_t)blockIdx.x * ROWS + step - 1) / step;   // the same for every row group
    RowPart<SRC, CH> ahead[AHEAD];
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) load(i + d * step, ahead[d]);
    // one round: the row i whose loads `next` holds, which then takes those of row i + AHEAD * step
    auto round = [&](int64_t n, RowPart<SRC, CH>& next) {
        // With t = x - mean: h = t rstd, so that
        //   dgamma += (dy rstd) t,  sum(g h) = rstd sum(g t),
        //   dx = rstd g - rstd mean(g) - t rstd^2 mean(g h).
        const float mean = next.mean, rstd = next.rstd;
        float tv[CH][8], gv[CH][8], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            float d[8], gamma_f[8];
            asm volatile("" : "+v"(gamma[t]));      // widened anew for each row: half the registers
            widen<DT>(gamma[t], gamma_f);
            widen<DT>(next.g[t], d);
            if constexpr (SRC == 0) widen<DT>(next.x[t], tv[t]);
            else decode8<SRC - 1>(next.code[t], scale_of(next.scale[t]), tv[t]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                tv[t][e] -= mean;
                dgamma[t][e] += (d[e] * rstd) * tv[t][e];
                dbeta[t][e] += d[e];
                gv[t][e] = d[e] * gamma_f[e];
                s1 += gv[t][e];
                s2 += gv[t][e] * tv[t][e];
            }
        }
        float tt = 0.0f, gt = 0.0f;
        if (tail) {
            float d = to_f32<DT>(next.gt);
            if constexpr (SRC == 0) tt = to_f32<DT>(next.xt) - mean;
            else tt = decode1<SRC - 1>(next.xt, scale_of(next.st)) - mean;
            dgamma_t += (d * rstd) * tt;
            dbeta_t += d;
            gt = d * gamma_t;
            s1 += gt;
            s2 += gt * tt;
        }
        load(i + AHEAD * step, next);
        if constexpr (TH < 64) {
            s1 = lanes_sum<TH>(s1);
            s2 = lanes_sum<TH>(s2);
        } else {
            wave_sums(s1, s2);
        }
        if constexpr (kRowWaves > 1) {
            // (two sets of words, so that one barrier per row is enough)
            const int set = (int)(n & 1), wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) {
                s_sum[set][0][wave] = s1;
                s_sum[set][1][wave] = s2;
            }
            __syncthreads();
            const int w = threadIdx.x & 63;
            s1 = first_sum<kRowWaves>(w < kRowWaves ? s_sum[set][0][group * kRowWaves + w] : 0.0f);
            s2 = first_sum<kRowWaves>(w < kRowWaves ? s_sum[set][1][group * kRowWaves + w] : 0.0f);
        }
        if (a.dx && i < a.M) {
            const float c1 = a.layer ? rstd * (s1 * inv_n) : 0.0f;
            const float c2 = rstd * rstd * (rstd * s2 * inv_n);
            uint16_t* out = a.dx + i * a.lddx;
#pragma unroll
            for (int t = 0; t < CH; ++t) {
                const int c = lane + TH * t;
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = rstd * gv[t][e] - c1 - tv[t][e] * c2;
                if (c < full) stream8(out + 8 * c, narrow<DT>(d));
            }
            if (has_tail) out[8 * full + lane] = (uint16_t)from_f32<DT>(rstd * gt - c1 - tt * c2);
        }
        i += step;
    };
    for (int64_t n = 0; n < rounds; n += AHEAD) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d)
            if (n + d < rounds) round(n + d, ahead[d]);
    }
    if (!a.partial) return;
    // The row groups' sums, added in halves: group g takes group g + h's.
    float* partial = a.partial + (int64_t)blockIdx.x * 2 * norm_partial_cols(a.N);
    auto add_up = [&](float (&cols)[CH][8], float& one, float* out) {
        if constexpr (ROWS > 1) {
#pragma unroll
            for (int h = ROWS / 2; h > 0; h >>= 1) {
                __syncthreads();
                if (group >= h && group < 2 * h) {
#pragma unroll
                    for (int t = 0; t < CH; ++t)
#pragma unroll
                        for (int e = 0; e < 8; ++e) s_cols[group - h][8 * t + e][lane] = cols[t][e];
                    s_cols[group - h][8 * CH][lane] = one;
                }
                __syncthreads();
                if (group < h) {
#pragma unroll
                    for (int t = 0; t < CH; ++t)
#pragma unroll
                        for (int e = 0; e < 8; ++e) cols[t][e] += s_cols[group][8 * t + e][lane];
                    one += s_cols[group][8 * CH][lane];
                }
            }
        }
        if (group == 0) {
#pragma unroll
            for (int t = 0; t < CH; ++t) {
                const int c = lane + TH * t;
                if (c < full) {
                    f32x4_t lo, hi;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        lo[e] = cols[t][e];
                        hi[e] = cols[t][e + 4];
                    }
                    reinterpret_cast<f32x4_t*>(out)[2 * c] = lo;
                    reinterpret_cast<f32x4_t*>(out)[2 * c + 1] = hi;
                }
            }
            if (has_tail) out[8 * full + lane] = one;
        }
    };
    add_up(dgamma, dgamma_t, partial);
    if (a.with_beta) add_up(dbeta, dbeta_t, partial + norm_partial_cols(a.N));
}

// Rows of more than kHeldCols columns: the registers of sixteen waves cannot hold a row and
// its columns' sums (four chunks per thread spilled: 0.7 TB/s; a row kept in LDS was not
// tried). Two launches instead, which read dy and x twice: a workgroup per row for the row's
// two sums, then 256 threads per 2048 columns (a chunk each, kept sums as above) that go
// down every kWideGroups-th row. bf16, from x and from int8: 1024x32768 74 and 71 us with
// the last launch (2.7 and 2.4 TB/s of what the gradients need), 8192x32768 505 and 466.
constexpr int64_t kHeldCols = 16384;
constexpr int kWideThreads = 256, kWideGroups = 64;

// Chunk c of row i as it is read, and what it stands for: dy and x - mean.
template <int SRC>
struct WideChunk {
    u32x4_t g, x;
    u32x2_t code;
    uint32_t scale;
};
template <int SRC>
__device__ __forceinline__ WideChunk<SRC> wide_chunk(const NormArgs& a, int64_t i, int c) {
    const int64_t left = a.N - 8 * (int64_t)c;
    WideChunk<SRC> p;
    p.g = read_chunk<kCached>(a.dy + i * a.ldy + 8 * c, left);
    if constexpr (SRC == 0) {
        p.x = read_chunk<kCached>(a.x + i * a.ldx + 8 * c, left);
    } else {
        const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK;
        p.code = *reinterpret_cast<const u32x2_t*>(a.packed + i * blocks * FO_PACK_BLOCK + 8 * c);
        p.scale = a.scales[i * blocks + (c >> 2)];
    }
    return p;
}
template <int DT, int SRC>
__device__ __forceinline__ void wide_values(const WideChunk<SRC>& p, float mean, float* d, float* t) {
    widen<DT>(p.g, d);
    if constexpr (SRC == 0) widen<DT>(p.x, t);
    else decode8<SRC - 1>(p.code, scale_of(p.scale), t);
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] -= mean;
}

// dots[2 i] = rstd mean(g), dots[2 i + 1] = rstd^2 mean(g h) of row i.
template <int DT, int SRC>
__global__ __launch_bounds__(1024) void norm_wide_dots_kernel(const NormArgs a) {
    __shared__ float s_sum[2][2][16];
    const int chunks = (int)((a.N + 7) >> 3), wave = threadIdx.x >> 6, w = threadIdx.x & 63;
    int set = 0;
    for (int64_t i = blockIdx.x; i < a.M; i += gridDim.x, set ^= 1) {
        const float mean = a.layer ? a.mean[i] : 0.0f, rstd = a.rstd[i];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll 4
        for (int c = threadIdx.x; c < chunks; c += 1024) {
            float d[8], t[8], g[8];
            wide_values<DT, SRC>(wide_chunk<SRC>(a, i, c), mean, d, t);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = 1.0f;
            if (a.gamma) widen<DT>(read_chunk<kCached>(a.gamma + 8 * c, a.N - 8 * (int64_t)c), g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s1 += d[e] * g[e];
                s2 += (d[e] * g[e]) * t[e];
            }
        }
        wave_sums(s1, s2);
        if (w == 0) {
            s_sum[set][0][wave] = s1;
            s_sum[set][1][wave] = s2;
        }
        __syncthreads();
        s1 = first_sum<16>(w < 16 ? s_sum[set][0][w] : 0.0f);
        s2 = first_sum<16>(w < 16 ? s_sum[set][1][w] : 0.0f);
        if (threadIdx.x == 0) {
            const float inv_n = 1.0f / (float)a.N;
            a.dots[2 * i] = a.layer ? rstd * (s1 * inv_n) : 0.0f;
            a.dots[2 * i + 1] = rstd * rstd * (rstd * s2 * inv_n);
        }
    }
}

template <int DT, int SRC>
__global__ __launch_bounds__(kWideThreads) void norm_wide_columns_kernel(const NormArgs a) {
    const int c = blockIdx.x * kWideThreads + threadIdx.x;
    const int64_t left = a.N - 8 * (int64_t)c;
    if (left <= 0) return;
    float gamma[8], dgamma[8] = {}, dbeta[8] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) gamma[e] = 1.0f;
    if (a.gamma) widen<DT>(read_chunk<kCached>(a.gamma + 8 * c, left), gamma);
    constexpr int kAhead = 4;           // rows whose loads are in flight together
    for (int64_t i0 = blockIdx.y; i0 < a.M; i0 += kAhead * kWideGroups) {
        WideChunk<SRC> p[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t i = i0 + j * kWideGroups;
            p[j] = wide_chunk<SRC>(a, i < a.M ? i : i0, c);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t i = i0 + j * kWideGroups;
            if (i >= a.M) break;
            const float mean = a.layer ? a.mean[i] : 0.0f, rstd = a.rstd[i];
            float d[8], t[8];
            wide_values<DT, SRC>(p[j], mean, d, t);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dgamma[e] += (d[e] * rstd) * t[e];
                dbeta[e] += d[e];
            }
            if (a.dx) {
                const float c1 = a.dots[2 * i], c2 = a.dots[2 * i + 1];
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = rstd * (d[e] * gamma[e]) - c1 - t[e] * c2;
                write_chunk(a.dx + i * a.lddx + 8 * c, narrow<DT>(d), left);
            }
        }
    }
    if (!a.partial) return;
    float* out = a.partial + (int64_t)blockIdx.y * 2 * norm_partial_cols(a.N) + 8 * c;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        out[e] = dgamma[e];
        if (a.with_beta) out[norm_partial_cols(a.N) + e] = dbeta[e];
    }
}

// dgamma and dbeta: the sums of `count` workgroups' sums (2 * cols each), 32 columns
// per workgroup: 8 threads of four columns, 32 rows at a time.
constexpr int kReduceThreads = 256, kReduceCols = 32;
__global__ __launch_bounds__(kReduceThreads) void norm_reduce_kernel(const float* partial, int count, int64_t N,
                                                                      float* dgamma, float* dbeta) {
    constexpr int kRows = kReduceThreads / (kReduceCols / 4);
    __shared__ f32x4_t s[kRows / 2][kReduceCols / 4];
    const int quad = threadIdx.x % (kReduceCols / 4), part = threadIdx.x / (kReduceCols / 4);
    const int64_t cols = norm_partial_cols(N), per = (cols + kReduceCols - 1) / kReduceCols;
    const bool beta = !dgamma || blockIdx.x >= per;
    const int64_t c = (int64_t)(blockIdx.x % per) * kReduceCols + 4 * quad;
    const float* from = partial + (beta ? cols : 0) + c;
    f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < cols) {
#pragma unroll 8
        for (int g = part; g < count; g += kRows) sum += *reinterpret_cast<const f32x4_t*>(from + (int64_t)g * 2 * cols);
    }
#pragma unroll
    for (int h = kRows / 2; h > 0; h >>= 1) {
        if (part >= h && part < 2 * h) s[part - h][quad] = sum;
        __syncthreads();
        if (part < h) sum += s[part][quad];
        __syncthreads();
    }
    float* out = beta ? dbeta : dgamma;
    if (part == 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < N) out[c + e] = sum[e];
    }
}

template <int N>
using Int = std::integral_constant<int, N>;

// A form's constants, as go(chunks, threads, rows): rows of MAX, MAX / STEP, .. MIN.
template <int CH, int TH, int MAX, int MIN, int STEP, typename F>
hipError_t for_rows(const NormForm& f, F go) {
    if constexpr (MAX > MIN) {
        if (f.rows < MAX) return for_rows<CH, TH, MAX / STEP, MIN, STEP>(f, go);
    }
    return go(Int<CH>(), Int<TH>(), Int<MAX>());
}
template <typename F>
hipError_t for_forward(const NormForm& f, F go) {
    switch (f.threads) {
        case 8: return for_rows<2, 8, 64, 16, 4>(f, go);
        case 16: return for_rows<2, 16, 32, 8, 4>(f, go);
        case 32: return for_rows<2, 32, 16, 4, 4>(f, go);
        case 64: return for_rows<2, 64, 8, 1, 2>(f, go);
        case 128: return for_rows<2, 128, 4, 1, 2>(f, go);
        case 256: return for_rows<2, 256, 2, 1, 2>(f, go);
        case 512: return f.chunks == 2 ? for_rows<2, 512, 1, 1, 2>(f, go) : for_rows<3, 512, 1, 1, 2>(f, go);
        default: return f.chunks == 2 ? for_rows<2, 1024, 1, 1, 2>(f, go) : for_rows<4, 1024, 1, 1, 2>(f, go);
    }
}
template <typename F>
hipError_t for_backward(const NormForm& f, F go) {
    switch (f.threads) {
        case 8: return for_rows<1, 8, 128, 32, 4>(f, go);
        case 16: return for_rows<1, 16, 64, 16, 4>(f, go);
        case 32: return for_rows<1, 32, 32, 8, 4>(f, go);
        case 64: return for_rows<1, 64, 16, 1, 2>(f, go);
        case 128: return for_rows<1, 128, 8, 1, 2>(f, go);
        case 256: return for_rows<1, 256, 4, 1, 2>(f, go);
        case 512: return for_rows<1, 512, 2, 1, 2>(f, go);
        case 768: return for_rows<2, 768, 1, 1, 2>(f, go);
        default:
            return f.chunks == 1 ? for_rows<1, 1024, 1, 1, 2>(f, go) : for_rows<2, 1024, 1, 1, 2>(f, go);
    }
}

// As many rows at a time, in a workgroup of up to `threads`, as leave every one of
// `units` workgroups some; where rows share waves, all that fit or a quarter.
void set_rows(NormForm& f, int64_t M, int threads, int64_t units) {
    const int most = std::max(1, threads / f.threads);
    const int least = f.threads < 64 ? most / 4 : 1, step = f.threads < 64 ? 4 : 2;
    f.rows = most;
    while (f.rows > least && f.rows * units > M) f.rows /= step;
    f.blocks = (uint32_t)std::min<int64_t>((M + f.rows - 1) / f.rows, units);
}

}  // namespace

// Forward: two workgroups of eight waves per compute unit (8192x8192 fp16 49 us,
// 16384x4096 bf16 with a checkpoint 55; three, which fit, 53 and 57; one of 16 waves, on
// more rows, 66 for the second; registers held down to two of 16 waves 69 and 83; a
// workgroup per row and nothing ahead 60 and 61). Up to 12288 columns eight waves
// take a row in three chunks, two workgroups per compute unit for fewer than 4096 rows
// and one from there on (bf16, two against one, us: 1280x12288 10.9 and 12.0, with a
// checkpoint 16.5 and 18.7; 4096x12288 37.0 and 36.8, 44.9 and 45.0; 16384x12288 149 and
// 144, 178 and 162; 16 waves and two chunks 13.1, 18.6, 40.4, 46.3, 145 and 168). Past that a row has 16 waves and they fit once
// (eight waves of four chunks: 16384x13000 with a checkpoint 190, 16 waves 181). Past 16384
// columns, at four chunks a thread, 7 of the 128 registers go to scratch (24 bytes a
// thread): bf16 8192x32768 209 us (5.1 TB/s), with a checkpoint 231 (5.9); 1024x32768 28.6
// (4.7). Classes end at powers of two: a row just past one leaves half of the lanes
// idle (33.5 million values: 4096 columns 24.9 us, 4160 30.9; 2048 25.8, 2112 34.0).
NormForm norm_forward_form(int64_t M, int64_t N) {
    NormForm f{};
    f.threads = N <= 128 ? 8 : N <= 256 ? 16 : N <= 512 ? 32 : N <= 1024 ? 64 : N <= 2048 ? 128 : N <= 4096 ? 256 : N <= 12288 ? 512 : 1024;
    f.chunks = N <= 8192 ? 2 : N <= 12288 ? 3 : N <= 16384 ? 2 : 4;
    set_rows(f, M, 512, N <= 8192 || (N <= 12288 && M < 4096) ? 512 : 256);
    return f;
}

// Backward: one workgroup of 16 waves per compute unit. One chunk of a row per thread
// while 16 waves take a row so: its registers leave room for the loads of three rows
// ahead (16384x4096 bf16 from an int8 checkpoint 57 us, one row ahead 63, four 58; two
// chunks and one row ahead 66, two rows ahead do not fit and take 140). 8193 to 12288 columns
// have two chunks a thread and two rows ahead, 12289 to 16384 one row ahead on 16 waves, whose
// 128 registers do not suffice: 3 go to scratch from x (16 bytes a thread), 9 from a
// checkpoint (40 bytes). bf16, from x and from int8, the second launch not counted:
// 8192x16384 154 us (5.2 TB/s) and 162 (4.2), 16384x13000 237 (5.4) and 256 (4.2), 4000x14336 63
// (5.5) and 74 (3.9). Rows just past a class as in the forward pass: 4096 columns 34.2 us,
// 4160 41.1; 2048 34.9, 2112 46.3.
NormForm norm_backward_form(int64_t M, int64_t N) {
    NormForm f{};
    f.threads = N <= 64 ? 8 : N <= 128 ? 16 : N <= 256 ? 32 : N <= 512 ? 64 : N <= 1024 ? 128 : N <= 2048 ? 256
              : N <= 4096 ? 512 : N <= 8192 ? 1024 : N <= 12288 ? 768 : 1024;
    f.chunks = N <= 8192 ? 1 : 2;
    set_rows(f, M, 1024, 256);
    if (N > kHeldCols) f.blocks = (uint32_t)std::min<int64_t>(M, kWideGroups);       // rows of partial sums
    return f;
}
int64_t norm_dots_bytes(int64_t M, int64_t N) { return N > kHeldCols ? 8 * M : 0; }

hipError_t launch_norm_forward(int dtype, const NormArgs& a, hipStream_t s) {
    const NormForm f = norm_forward_form(a.M, a.N);
    return for_forward(f, [&](auto ch, auto th, auto rows) {
        constexpr int CH = decltype(ch)::value, TH = decltype(th)::value, ROWS = decltype(rows)::value;
        return launch(dtype == FO_FP16 ? norm_forward_kernel<FO_FP16, CH, TH, ROWS>
                                       : norm_forward_kernel<FO_BF16, CH, TH, ROWS>,
                      f.blocks, TH * ROWS, s, a);
    });
}

hipError_t launch_norm_backward(int dtype, const NormArgs& a, float* dgamma, float* dbeta, hipStream_t s) {
    const NormForm f = norm_backward_form(a.M, a.N);
    hipError_t e = hipSuccess;
    if (a.M > 0 && a.N > kHeldCols) {
        auto from = [&](auto dt, auto src) {
            constexpr int DT = decltype(dt)::value, SRC = decltype(src)::value;
            if (a.dx) e = launch(norm_wide_dots_kernel<DT, SRC>, (uint32_t)std::min<int64_t>(a.M, 1024), 1024, s, a);
            const uint32_t slabs = (uint32_t)((a.N + 8 * kWideThreads - 1) / (8 * kWideThreads));
            return e == hipSuccess ? launch(norm_wide_columns_kernel<DT, SRC>, dim3(slabs, f.blocks), kWideThreads, s, a) : e;
        };
        auto any = [&](auto dt) {
            return !a.packed                     ? from(dt, Int<0>())
                   : a.format == FO_PACK_INT8 ? from(dt, Int<1 + FO_PACK_INT8>()) : from(dt, Int<1 + FO_PACK_E4M3>());
        };
        e = dtype == FO_FP16 ? any(Int<FO_FP16>()) : any(Int<FO_BF16>());
    } else if (a.M > 0) {
        e = for_backward(f, [&](auto ch, auto th, auto rows) {
            constexpr int CH = decltype(ch)::value, TH = decltype(th)::value, ROWS = decltype(rows)::value;
            // rows ahead, as the registers of the workgroup's waves allow
            constexpr int AHEAD = CH == 1 ? 3 : TH == 768 ? 2 : 1;
            auto from = [&](auto dt) {
                constexpr int DT = decltype(dt)::value;
                return launch(!a.packed ? norm_backward_kernel<DT, 0, CH, TH, ROWS, AHEAD>
                              : a.format == FO_PACK_INT8
                                  ? norm_backward_kernel<DT, 1 + FO_PACK_INT8, CH, TH, ROWS, AHEAD>
                                  : norm_backward_kernel<DT, 1 + FO_PACK_E4M3, CH, TH, ROWS, AHEAD>,
                              f.blocks, TH * ROWS, s, a);
            };
            return dtype == FO_FP16 ? from(Int<FO_FP16>()) : from(Int<FO_BF16>());
        });
    }
    if (e == hipSuccess && (dgamma || dbeta)) {
        const int count = a.M > 0 ? (int)f.blocks : 0;
        const int64_t per = (norm_partial_cols(a.N) + kReduceCols - 1) / kReduceCols;
        e = launch(norm_reduce_kernel, (uint32_t)(per * (dgamma && dbeta ? 2 : 1)), kReduceThreads, s, a.partial, count, a.N,
                   dgamma, dbeta);
    }
    return e;
}

}  // namespace fo
