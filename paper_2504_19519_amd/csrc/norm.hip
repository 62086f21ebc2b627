// Layer norm and RMS norm, forward and backward.
//
//   mu = sum(x) / N (RMS norm: 0), r = 1 / sqrt(sum((x - mu)^2) / N + eps),
//   y = (x - mu) r gamma + beta;
//   with h = (x - mu) r and g = dy gamma:
//   dx = r (g - mean(g) - h mean(g h))   (RMS norm: without mean(g)),
//   dgamma = sum over rows of dy h, dbeta = sum over rows of dy.
//
// Both are bound by memory. A row is read once and held in registers, as eight
// values per chunk in 16 bits, between its statistics and its output: a wave per
// row for short rows, a workgroup per row for longer ones. All sums are in fp32;
// the variance is the mean square of the differences from the mean, so that a
// large mean costs it no digits.
//
// Backward: a workgroup takes rows blocks apart and keeps its columns' sums of
// dy h and dy in registers over all of them; the workgroups' sums are added in
// a second launch, in one order, so that equal calls give equal bits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "rowops.h"
#include "rows.h"

namespace fo {
namespace {

// Sums of `v` over the TH threads of a row (TH > 64: the whole workgroup; `lds`
// has TH / 64 words that nothing else uses until the next barrier).
template <int TH>
__device__ __forceinline__ float row_sum(float v, float* lds) {
    v = wave_sum(v);
    if constexpr (TH > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < TH / 64; ++w) v += lds[w];
    }
    return v;
}

template <int DT, int CH, int TH, int ROWS>
__global__ __launch_bounds__(TH * ROWS) void norm_forward_kernel(const NormArgs a) {
    static_assert(TH == 64 || ROWS == 1, "a barrier per row");
    __shared__ float s_mean[TH / 64], s_square[TH / 64];
    const int lane = threadIdx.x % TH;
    const int64_t i = (int64_t)blockIdx.x * ROWS + threadIdx.x / TH;
    if (i >= a.M) return;
    const uint16_t* row = a.x + i * a.ldx;
    const int full = (int)(a.N >> 3), tail = (int)(a.N & 7);
    // A lane's sum is scaled by the power of two that makes N at most 1, so that the
    // row's sums (of squares: up to 2^120 on average) stay in fp32's range.
    const float n = (float)a.N * a.scale;

    u32x4_t v[CH];
#pragma unroll
    for (int t = 0; t < CH; ++t) {
        const int c = lane + TH * t;
        v[t] = u32x4_t{0u, 0u, 0u, 0u};
        if (c < full) v[t] = load8(row + 8 * c);
    }
    const bool has_tail = lane < tail;
    const float xt = has_tail ? to_f32<DT>(row[8 * full + lane]) : 0.0f;

    if (a.packed) {
        const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK;
        uint8_t* packed = a.packed + i * blocks * FO_PACK_BLOCK;
        uint8_t* scales = a.scales + i * blocks;
        const int whole = (int)(a.N / FO_PACK_BLOCK) * 4;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = lane + TH * t;
            if (c < whole) {
                if (a.format == FO_PACK_INT8) pack_chunk<DT, FO_PACK_INT8>(v[t], c, packed, scales);
                else pack_chunk<DT, FO_PACK_E4M3>(v[t], c, packed, scales);
            }
        }
        // (read again here, ahead of any store to y, which may be x)
        if (a.N % FO_PACK_BLOCK && lane < 64) {
            if (a.format == FO_PACK_INT8) pack_last<DT, FO_PACK_INT8>(row, a.N, lane, packed, scales);
            else pack_last<DT, FO_PACK_E4M3>(row, a.N, lane, packed, scales);
        }
    }

    float mean = 0.0f;
    if (a.layer) {
        float sum = xt;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            float f[8];
            widen<DT>(v[t], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += f[e];
        }
        mean = row_sum<TH>(sum * a.scale, s_mean) / n;
    }
    float square = has_tail ? (xt - mean) * (xt - mean) : 0.0f;
#pragma unroll
    for (int t = 0; t < CH; ++t) {
        float f[8], q = 0.0f;
        widen<DT>(v[t], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) q += (f[e] - mean) * (f[e] - mean);
        if (lane + TH * t < full) square += q;
    }
    const float rstd = 1.0f / sqrtf(row_sum<TH>(square * a.scale, s_square) / n + a.eps);
    if (lane == 0) {
        if (a.mean) a.mean[i] = mean;
        if (a.rstd) a.rstd[i] = rstd;
    }

    uint16_t* out = a.y + i * a.ldy;
#pragma unroll
    for (int t = 0; t < CH; ++t) {
        const int c = lane + TH * t;
        if (c < full) {
            float f[8], p[8];
            widen<DT>(v[t], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = (f[e] - mean) * rstd;
            if (a.gamma) {
                widen<DT>(load8(a.gamma + 8 * c), p);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] *= p[e];
            }
            if (a.beta) {
                widen<DT>(load8(a.beta + 8 * c), p);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] += p[e];
            }
            store8(out + 8 * c, narrow<DT>(f));
        }
    }
    if (has_tail) {
        const int c = 8 * full + lane;
        float f = (xt - mean) * rstd;
        if (a.gamma) f *= to_f32<DT>(a.gamma[c]);
        if (a.beta) f += to_f32<DT>(a.beta[c]);
        out[c] = (uint16_t)from_f32<DT>(f);
    }
}

// SRC: where x comes from: 0 the input itself, 1 + format a checkpoint of it.
template <int DT, int SRC, int CH, int TH, int ROWS>
__global__ __launch_bounds__(TH * ROWS) void norm_backward_kernel(const NormArgs a) {
    static_assert(TH == 64 || ROWS == 1, "a barrier per row");
    __shared__ float s_sum[2][2][TH / 64];
    const int lane = threadIdx.x % TH;
    const int full = (int)(a.N >> 3), tail = (int)(a.N & 7);
    const float inv_n = 1.0f / (float)a.N;
    const bool has_tail = lane < tail;
    const int64_t blocks = (a.N + FO_PACK_BLOCK - 1) / FO_PACK_BLOCK;
    const int64_t first = (int64_t)blockIdx.x * ROWS + threadIdx.x / TH, step = (int64_t)gridDim.x * ROWS;

    float dgamma[CH][8], dbeta[CH][8], dgamma_t = 0.0f, dbeta_t = 0.0f;
#pragma unroll
    for (int t = 0; t < CH; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) dgamma[t][e] = dbeta[t][e] = 0.0f;

    int parity = 0;
    for (int64_t i = first; i < a.M; i += step, parity ^= 1) {
        const uint16_t* grow = a.dy + i * a.ldy;
        const uint16_t* row = SRC == 0 ? a.x + i * a.ldx : nullptr;
        const uint8_t* packed = SRC ? a.packed + i * blocks * FO_PACK_BLOCK : nullptr;
        const uint8_t* scales = SRC ? a.scales + i * blocks : nullptr;
        u32x4_t vg[CH];
        u32x4_t vx[SRC ? 1 : CH];
        u32x2_t code[SRC ? CH : 1];
        uint32_t sb[SRC ? CH : 1];
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = lane + TH * t;
            vg[t] = u32x4_t{0u, 0u, 0u, 0u};
            if constexpr (SRC == 0) {
                vx[t] = vg[t];
            } else {
                code[t] = u32x2_t{0u, 0u};
                sb[t] = 0u;
            }
            if (c < full) {
                vg[t] = load8(grow + 8 * c);
                if constexpr (SRC == 0) {
                    vx[t] = load8(row + 8 * c);
                } else {
                    code[t] = *reinterpret_cast<const u32x2_t*>(packed + 8 * c);
                    sb[t] = scales[c >> 2];
                }
            }
        }
        const float mean = a.layer ? a.mean[i] : 0.0f, rstd = a.rstd[i];
        auto values = [&](int t, float* h, float* d) {
            widen<DT>(vg[t], d);
            if constexpr (SRC == 0) widen<DT>(vx[t], h);
            else decode8<SRC - 1>(code[t], scale_of(sb[t]), h);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = (h[e] - mean) * rstd;
        };
        auto scaled = [&](int c, float* d) {
            if (a.gamma) {
                float p[8];
                widen<DT>(load8(a.gamma + 8 * c), p);
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] *= p[e];
            }
        };
        float s1 = 0.0f, s2 = 0.0f, ht = 0.0f, gt = 0.0f;
        if (has_tail) {
            const int c = 8 * full + lane;
            if constexpr (SRC == 0) ht = to_f32<DT>(row[c]);
            else ht = decode1<SRC - 1>(packed[c], scale_of(scales[c / FO_PACK_BLOCK]));
            ht = (ht - mean) * rstd;
            gt = to_f32<DT>(grow[c]);
            dgamma_t += gt * ht;
            dbeta_t += gt;
            if (a.gamma) gt *= to_f32<DT>(a.gamma[c]);
            s1 = gt;
            s2 = gt * ht;
        }
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = lane + TH * t;
            if (c < full) {
                float h[8], d[8];
                values(t, h, d);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dgamma[t][e] += d[e] * h[e];
                    dbeta[t][e] += d[e];
                }
                scaled(c, d);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s1 += d[e];
                    s2 += d[e] * h[e];
                }
            }
        }
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if constexpr (TH > 64) {
            // (two sets of words, so that one barrier per row is enough)
            if ((threadIdx.x & 63) == 0) {
                s_sum[parity][0][threadIdx.x >> 6] = s1;
                s_sum[parity][1][threadIdx.x >> 6] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int w = 0; w < TH / 64; ++w) {
                s1 += s_sum[parity][0][w];
                s2 += s_sum[parity][1][w];
            }
        }
        if (a.dx) {
            const float m1 = a.layer ? s1 * inv_n : 0.0f, m2 = s2 * inv_n;
            uint16_t* out = a.dx + i * a.lddx;
#pragma unroll
            for (int t = 0; t < CH; ++t) {
                const int c = lane + TH * t;
                if (c < full) {
                    float h[8], d[8];
                    values(t, h, d);
                    scaled(c, d);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[e] = rstd * (d[e] - m1 - h[e] * m2);
                    store8(out + 8 * c, narrow<DT>(d));
                }
            }
            if (has_tail) out[8 * full + lane] = (uint16_t)from_f32<DT>(rstd * (gt - m1 - ht * m2));
        }
    }
    if (a.partial) {
        float* pg = a.partial + first * 2 * a.N;
        float* pb = pg + a.N;
#pragma unroll
        for (int t = 0; t < CH; ++t) {
            const int c = lane + TH * t;
            if (c < full) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    pg[8 * c + e] = dgamma[t][e];
                    pb[8 * c + e] = dbeta[t][e];
                }
            }
        }
        if (has_tail) {
            pg[8 * full + lane] = dgamma_t;
            pb[8 * full + lane] = dbeta_t;
        }
    }
}

// dgamma and dbeta: the sums of `count` rows of partial sums, 32 columns per
// workgroup (the 2 N columns of both), eight rows at a time.
__global__ __launch_bounds__(256) void norm_reduce_kernel(const float* partial, int count, int64_t N, float* dgamma,
                                                          float* dbeta) {
    __shared__ float s[8][33];
    const int col = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + col;
    float sum = 0.0f;
    if (c < 2 * N)
        for (int g = part; g < count; g += 8) sum += partial[(int64_t)g * 2 * N + c];
    s[part][col] = sum;
    __syncthreads();
    if (part == 0 && c < 2 * N) {
        float* out = c < N ? dgamma : dbeta;
        sum = 0.0f;
#pragma unroll
        for (int p = 0; p < 8; ++p) sum += s[p][col];
        if (out) out[c < N ? c : c - N] = sum;
    }
}

template <int N>
using Int = std::integral_constant<int, N>;

// The form's constants, as f(chunks, threads, rows).
template <typename F>
void for_form(const NormForm& f, F go) {
    if (f.threads == 64) {
        if (f.chunks == 1) go(Int<1>(), Int<64>(), Int<4>());
        else if (f.chunks == 2) go(Int<2>(), Int<64>(), Int<4>());
        else go(Int<4>(), Int<64>(), Int<4>());
    } else if (f.threads == 256) {
        if (f.chunks == 2) go(Int<2>(), Int<256>(), Int<1>());
        else go(Int<4>(), Int<256>(), Int<1>());
    } else if (f.threads == 512) {
        go(Int<4>(), Int<512>(), Int<1>());
    } else {
        go(Int<4>(), Int<1024>(), Int<1>());
    }
}

NormForm row_form(int64_t N) {
    NormForm f{};
    f.threads = N <= 2048 ? 64 : N <= 8192 ? 256 : N <= 16384 ? 512 : 1024;
    const int64_t per = (N / 8 + f.threads - 1) / f.threads;
    f.chunks = per <= 1 && f.threads == 64 ? 1 : per <= 2 && f.threads <= 256 ? 2 : 4;
    f.rows = f.threads == 64 ? 4 : 1;
    return f;
}

}  // namespace

NormForm norm_forward_form(int64_t M, int64_t N) {
    NormForm f = row_form(N);
    f.blocks = (uint32_t)((M + f.rows - 1) / f.rows);
    return f;
}

NormForm norm_backward_form(int64_t M, int64_t N) {
    NormForm f = row_form(N);
    f.blocks = (uint32_t)std::min<int64_t>((M + f.rows - 1) / f.rows, 512);
    return f;
}

hipError_t launch_norm_forward(int dtype, const NormArgs& a, hipStream_t s) {
    const NormForm f = norm_forward_form(a.M, a.N);
    for_form(f, [&](auto ch, auto th, auto rows) {
        constexpr int CH = decltype(ch)::value, TH = decltype(th)::value, ROWS = decltype(rows)::value;
        const dim3 g(f.blocks), b(TH * ROWS);
        if (dtype == FO_FP16) hipLaunchKernelGGL((norm_forward_kernel<FO_FP16, CH, TH, ROWS>), g, b, 0, s, a);
        else hipLaunchKernelGGL((norm_forward_kernel<FO_BF16, CH, TH, ROWS>), g, b, 0, s, a);
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(int dtype, const NormArgs& a, float* dgamma, float* dbeta, hipStream_t s) {
    const NormForm f = norm_backward_form(a.M, a.N);
    if (a.M > 0) {
        for_form(f, [&](auto ch, auto th, auto rows) {
            constexpr int CH = decltype(ch)::value, TH = decltype(th)::value, ROWS = decltype(rows)::value;
            const dim3 g(f.blocks), b(TH * ROWS);
            auto go = [&](auto dt, auto src) {
                hipLaunchKernelGGL((norm_backward_kernel<decltype(dt)::value, decltype(src)::value, CH, TH, ROWS>), g, b,
                                   0, s, a);
            };
            const int src = a.packed ? 1 + a.format : 0;
            auto from = [&](auto dt) {
                if (src == 0) go(dt, Int<0>());
                else if (src == 1) go(dt, Int<1>());
                else go(dt, Int<2>());
            };
            if (dtype == FO_FP16) from(Int<FO_FP16>());
            else from(Int<FO_BF16>());
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (dgamma || dbeta) {
        const int count = a.M > 0 ? (int)f.blocks * f.rows : 0;
        hipLaunchKernelGGL(norm_reduce_kernel, dim3((uint32_t)((2 * a.N + 31) / 32)), dim3(256), 0, s, a.partial, count,
                           a.N, dgamma, dbeta);
    }
    return hipGetLastError();
}

}  // namespace fo
