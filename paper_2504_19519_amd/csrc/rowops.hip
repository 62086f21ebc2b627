// C ABI entry points of the row operators: argument checks and launches.
#include "rowops.h"

#include <algorithm>
#include <string>

#include "fo_internal.h"

namespace fo {
namespace {

bool is_dtype(int32_t d) { return d == FO_FP16 || d == FO_BF16; }
bool is_format(int32_t f) { return f == FO_PACK_INT8 || f == FO_PACK_E4M3; }
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Whether two matrices of 16-bit values, Mp and Mq rows of N, ldp and ldq apart, share
// memory other than by being the same one (where that is allowed).
bool clash(const void* p, int64_t Mp, int64_t ldp, const void* q, int64_t Mq, int64_t ldq, int64_t N, bool same_allowed) {
    if (!p || !q || Mp == 0 || Mq == 0 || N == 0) return false;
    if (Mp == 1) ldp = ldq;         // one row has no distance of its own
    if (Mq == 1) ldq = ldp;
    if (same_allowed && p == q && ldp == ldq) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
    const uintptr_t xe = x + 2 * (uintptr_t)((Mp - 1) * ldp + N), ye = y + 2 * (uintptr_t)((Mq - 1) * ldq + N);
    if (xe <= y || ye <= x) return false;
    if (ldp != ldq) return true;
    // columns side by side in rows of one length
    const uintptr_t d = (x < y ? y - x : x - y) % (2 * (uintptr_t)ldp);
    return d < 2 * (uintptr_t)N || d + 2 * (uintptr_t)N > 2 * (uintptr_t)ldp;
}

// A matrix argument of 16-bit values.
fo_status check_rows(const char* what, const void* p, int64_t N, int64_t ld) {
    if (!p) return fail(FO_ERR_ARG, std::string(what) + " is NULL");
    if (!aligned(p, 2)) return fail(FO_ERR_ARG, std::string(what) + " must be 2-byte aligned");
    if (ld < N) return fail(FO_ERR_ARG, std::string(what) + ": rows are closer together than their length");
    return FO_OK;
}

fo_status check_pack(const void* packed, const void* scales, int32_t format) {
    if (!packed || !scales) return fail(FO_ERR_ARG, "a checkpoint needs packed and scales");
    if (!is_format(format)) return fail(FO_ERR_ARG, "bad checkpoint format");
    if (!aligned(packed, 16)) return fail(FO_ERR_ARG, "packed must be 16-byte aligned");
    return FO_OK;
}

fo_status check_vectors(const void* gamma, const void* beta, const void* mean, const void* rstd) {
    if (!aligned(gamma, 2) || !aligned(beta, 2)) return fail(FO_ERR_ARG, "gamma and beta must be 2-byte aligned");
    if (!aligned(mean, 4) || !aligned(rstd, 4)) return fail(FO_ERR_ARG, "mean and rstd must be 4-byte aligned");
    return FO_OK;
}

// Whether `blocks` workgroups of `threads` fit one launch.
bool launchable(int64_t blocks, int64_t threads) { return blocks <= (int64_t)UINT32_MAX / threads; }

fo_status done(hipError_t e, const char* what) {
    return e == hipSuccess ? FO_OK : fail(FO_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// Eighths of a wave that a row takes, at most (route.hip).
int64_t slices_of(int64_t n) { return (n + 63) / 64; }

int64_t norm_partial_bytes(int64_t M, int64_t N) {
    const NormForm f = norm_backward_form(M, N);
    return M > 0 && N > 0 ? (int64_t)f.blocks * 2 * norm_partial_cols(N) * 4 : 0;
}

fo_status check_route(int32_t dtype, int64_t T, int32_t K, int64_t H, const void* slot_of, const void* weights,
                      int64_t capacity) {
    if (!is_dtype(dtype)) return fail(FO_ERR_ARG, "bad dtype");
    if (T < 0 || H < 0 || capacity < 0) return fail(FO_ERR_ARG, "negative size");
    if (K < 1 || K > FO_ROUTE_MAX_CHOICES) return fail(FO_ERR_ARG, "K must be in [1, 64]");
    if (T > INT32_MAX || T * K > INT32_MAX || capacity > INT32_MAX || H > INT32_MAX)
        return fail(FO_ERR_SHAPE, "T * K, H and capacity must be below 2^31");
    if (T > 0 && !slot_of) return fail(FO_ERR_ARG, "slot_of is NULL");
    if (!aligned(slot_of, 4) || !aligned(weights, 4))
        return fail(FO_ERR_ARG, "slot_of and weights must be 4-byte aligned");
    if (T * slices_of(H) > (int64_t)UINT32_MAX - 64 ||
        !launchable((T * std::max<int64_t>((H + 511) / 512 + 1, K) + 3) / 4 + 16 * FO_ROUTE_MAX_EXPERTS, 256))
        return fail(FO_ERR_SHAPE, "too many rows for one launch");
    return FO_OK;
}

fo_status check_padding(const int32_t* offsets, const int32_t* counts, int32_t E) {
    if (!offsets != !counts) return fail(FO_ERR_ARG, "offsets and counts go together");
    if (offsets && (E < 1 || E > FO_ROUTE_MAX_EXPERTS)) return fail(FO_ERR_ARG, "E must be in [1, 1024]");
    if (!aligned(offsets, 4) || !aligned(counts, 4))
        return fail(FO_ERR_ARG, "offsets and counts must be 4-byte aligned");
    return FO_OK;
}

}  // namespace
}  // namespace fo

extern "C" {

fo_status fo_norm_forward(int32_t kind, int32_t dtype, int64_t M, int64_t N, const void* x, int64_t ldx,
                          const void* gamma, const void* beta, float eps, void* y, int64_t ldy, float* mean,
                          float* rstd, void* packed, void* scales, int32_t format, void* stream) {
    fo::clear_error();
    fo_status st;
    if (kind != FO_NORM_LAYER && kind != FO_NORM_RMS) return fo::fail(FO_ERR_ARG, "bad norm kind");
    if (!fo::is_dtype(dtype)) return fo::fail(FO_ERR_ARG, "bad dtype");
    if (M < 0 || N < 0) return fo::fail(FO_ERR_ARG, "negative size");
    if (!(eps >= 0.0f)) return fo::fail(FO_ERR_ARG, "eps must be >= 0");
    if (N > fo::kMaxNormCols) return fo::fail(FO_ERR_UNSUPPORTED, "rows of more than 32768 columns");
    if (M == 0 || N == 0) return FO_OK;
    if ((st = fo::check_rows("x", x, N, ldx)) != FO_OK || (st = fo::check_rows("y", y, N, ldy)) != FO_OK ||
        (st = fo::check_vectors(gamma, beta, mean, rstd)) != FO_OK ||
        ((packed || scales) && (st = fo::check_pack(packed, scales, format)) != FO_OK))
        return st;
    if (M > INT32_MAX) return fo::fail(FO_ERR_SHAPE, "2^31 rows or more");
    if (fo::clash(x, M, ldx, y, M, ldy, N, true)) return fo::fail(FO_ERR_ARG, "y overlaps x without being x");
    fo::NormArgs a{};
    a.x = static_cast<const uint16_t*>(x);
    a.gamma = static_cast<const uint16_t*>(gamma);
    a.beta = static_cast<const uint16_t*>(beta);
    a.y = static_cast<uint16_t*>(y);
    a.mean = mean;
    a.rstd = rstd;
    a.packed = static_cast<uint8_t*>(packed);
    a.scales = static_cast<uint8_t*>(scales);
    a.M = M; a.N = N; a.ldx = ldx; a.ldy = ldy;
    a.eps = eps;
    a.scale = 1.0f;
    while ((double)N * a.scale > 1.0) a.scale *= 0.5f;
    a.layer = kind == FO_NORM_LAYER;
    a.format = format;
    return fo::done(fo::launch_norm_forward(dtype, a, (hipStream_t)stream), "norm launch");
}

int64_t fo_norm_workspace_bytes(int64_t M, int64_t N) {
    return M < 0 || N < 0 || M > INT32_MAX || N > fo::kMaxNormCols ? 0
                                                                   : fo::norm_partial_bytes(M, N) + fo::norm_dots_bytes(M, N);
}

fo_status fo_norm_backward(int32_t kind, int32_t dtype, int64_t M, int64_t N, const void* dy, int64_t lddy,
                           const void* x, int64_t ldx, const void* packed, const void* scales, int32_t format,
                           const void* gamma, const float* mean, const float* rstd, void* dx, int64_t lddx,
                           float* dgamma, float* dbeta, void* workspace, int64_t workspace_bytes, void* stream) {
    fo::clear_error();
    fo_status st;
    if (kind != FO_NORM_LAYER && kind != FO_NORM_RMS) return fo::fail(FO_ERR_ARG, "bad norm kind");
    if (!fo::is_dtype(dtype)) return fo::fail(FO_ERR_ARG, "bad dtype");
    if (M < 0 || N < 0) return fo::fail(FO_ERR_ARG, "negative size");
    if (N > fo::kMaxNormCols) return fo::fail(FO_ERR_UNSUPPORTED, "rows of more than 32768 columns");
    if (!dx && !dgamma && !dbeta) return fo::fail(FO_ERR_ARG, "no gradient asked for");
    if (!fo::aligned(dgamma, 4) || !fo::aligned(dbeta, 4))
        return fo::fail(FO_ERR_ARG, "dgamma and dbeta must be 4-byte aligned");
    if (N == 0) return FO_OK;
    if (M > INT32_MAX) return fo::fail(FO_ERR_SHAPE, "2^31 rows or more");
    const bool sums = dgamma || dbeta;
    if (M > 0) {
        if (!x == !(packed || scales)) return fo::fail(FO_ERR_ARG, "x or a checkpoint of it, one of the two");
        if ((st = fo::check_rows("dy", dy, N, lddy)) != FO_OK || (x && (st = fo::check_rows("x", x, N, ldx)) != FO_OK) ||
            (!x && (st = fo::check_pack(packed, scales, format)) != FO_OK) ||
            (dx && (st = fo::check_rows("dx", dx, N, lddx)) != FO_OK) ||
            (st = fo::check_vectors(gamma, nullptr, mean, rstd)) != FO_OK)
            return st;
        if (!rstd || (kind == FO_NORM_LAYER && !mean)) return fo::fail(FO_ERR_ARG, "the rows' statistics are missing");
        if (fo::clash(dx, M, lddx, dy, M, lddy, N, true) || fo::clash(dx, M, lddx, x, M, ldx, N, true))
            return fo::fail(FO_ERR_ARG, "dx overlaps dy or x without being it");
        if ((sums || fo::norm_dots_bytes(M, N) > 0) &&
            (!workspace || !fo::aligned(workspace, 16) || workspace_bytes < fo_norm_workspace_bytes(M, N)))
            return fo::fail(FO_ERR_ARG, "workspace: fo_norm_workspace_bytes(M, N) bytes, 16-byte aligned");
    }
    fo::NormArgs a{};
    a.x = static_cast<const uint16_t*>(x);
    a.gamma = static_cast<const uint16_t*>(gamma);
    a.dy = static_cast<const uint16_t*>(dy);
    a.dx = static_cast<uint16_t*>(dx);
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.packed = static_cast<uint8_t*>(const_cast<void*>(packed));
    a.scales = static_cast<uint8_t*>(const_cast<void*>(scales));
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    if (fo::norm_dots_bytes(M, N) > 0)
        a.dots = reinterpret_cast<float*>(static_cast<char*>(workspace) + fo::norm_partial_bytes(M, N));
    a.M = M; a.N = N; a.ldx = ldx; a.ldy = lddy; a.lddx = lddx;
    a.layer = kind == FO_NORM_LAYER;
    a.format = format;
    a.with_beta = dbeta != nullptr;
    return fo::done(fo::launch_norm_backward(dtype, a, dgamma, dbeta, (hipStream_t)stream), "norm backward launch");
}

static fo_status pack_args(int32_t dtype, int32_t format, int64_t M, int64_t N, const void* x, int64_t ldx,
                           const void* packed, const void* scales, fo::PackArgs* a) {
    fo_status st;
    if (!fo::is_dtype(dtype)) return fo::fail(FO_ERR_ARG, "bad dtype");
    if (!fo::is_format(format)) return fo::fail(FO_ERR_ARG, "bad checkpoint format");
    if (M < 0 || N < 0) return fo::fail(FO_ERR_ARG, "negative size");
    if (M == 0 || N == 0) return FO_OK;
    if ((st = fo::check_rows("x", x, N, ldx)) != FO_OK || (st = fo::check_pack(packed, scales, format)) != FO_OK)
        return st;
    if (N > INT32_MAX || M > INT32_MAX || M * 4 * fo::pack_blocks(N) > (int64_t)UINT32_MAX - 1024)
        return fo::fail(FO_ERR_SHAPE, "too many values for one launch");
    a->x = static_cast<uint16_t*>(const_cast<void*>(x));
    a->packed = static_cast<uint8_t*>(const_cast<void*>(packed));
    a->scales = static_cast<uint8_t*>(const_cast<void*>(scales));
    a->M = M; a->N = N; a->ldx = ldx;
    return FO_OK;
}

fo_status fo_pack_rows(int32_t dtype, int32_t format, int64_t M, int64_t N, const void* x, int64_t ldx, void* packed,
                       void* scales, void* stream) {
    fo::clear_error();
    fo::PackArgs a{};
    const fo_status st = pack_args(dtype, format, M, N, x, ldx, packed, scales, &a);
    if (st != FO_OK || M == 0 || N == 0) return st;
    return fo::done(fo::launch_pack(dtype, format, a, (hipStream_t)stream), "pack launch");
}

fo_status fo_unpack_rows(int32_t dtype, int32_t format, int64_t M, int64_t N, const void* packed, const void* scales,
                         void* out, int64_t ldo, void* stream) {
    fo::clear_error();
    fo::PackArgs a{};
    const fo_status st = pack_args(dtype, format, M, N, out, ldo, packed, scales, &a);
    if (st != FO_OK || M == 0 || N == 0) return st;
    return fo::done(fo::launch_unpack(dtype, format, a, (hipStream_t)stream), "unpack launch");
}

int64_t fo_route_capacity(int64_t T, int32_t K, int32_t E, int32_t align) {
    if (T < 0 || T > INT32_MAX || K < 1 || E < 1 || align < 1) return 0;
    const int64_t pairs = T * K;
    return pairs + std::min<int64_t>(E, pairs) * (align - 1);
}

int64_t fo_route_workspace_bytes(int64_t T, int32_t K, int32_t E) {
    if (T < 0 || T > INT32_MAX || K < 1 || E < 1) return 0;
    const int64_t blocks = fo::sort_blocks(T * K);
    return blocks > 1 ? blocks * E * 4 : 0;
}

fo_status fo_route_sort(const void* ids, int32_t id_bytes, int64_t T, int32_t K, int32_t E, int32_t align,
                        int32_t* offsets, int32_t* counts, int32_t* slot_of, int32_t* pair_of, int64_t capacity,
                        void* workspace, int64_t workspace_bytes, void* stream) {
    fo::clear_error();
    if (T < 0) return fo::fail(FO_ERR_ARG, "negative size");
    if (K < 1 || K > FO_ROUTE_MAX_CHOICES) return fo::fail(FO_ERR_ARG, "K must be in [1, 64]");
    if (E < 1 || E > FO_ROUTE_MAX_EXPERTS) return fo::fail(FO_ERR_ARG, "E must be in [1, 1024]");
    if (align < 1) return fo::fail(FO_ERR_ARG, "align must be >= 1");
    if (id_bytes != 4 && id_bytes != 8) return fo::fail(FO_ERR_ARG, "ids are of 4 or 8 bytes");
    const int64_t need = fo_route_capacity(T, K, E, align);
    if (T > INT32_MAX || T * K > INT32_MAX || need > INT32_MAX)
        return fo::fail(FO_ERR_SHAPE, "more than 2^31 - 1 pairs or rows");
    if (!offsets || !counts || (T > 0 && (!ids || !slot_of))) return fo::fail(FO_ERR_ARG, "null ids or output");
    if (!fo::aligned(ids, id_bytes) || !fo::aligned(offsets, 4) || !fo::aligned(counts, 4) || !fo::aligned(slot_of, 4) ||
        !fo::aligned(pair_of, 4))
        return fo::fail(FO_ERR_ARG, "ids and outputs must be aligned to their elements");
    if (pair_of && capacity < need)
        return fo::fail(FO_ERR_ARG, "capacity: fo_route_capacity(T, K, E, align) rows at least");
    if (fo_route_workspace_bytes(T, K, E) > 0 &&
        (!workspace || !fo::aligned(workspace, 4) || workspace_bytes < fo_route_workspace_bytes(T, K, E)))
        return fo::fail(FO_ERR_ARG, "workspace: fo_route_workspace_bytes(T, K, E) bytes, 4-byte aligned");
    fo::SortArgs a{};
    a.ids = ids;
    a.pairs = T * K;
    a.experts = E;
    a.align = align;
    a.id_bytes = id_bytes;
    a.offsets = offsets;
    a.counts = counts;
    a.slot_of = slot_of;
    a.pair_of = pair_of;
    a.hist = static_cast<int32_t*>(workspace);
    return fo::done(fo::launch_sort(a, (hipStream_t)stream), "route sort launch");
}

fo_status fo_route_permute(int32_t dtype, int64_t T, int32_t K, int64_t H, const void* x, int64_t ldx,
                           const int32_t* slot_of, void* rows, int64_t ldr, int64_t capacity, const int32_t* offsets,
                           const int32_t* counts, int32_t E, void* stream) {
    fo::clear_error();
    fo_status st;
    if ((st = fo::check_route(dtype, T, K, H, slot_of, nullptr, capacity)) != FO_OK ||
        (st = fo::check_padding(offsets, counts, E)) != FO_OK)
        return st;
    if (T == 0 || H == 0 || capacity == 0) return FO_OK;
    if ((st = fo::check_rows("x", x, H, ldx)) != FO_OK || (st = fo::check_rows("rows", rows, H, ldr)) != FO_OK) return st;
    if (fo::clash(x, T, ldx, rows, capacity, ldr, H, false)) return fo::fail(FO_ERR_ARG, "rows overlaps x");
    fo::RouteArgs a{};
    a.x = static_cast<const uint16_t*>(x);
    a.rows = static_cast<uint16_t*>(rows);
    a.slot_of = slot_of;
    a.offsets = offsets;
    a.counts = counts;
    a.H = H; a.ldx = ldx; a.ldr = ldr;
    a.T = (int32_t)T; a.K = K; a.E = E; a.capacity = (int32_t)capacity;
    return fo::done(fo::launch_permute(a, (hipStream_t)stream), "route permute launch");
}

fo_status fo_route_combine(int32_t dtype, int64_t T, int32_t K, int64_t H, const void* rows, int64_t ldr,
                           int64_t capacity, const int32_t* slot_of, const float* weights, void* out, int64_t ldo,
                           void* packed, void* scales, int32_t format, void* stream) {
    fo::clear_error();
    fo_status st;
    if ((st = fo::check_route(dtype, T, K, H, slot_of, weights, capacity)) != FO_OK) return st;
    if (T == 0 || H == 0) return FO_OK;
    if ((capacity > 0 && (st = fo::check_rows("rows", rows, H, ldr)) != FO_OK) ||
        (st = fo::check_rows("out", out, H, ldo)) != FO_OK ||
        ((packed || scales) && (st = fo::check_pack(packed, scales, format)) != FO_OK))
        return st;
    if (fo::clash(rows, capacity, ldr, out, T, ldo, H, false)) return fo::fail(FO_ERR_ARG, "out overlaps rows");
    fo::RouteArgs a{};
    a.rows = static_cast<uint16_t*>(const_cast<void*>(rows));
    a.out = static_cast<uint16_t*>(out);
    a.slot_of = slot_of;
    a.weights = weights;
    a.packed = static_cast<uint8_t*>(packed);
    a.scales = static_cast<uint8_t*>(scales);
    a.H = H; a.ldr = ldr; a.ldo = ldo;
    a.T = (int32_t)T; a.K = K; a.capacity = (int32_t)capacity; a.format = format;
    return fo::done(fo::launch_combine(dtype, a, (hipStream_t)stream), "route combine launch");
}

fo_status fo_route_combine_backward(int32_t dtype, int64_t T, int32_t K, int64_t H, const void* dout, int64_t lddo,
                                    const void* rows, int64_t ldr, const void* packed, const void* scales,
                                    int32_t format, int64_t capacity, const int32_t* slot_of, const float* weights,
                                    void* drows, int64_t lddr, float* dweights, const int32_t* offsets,
                                    const int32_t* counts, int32_t E, void* stream) {
    fo::clear_error();
    fo_status st;
    if ((st = fo::check_route(dtype, T, K, H, slot_of, weights, capacity)) != FO_OK ||
        (st = fo::check_padding(offsets, counts, E)) != FO_OK)
        return st;
    if (!drows && !dweights) return fo::fail(FO_ERR_ARG, "no gradient asked for");
    if (!fo::aligned(dweights, 4)) return fo::fail(FO_ERR_ARG, "dweights must be 4-byte aligned");
    if (T == 0) return FO_OK;
    const bool read = dweights && H > 0 && capacity > 0;
    if (read && !rows == !(packed || scales))
        return fo::fail(FO_ERR_ARG, "dweights needs rows or a checkpoint of them, one of the two");
    if (H > 0 && ((st = fo::check_rows("dout", dout, H, lddo)) != FO_OK ||
                  (read && rows && (st = fo::check_rows("rows", rows, H, ldr)) != FO_OK) ||
                  (read && !rows && (st = fo::check_pack(packed, scales, format)) != FO_OK) ||
                  (drows && capacity > 0 && (st = fo::check_rows("drows", drows, H, lddr)) != FO_OK)))
        return st;
    if (fo::clash(drows, capacity, lddr, read ? rows : nullptr, capacity, ldr, H, true))
        return fo::fail(FO_ERR_ARG, "drows overlaps rows without being it");
    if (fo::clash(drows, capacity, lddr, dout, T, lddo, H, false)) return fo::fail(FO_ERR_ARG, "drows overlaps dout");
    fo::RouteArgs a{};
    a.x = static_cast<const uint16_t*>(dout);
    a.rows = static_cast<uint16_t*>(const_cast<void*>(rows));
    a.out = static_cast<uint16_t*>(drows);
    a.slot_of = slot_of;
    a.weights = weights;
    a.dweights = dweights;
    a.offsets = offsets;
    a.counts = counts;
    if (read && !rows) {
        a.packed = static_cast<uint8_t*>(const_cast<void*>(packed));
        a.scales = static_cast<uint8_t*>(const_cast<void*>(scales));
    }
    a.H = H; a.ldx = lddo; a.ldr = ldr; a.ldo = lddr;
    a.T = (int32_t)T; a.K = K; a.E = E; a.capacity = (int32_t)capacity; a.format = format;
    return fo::done(fo::launch_combine_backward(dtype, a, (hipStream_t)stream), "route combine backward launch");
}

}  // extern "C"
