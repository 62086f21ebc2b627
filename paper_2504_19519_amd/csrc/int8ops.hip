// C ABI entry points of the 8-bit operators: argument checks and launches.
#include "int8ops.h"

#include <algorithm>
#include <string>

#include "checks.h"
#include "fo_internal.h"
#include "rowops.h"

namespace fo {
namespace {

// A matrix argument of 8-bit codes.
fo_status check_codes(const char* what, const void* p, int64_t n, int64_t ld) {
    if (!p) return fail(FO_ERR_ARG, std::string(what) + " is NULL");
    if (!aligned(p, 16) || ld % 16 != 0) return fail(FO_ERR_ARG, std::string(what) + ": rows must be 16-byte aligned");
    if (ld < int8_row_bytes(n)) return fail(FO_ERR_ARG, std::string(what) + ": rows are closer together than their length");
    if (ld > kMaxInt8Row) return fail(FO_ERR_SHAPE, std::string(what) + ": rows more than 2^22 bytes apart");
    return FO_OK;
}

// Bytes from a matrix's first element to its last.
int64_t extent(int64_t rows, int64_t n, int64_t ld, int64_t bytes) { return rows > 0 && n > 0 ? ((rows - 1) * ld + n) * bytes : 0; }
int64_t codes_extent(int64_t rows, int64_t n, int64_t ld) { return extent(rows, int8_row_bytes(n), ld, 1); }

struct Piece {
    const void* p;
    int64_t bytes;
};
template <size_t N>
bool overlaps(const Piece& a, const Piece (&others)[N]) {
    return std::any_of(others, others + N, [&](const Piece& b) { return overlap(a.p, a.bytes, b.p, b.bytes); });
}

fo_status check_scales(const char* what, const void* p) {
    if (!p) return fail(FO_ERR_ARG, std::string(what) + " is NULL");
    if (!aligned(p, 4)) return fail(FO_ERR_ARG, std::string(what) + " must be 4-byte aligned");
    return FO_OK;
}

// The scales of M rows without values: zeros.
fo_status no_values(int32_t dtype, int64_t M, float* scales, void* stream) {
    if (!scales) return FO_OK;
    if (M > INT32_MAX) return fail(FO_ERR_SHAPE, "2^31 rows or more");
    fo_status st;
    if ((st = check_scales("scales", scales)) != FO_OK) return st;
    Rows8Args a{};
    a.scales = scales;
    a.M = M;
    a.scale = 1.0f;
    return done(launch_quantize(dtype, a, (hipStream_t)stream), "quantize launch");
}

fo_status check_product(int32_t dtype, int64_t rows, int64_t N, int64_t K) {
    if (!is_dtype(dtype)) return fail(FO_ERR_ARG, "bad dtype");
    if (rows < 0 || N < 0 || K < 0) return fail(FO_ERR_ARG, "negative size");
    if (K > kMaxInt8Inner) return fail(FO_ERR_UNSUPPORTED, "sums of more than 131071 products");
    if (rows > INT32_MAX || N > INT32_MAX) return fail(FO_ERR_SHAPE, "2^31 rows or columns or more");
    return FO_OK;
}

fo_status check_operands(const void* a, const void* a_scales, int64_t lda, const void* b, const void* b_scales, int64_t ldb,
                         const void* bias, const void* c, int64_t ldc, int64_t N, int64_t K) {
    fo_status st;
    if ((K > 0 && ((st = check_codes("a", a, K, lda)) != FO_OK || (st = check_codes("b", b, K, ldb)) != FO_OK)) ||
        (st = check_scales("a_scales", a_scales)) != FO_OK || (st = check_scales("b_scales", b_scales)) != FO_OK ||
        (st = check_rows("c", c, N, ldc)) != FO_OK)
        return st;
    if (!aligned(bias, 2)) return fail(FO_ERR_ARG, "bias must be 2-byte aligned");
    return FO_OK;
}

}  // namespace
}  // namespace fo

extern "C" {

int64_t fo_int8_row_bytes(int64_t n) { return n < 0 || n > INT32_MAX ? 0 : fo::int8_row_bytes(n); }

fo_status fo_quantize_rows(int32_t dtype, int64_t M, int64_t N, const void* x, int64_t ldx, void* codes, int64_t ldc,
                           float* scales, void* stream) {
    fo::clear_error();
    fo_status st;
    if (!fo::is_dtype(dtype)) return fo::fail(FO_ERR_ARG, "bad dtype");
    if (M < 0 || N < 0) return fo::fail(FO_ERR_ARG, "negative size");
    if (M == 0) return FO_OK;
    if (N == 0) return fo::no_values(dtype, M, scales, stream);
    if (M > INT32_MAX || N > (int64_t)1 << 30) return fo::fail(FO_ERR_SHAPE, "2^31 rows or more, or rows of more than 2^30 values");
    if ((st = fo::check_rows("x", x, N, ldx)) != FO_OK) return st;
    if (!codes) return fo::fail(FO_ERR_ARG, "codes is NULL");
    if (!fo::aligned(codes, 16) || ldc % 16 != 0) return fo::fail(FO_ERR_ARG, "codes: rows must be 16-byte aligned");
    if (ldc < fo::int8_row_bytes(N)) return fo::fail(FO_ERR_ARG, "codes: rows are closer together than their length");
    if ((st = fo::check_scales("scales", scales)) != FO_OK) return st;
    if (fo::overlap(codes, fo::codes_extent(M, N, ldc), x, fo::extent(M, N, ldx, 2)) ||
        fo::overlap(scales, 4 * M, x, fo::extent(M, N, ldx, 2)) || fo::overlap(scales, 4 * M, codes, fo::codes_extent(M, N, ldc)))
        return fo::fail(FO_ERR_ARG, "x, codes and scales overlap");
    fo::Rows8Args a{};
    a.x = static_cast<const uint16_t*>(x);
    a.codes = static_cast<int8_t*>(codes);
    a.scales = scales;
    a.M = M; a.N = N; a.ldx = ldx; a.ldc = ldc;
    a.scale = 1.0f;
    return fo::done(fo::launch_quantize(dtype, a, (hipStream_t)stream), "quantize launch");
}

fo_status fo_norm_add_forward(int32_t dtype, int64_t M, int64_t N, const void* x, int64_t ldx, const void* residual,
                              int64_t ldr, const void* gamma, float eps, void* h, int64_t ldh, void* y, int64_t ldy,
                              float* rstd, void* codes, int64_t ldc, float* scales, void* stream) {
    fo::clear_error();
    fo_status st;
    if (!fo::is_dtype(dtype)) return fo::fail(FO_ERR_ARG, "bad dtype");
    if (M < 0 || N < 0) return fo::fail(FO_ERR_ARG, "negative size");
    if (!(eps >= 0.0f)) return fo::fail(FO_ERR_ARG, "eps must be >= 0");
    if (N > fo::kMaxNormCols) return fo::fail(FO_ERR_UNSUPPORTED, "rows of more than 32768 columns");
    if (M == 0) return FO_OK;
    if (N == 0) return fo::no_values(dtype, M, scales, stream);
    if (M > INT32_MAX) return fo::fail(FO_ERR_SHAPE, "2^31 rows or more");
    if (!y && !codes && !scales) return fo::fail(FO_ERR_ARG, "no output asked for: y, or codes and scales");
    if ((st = fo::check_rows("x", x, N, ldx)) != FO_OK || (residual && (st = fo::check_rows("residual", residual, N, ldr)) != FO_OK) ||
        (h && (st = fo::check_rows("h", h, N, ldh)) != FO_OK) || (y && (st = fo::check_rows("y", y, N, ldy)) != FO_OK) ||
        ((codes || scales) && ((st = fo::check_codes("codes", codes, N, ldc)) != FO_OK ||
                               (st = fo::check_scales("scales", scales)) != FO_OK)))
        return st;
    if (!fo::aligned(gamma, 2)) return fo::fail(FO_ERR_ARG, "gamma must be 2-byte aligned");
    if (!fo::aligned(rstd, 4)) return fo::fail(FO_ERR_ARG, "rstd must be 4-byte aligned");
    if (fo::clash(x, M, ldx, h, M, ldh, N, true) || fo::clash(residual, M, ldr, h, M, ldh, N, true) ||
        fo::clash(x, M, ldx, y, M, ldy, N, true) || fo::clash(residual, M, ldr, y, M, ldy, N, true))
        return fo::fail(FO_ERR_ARG, "h or y overlaps x or residual without being it");
    if (fo::clash(h, M, ldh, y, M, ldy, N, false)) return fo::fail(FO_ERR_ARG, "h and y overlap");
    if (fo::overlap(gamma, 2 * N, h, fo::extent(M, N, ldh, 2)) || fo::overlap(gamma, 2 * N, y, fo::extent(M, N, ldy, 2)))
        return fo::fail(FO_ERR_ARG, "h or y overlaps gamma");
    const fo::Piece out[] = {{codes, fo::codes_extent(M, N, ldc)}, {scales, 4 * M}, {rstd, 4 * M}};
    const fo::Piece others[] = {{x, fo::extent(M, N, ldx, 2)}, {residual, fo::extent(M, N, ldr, 2)}, {h, fo::extent(M, N, ldh, 2)},
                                {y, fo::extent(M, N, ldy, 2)}, {gamma, 2 * N}};
    for (int i = 0; i < 3; ++i) {
        if (fo::overlaps(out[i], others) || fo::overlap(out[i].p, out[i].bytes, out[(i + 1) % 3].p, out[(i + 1) % 3].bytes))
            return fo::fail(FO_ERR_ARG, "codes, scales or rstd overlaps another argument");
    }
    fo::Rows8Args a{};
    a.x = static_cast<const uint16_t*>(x);
    a.residual = static_cast<const uint16_t*>(residual);
    a.gamma = static_cast<const uint16_t*>(gamma);
    a.h = static_cast<uint16_t*>(h);
    a.y = static_cast<uint16_t*>(y);
    a.rstd = rstd;
    a.codes = static_cast<int8_t*>(codes);
    a.scales = scales;
    a.M = M; a.N = N; a.ldx = ldx; a.ldr = ldr; a.ldh = ldh; a.ldy = ldy; a.ldc = ldc;
    a.eps = eps;
    a.scale = 1.0f;
    while ((double)N * a.scale > 1.0) a.scale *= 0.5f;
    return fo::done(fo::launch_norm_add_forward(dtype, a, (hipStream_t)stream), "norm launch");
}

fo_status fo_norm_add_backward(int32_t dtype, int64_t M, int64_t N, const void* dy, int64_t lddy, const void* dh,
                               int64_t lddh, const void* h, int64_t ldh, const void* gamma, const float* rstd, void* dx,
                               int64_t lddx, float* dgamma, void* workspace, int64_t workspace_bytes, void* stream) {
    fo::clear_error();
    fo_status st;
    if (!fo::is_dtype(dtype)) return fo::fail(FO_ERR_ARG, "bad dtype");
    if (M < 0 || N < 0) return fo::fail(FO_ERR_ARG, "negative size");
    if (N > fo::kMaxNormCols) return fo::fail(FO_ERR_UNSUPPORTED, "rows of more than 32768 columns");
    if (!dx && !dgamma) return fo::fail(FO_ERR_ARG, "no gradient asked for");
    if (!fo::aligned(dgamma, 4)) return fo::fail(FO_ERR_ARG, "dgamma must be 4-byte aligned");
    if (N == 0) return FO_OK;
    if (M > INT32_MAX) return fo::fail(FO_ERR_SHAPE, "2^31 rows or more");
    if (M > 0) {
        if ((st = fo::check_rows("dy", dy, N, lddy)) != FO_OK || (dh && (st = fo::check_rows("dh", dh, N, lddh)) != FO_OK) ||
            (st = fo::check_rows("h", h, N, ldh)) != FO_OK || (dx && (st = fo::check_rows("dx", dx, N, lddx)) != FO_OK))
            return st;
        if (!fo::aligned(gamma, 2)) return fo::fail(FO_ERR_ARG, "gamma must be 2-byte aligned");
        if (!rstd || !fo::aligned(rstd, 4)) return fo::fail(FO_ERR_ARG, "rstd is missing or not 4-byte aligned");
        if (fo::clash(dx, M, lddx, dy, M, lddy, N, true) || fo::clash(dx, M, lddx, dh, M, lddh, N, true) ||
            fo::clash(dx, M, lddx, h, M, ldh, N, true))
            return fo::fail(FO_ERR_ARG, "dx overlaps dy, dh or h without being it");
        const int64_t need = dgamma || fo::norm_dots_bytes(M, N) > 0 ? fo_norm_workspace_bytes(M, N) : 0;
        if (need > 0 && (!workspace || !fo::aligned(workspace, 16) || workspace_bytes < need))
            return fo::fail(FO_ERR_ARG, "workspace: fo_norm_workspace_bytes(M, N) bytes, 16-byte aligned");
        const fo::Piece read[] = {{dy, fo::extent(M, N, lddy, 2)}, {dx ? dh : nullptr, fo::extent(M, N, lddh, 2)},
                                  {h, fo::extent(M, N, ldh, 2)}, {gamma, 2 * N}, {rstd, 4 * M}};
        const fo::Piece into = {dx, fo::extent(M, N, lddx, 2)}, sums = {dgamma, 4 * N}, space = {workspace, need};
        const fo::Piece beside[] = {{gamma, 2 * N}, {rstd, 4 * M}, sums, space};        // (the matrices: above)
        if (fo::overlaps(into, beside)) return fo::fail(FO_ERR_ARG, "dx overlaps gamma, rstd, dgamma or the workspace");
        if (fo::overlaps(sums, read) || fo::overlap(dgamma, sums.bytes, workspace, need))
            return fo::fail(FO_ERR_ARG, "dgamma overlaps an input or the workspace");
        if (fo::overlaps(space, read)) return fo::fail(FO_ERR_ARG, "the workspace overlaps an input");
    }
    fo::NormAddArgs a{};
    a.dy = static_cast<const uint16_t*>(dy);
    a.dh = static_cast<const uint16_t*>(dh);
    a.h = static_cast<const uint16_t*>(h);
    a.gamma = static_cast<const uint16_t*>(gamma);
    a.rstd = rstd;
    a.dx = static_cast<uint16_t*>(dx);
    a.partial = dgamma ? static_cast<float*>(workspace) : nullptr;
    if (fo::norm_dots_bytes(M, N) > 0)
        a.dots = reinterpret_cast<float*>(static_cast<char*>(workspace) + fo_norm_workspace_bytes(M, N) - fo::norm_dots_bytes(M, N));
    a.M = M; a.N = N; a.lddy = lddy; a.lddh = lddh; a.ldh = ldh; a.lddx = lddx;
    return fo::done(fo::launch_norm_add_backward(dtype, a, dgamma, (hipStream_t)stream), "norm backward launch");
}

int64_t fo_int8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    return M < 0 || N < 0 || K < 0 || M > INT32_MAX || N > INT32_MAX || K > fo::kMaxInt8Inner ? 0 : fo::int8_workspace_bytes(M, N, K);
}

fo_status fo_int8_product(int32_t dtype, int64_t M, int64_t N, int64_t K, const void* a, int64_t lda, const float* a_scales,
                          const void* b, int64_t ldb, const float* b_scales, const void* bias, void* c, int64_t ldc,
                          void* workspace, int64_t workspace_bytes, void* stream) {
    fo::clear_error();
    fo_status st;
    if ((st = fo::check_product(dtype, M, N, K)) != FO_OK) return st;
    if (M == 0 || N == 0) return FO_OK;
    if ((st = fo::check_operands(a, a_scales, lda, b, b_scales, ldb, bias, c, ldc, N, K)) != FO_OK) return st;
    const int64_t need = fo_int8_workspace_bytes(M, N, K);
    if (need > 0 && (!workspace || !fo::aligned(workspace, 16) || workspace_bytes < need))
        return fo::fail(FO_ERR_ARG, "workspace: fo_int8_workspace_bytes(M, N, K) bytes, 16-byte aligned");
    const fo::Piece out = {c, fo::extent(M, N, ldc, 2)}, space = {workspace, need};
    const fo::Piece others[] = {{a, fo::codes_extent(M, K, lda)}, {b, fo::codes_extent(N, K, ldb)}, {a_scales, 4 * M},
                                {b_scales, 4 * N}, {bias, 2 * N}};
    if (fo::overlaps(out, others)) return fo::fail(FO_ERR_ARG, "c overlaps an operand");
    if (fo::overlaps(space, others) || fo::overlap(c, out.bytes, workspace, need))
        return fo::fail(FO_ERR_ARG, "the workspace overlaps another argument");
    fo::Int8Args p{};
    p.a = static_cast<const int8_t*>(a);
    p.a_scales = a_scales;
    p.b = static_cast<const int8_t*>(b);
    p.b_scales = b_scales;
    p.bias = static_cast<const uint16_t*>(bias);
    p.c = static_cast<uint16_t*>(c);
    p.partial = static_cast<int32_t*>(workspace);
    p.M = M; p.N = N; p.K = K; p.lda = lda; p.ldb = ldb; p.ldc = ldc;
    if (!fo::int8_launchable(p, false)) return fo::fail(FO_ERR_SHAPE, "too many rows and columns for one launch");
    return fo::done(fo::launch_int8_product(dtype, p, (hipStream_t)stream), "product launch");
}

fo_status fo_int8_experts(int32_t dtype, int64_t capacity, int64_t N, int64_t K, int32_t E, const void* a, int64_t a_rows,
                          int64_t lda, const float* a_scales, const int32_t* pair_of, int32_t choices, const void* b,
                          int64_t ldb, const float* b_scales, const void* bias, const int32_t* offsets, const int32_t* counts,
                          void* c, int64_t ldc, void* stream) {
    fo::clear_error();
    fo_status st;
    if ((st = fo::check_product(dtype, capacity, N, K)) != FO_OK) return st;
    if (a_rows < 0) return fo::fail(FO_ERR_ARG, "negative size");
    if (E < 1 || E > FO_ROUTE_MAX_EXPERTS) return fo::fail(FO_ERR_ARG, "E must be in [1, 1024]");
    if (pair_of && (choices < 1 || choices > FO_ROUTE_MAX_CHOICES)) return fo::fail(FO_ERR_ARG, "choices must be in [1, 64]");
    if (capacity == 0 || N == 0 || a_rows == 0) return FO_OK;
    if (!offsets || !counts) return fo::fail(FO_ERR_ARG, "offsets or counts is NULL");
    if (!fo::aligned(offsets, 4) || !fo::aligned(counts, 4) || !fo::aligned(pair_of, 4))
        return fo::fail(FO_ERR_ARG, "offsets, counts and pair_of must be 4-byte aligned");
    if ((st = fo::check_operands(a, a_scales, lda, b, b_scales, ldb, bias, c, ldc, N, K)) != FO_OK) return st;
    if (a_rows > INT32_MAX || E * N > INT32_MAX) return fo::fail(FO_ERR_SHAPE, "2^31 rows or more");
    if (pair_of && K > 0 && fo::codes_extent(a_rows, K, lda) > (int64_t)1 << 31)
        return fo::fail(FO_ERR_SHAPE, "rows taken through pair_of from more than 2^31 bytes");
    const fo::Piece out = {c, fo::extent(capacity, N, ldc, 2)};
    const fo::Piece others[] = {{a, fo::codes_extent(a_rows, K, lda)}, {b, fo::codes_extent(E * N, K, ldb)}, {a_scales, 4 * a_rows},
                                {b_scales, 4 * E * N}, {bias, 2 * E * N}, {pair_of, 4 * capacity}, {offsets, 4 * (E + 1)},
                                {counts, 4 * E}};
    if (fo::overlaps(out, others)) return fo::fail(FO_ERR_ARG, "c overlaps an operand");
    fo::Int8Args p{};
    p.a = static_cast<const int8_t*>(a);
    p.a_scales = a_scales;
    p.b = static_cast<const int8_t*>(b);
    p.b_scales = b_scales;
    p.bias = static_cast<const uint16_t*>(bias);
    p.c = static_cast<uint16_t*>(c);
    p.M = capacity; p.N = N; p.K = K; p.lda = lda; p.ldb = ldb; p.ldc = ldc;
    p.offsets = offsets;
    p.counts = counts;
    p.pair_of = pair_of;
    p.a_rows = a_rows;
    p.E = E; p.choices = choices; p.capacity = (int32_t)capacity;
    if (!fo::int8_launchable(p, true)) return fo::fail(FO_ERR_SHAPE, "too many rows and columns for one launch");
    return fo::done(fo::launch_int8_experts(dtype, p, (hipStream_t)stream), "experts launch");
}

}  // extern "C"
