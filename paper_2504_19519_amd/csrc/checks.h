// Argument checks that the C entry points of the row and 8-bit operators share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "fo_internal.h"

namespace fo {

inline bool is_dtype(int32_t d) { return d == FO_FP16 || d == FO_BF16; }
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Whether two matrices of 16-bit values, Mp and Mq rows of N, ldp and ldq apart, share
// memory other than by being the same one (where that is allowed).
inline bool clash(const void* p, int64_t Mp, int64_t ldp, const void* q, int64_t Mq, int64_t ldq, int64_t N, bool same_allowed) {
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
inline fo_status check_rows(const char* what, const void* p, int64_t N, int64_t ld) {
    if (!p) return fail(FO_ERR_ARG, std::string(what) + " is NULL");
    if (!aligned(p, 2)) return fail(FO_ERR_ARG, std::string(what) + " must be 2-byte aligned");
    if (ld < N) return fail(FO_ERR_ARG, std::string(what) + ": rows are closer together than their length");
    return FO_OK;
}

// Whether two pieces of memory share some.
inline bool overlap(const void* p, int64_t np, const void* q, int64_t nq) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
    return p && q && np > 0 && nq > 0 && x < y + (uintptr_t)nq && y < x + (uintptr_t)np;
}

// Whether `blocks` workgroups of `threads` fit one launch.
inline bool launchable(int64_t blocks, int64_t threads) { return blocks <= (int64_t)UINT32_MAX / threads; }

inline fo_status done(hipError_t e, const char* what) {
    return e == hipSuccess ? FO_OK : fail(FO_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace fo
