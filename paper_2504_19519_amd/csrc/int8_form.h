// Arguments of the products of 8-bit matrices, and the rules by which the host chooses
// their kernel and blocks (internal).
#pragma once

#include <stdint.h>

#include <algorithm>

#include "fo_internal.h"

namespace fo {

// Bytes of a row of n codes: whole chunks of 16.
FO_HD inline int64_t int8_row_bytes(int64_t n) { return (n + 15) / 16 * 16; }

// c = (a b^T) a_scales b_scales + bias: sums in 32-bit integers, exact.
constexpr int64_t kMaxInt8Inner = 131071;          // 2^14 times as much fits 31 bits
constexpr int64_t kMaxInt8Row = 1 << 22;           // bytes from row to row: a tile's rows within 31 bits
struct Int8Args {
    const int8_t* a;            // rows, lda apart
    const float* a_scales;
    const int8_t* b;            // [N] rows, ldb apart; experts: [E * N]
    const float* b_scales;      // [N]; [E * N]
    const uint16_t* bias;       // [N]; [E * N]; or null
    uint16_t* c;                // rows, ldc apart
    int32_t* partial;           // [parts][M][partial_cols(N)] sums over a part of K each, where it is split
    int64_t M, N, K, lda, ldb, ldc;
    // by experts: expert e's rows of c are offsets[e] .. offsets[e] + counts[e] - 1
    const int32_t* offsets;
    const int32_t* counts;
    const int32_t* pair_of;     // row r is of a's row pair_of[r] / choices; null: a's row r
    int64_t a_rows;
    int32_t E, choices, capacity;
    int32_t parts;              // of K; 1: not split
    int32_t span;               // blocks, side by side, of a workgroup
    int32_t blocks;             // 256 x 256 tiles, of all workgroups
};

// The kernel of a launch: blocks of rows x cols in a ring of `stages`, 256 x 256 tiles, or
// (rows 16) the kernel for few blocks; k in `parts` parts.
struct Int8Form {
    int rows, cols, stages, parts, span;
};

// Nanoseconds of a launch of `tiles` 256 x 256 tiles, one to a compute unit, and of `blocks`
// 128 x 128 blocks, two to a compute unit, of `steps` each; sums of a few steps wait for the
// results' way out. As measured, us in tiles and in blocks: 8192 x 8192 x 8192 393 and 530;
// 8192 x 8192 x 3584 181 and 231; 4096 x 4096 x 4096 54 and 70; 2048 x 4096 x 4096 48 and 34;
// 4768 x 4736 x 4672 109 and 145; 13893 x 15552 x 704 211 and 242; 12162 x 2368 x 2496 72 and 91;
// 11816 x 6080 x 512 68 and 65, x 128 53 and 43; 7596 x 5376 x 192 35 and 29; 3803 x 6976 x 256
// 27 and 22.
inline int64_t tiles_ns(int64_t tiles, int64_t steps) {
    const int64_t rest = tiles % 256, round = std::max(1460 * steps + 4400, 1100 * steps + 9000);
    return 6000 + tiles / 256 * round + (rest == 0 ? 0 : rest <= 128 ? 1250 * steps + 2000 : round);
}
inline int64_t blocks_ns(int64_t blocks, int64_t steps) {
    const int64_t rest = blocks % 512, round = std::max(1030 * steps + 1500, 850 * steps + 3800);
    return blocks / 512 * round + (rest == 0 ? 0 : rest <= 256 ? 700 * steps + 3000 : round);
}

// us, bf16: 1024 x 4096 x 4096 in blocks of 128 with three stages 21, with two 25, of 64 28; 512 x
// 4096 x 4096 of 64 15.8, of 128 25, of 128 x 64 13.8; 333 x 2881 x 1985 of 64 12.0, of 128 x 64
// 10.3; 1024 x 2048 x 7168 26 and 21, but 256 x 4096 x 4096, where those of 64 are one to a compute
// unit, 9.8 and 12.9; 128 x 4096 x 4096 of 32 9.4, of 64 9.5, of 64 x 32 8.7, 64 x 8192 x 1024 5.0,
// 4.9 and 4.6, 256 x 4096 x 4096 15.5, 10.6 and 12.3; 16 x 14336 x 4096 of 32 11.3, of 64 12.0. In
// parts: 16 x 256 x 16384 8.7 for 16.0, 128 x 1024 x 16384 13.1 for 18.5, but 16 x 256 x 4096 6.7 for
// 6.4, 1 x 4096 x 16384 15.8 for 12.0 in the kernel for few blocks.
inline Int8Form product_form(int64_t M, int64_t N, int64_t K) {
    const int64_t steps = (int8_row_bytes(K) + 127) / 128;
    const auto blocks = [&](int64_t size) { return ((M + size - 1) / size) * ((N + size - 1) / size); };
    // (blocks fare worse where rows share lines of 128 bytes: 5000 x 5000 x 1000 44 us in tiles and 52)
    const int64_t shared = int8_row_bytes(K) % 128 != 0 ? 23 : 20;
    if (M > 128 && K > 0 && tiles_ns(blocks(256), steps) < blocks_ns(blocks(128), steps) / 20 * shared) return {256, 256, 2, 1, 1};
    if (M > 40 && blocks(128) > 256) return {128, 128, 2, 1, 1};
    if (M > 40 && blocks(128) >= 144 && steps >= 8) return {128, 128, 3, 1, 1};
    if (M > 64 && blocks(64) > 256) return {128, 64, 3, 1, 1};
    if (M > 32 && blocks(32) > 512) return {64, 64, 4, 1, 1};
    if (M > 32 && blocks(32) > 256) return {64, 32, 4, 1, 1};
    if (blocks(32) <= 128 && steps >= 64 && (M > 4 || blocks(16) <= 128)) return {32, 32, 4, 4, 1};
    if (blocks(16) <= 256) return {16, 16, 0, 1, 1};
    return {32, 32, 4, 1, 1};
}

// By experts, whose rows the host does not know: as if those that can have some had the same
// number. Several blocks to a workgroup where the sums are short: it looks for its expert and
// rows once, and a block's first loads go ahead of the results of the one before it. us, bf16,
// blocks of 128 / 64 / 32 and how many to a workgroup:
//   309 tokens to 8 of 256, 2934 columns  K 128   1: 56 / - / -  2: 45 / 63 / 69  4: 44 / 54 / 53
//                                         K 1024  1: 145         2: 142 / 148 / 161  4: 153 / 145 / 150
//   16 tokens to 8 of 256, 7168 columns   K 2048  1: 200 / 202   2: 191 / 185 / 195  4: 188 / 183 / 189
//                          2048 columns   K 7168  1: 201 / 173 / 177  2: 230 / 179 / 183  4: - / 198 / 189
//   512 tokens to 8 of 64, 2048 columns   K 2048  1: 70 / 79     2: 85 / 77 / 103
//   1217 tokens to 4 of 60, 2881 columns  K 1409  1: 94 / 116    2: 95 / 115 / 154   (in tiles 104)
//   16 tokens to 8 of 256, 2048 columns   K 256   1: 18.8 / 24.7     K 128  1: 16.5 / 23.3
//   3352 tokens to 6 of 256, 64 columns   K 640   1: 11.3 / 9.2
// Tiles or blocks of 128, for experts of which each has more rows or fewer than the average (of
// a tile's rows behind the last whole one, half have a half tile): us, bf16, tiles and blocks:
//   1200 tokens to 8 of 64, 2048 columns  K 7168  280 / 272     1600 tokens  285 / 316
//   2400 tokens to 8 of 64, 7168 columns  K 2048  389 / 449     4096 tokens, K 512  246 / 307
//   900 tokens to 8 of 64, 7168 columns   K 2048  245 / 261     600 tokens   233 / 224
//   4000 tokens to 8 of 256, 7168 columns K 2048  957 / 1089
//   1000 tokens to 2 of 8,  4096 columns  K 4096   61 /  80     2000 tokens  105 / 106
//   8192 tokens to 4 of 60, 2881 columns  K 1409  248 / 285     6000 tokens, 300 columns, K 4000  110 / 83
//   8192 tokens to 1 of 16, 1024 columns  K 1024   23 /  21     1500 to 2 of 16, 1408 columns, K 2048  31 / 19
//   1316 tokens to 8 of 16, 3648 columns  K 151    41 /  35
inline int64_t pairs_of(const Int8Args& a) { return a.pair_of ? std::min<int64_t>(a.capacity, a.a_rows * a.choices) : a.capacity; }
inline Int8Form experts_form(const Int8Args& a) {
    const int64_t pairs = pairs_of(a);
    const int64_t experts = std::min<int64_t>(a.E, pairs), each = (pairs + experts - 1) / experts;
    const int64_t steps = (int8_row_bytes(a.K) + 127) / 128;
    const auto blocks = [&](int64_t size) { return experts * ((each + size - 1) / size) * ((a.N + size - 1) / size); };
    // (the last round of tiles or blocks half full; without pair_of, rows of padding count as well)
    const double tiles = (double)((a.N + 255) / 256) * ((double)pairs / 256 + 0.28 * (double)experts) / 256 + 0.5;
    const double pieces = (double)((a.N + 127) / 128) * ((double)pairs / 128 + 0.5 * (double)experts) / 512 + 0.5;
    const int64_t round = std::max<int64_t>(1460 * steps + 4400, 11000);       // (32 MB of results)
    if (each > (a.pair_of ? 96 : 160) && a.K > 0 && 6000 + tiles * (double)round < pieces * (double)(1030 * steps + 4000))
        return {256, 256, 2, 1, 1};
    if (each > 8 && a.N > 64 && blocks(128) >= 144) return {128, 128, 2, 1, blocks(128) < 2048 || steps > 8 ? 1 : steps > 2 ? 2 : 4};
    if (each <= 8 && a.N > 64 && steps <= 2 && blocks(32) > 2048 && blocks(64) < 6000) return {128, 128, 2, 1, 1};
    if (blocks(32) > 2048 || (each > 8 && blocks(32) > 512)) return {64, 64, 4, 1, blocks(64) < 6000 || steps > 16 ? 1 : 4};
    return {32, 32, 4, 1, 1};
}

// Whether the weights are read once by the call and too large to be found in the caches by the
// next one: their loads then leave the caches alone. Rows that do not begin with a line of 128
// bytes share lines between steps, and need them kept. us, loads kept and not: 16 tokens to 8
// of 256 experts, 2048 x 7168 171 and 157; 16 x 16384 x 16384 64 and 58; but 16 x 14336 x 4096,
// which the caches hold, 11.6 and 15.4; 1217 tokens to 4 of 60, rows of 1424 bytes 95 and 117.
inline bool weights_once(const Int8Args& a, const Int8Form& f, bool experts) {
    if (a.ldb % 128 != 0) return false;
    if (!experts) return a.M <= f.rows && a.N * a.ldb > (int64_t)1 << 27;
    const int64_t pairs = pairs_of(a), some = std::min<int64_t>(a.E, pairs);
    return pairs <= f.rows * some && some * a.N * a.ldb > (int64_t)1 << 27;
}

}  // namespace fo
