// Which kernel and tile a linear with 4-bit weights takes: a rule on sizes only, in plain host C++ with no GPU types, so that it can be evaluated for any size without a GPU.
#pragma once
#include <stdint.h>

// How the rows of A become operands: bf16 as they are; E4M3 widened to bf16 (exact, every product is); or E4M3 against E2M1 in one instruction.
enum { LVX_FP4_A_BF16 = 0, LVX_FP4_A_WIDEN = 1, LVX_FP4_A_NATIVE = 2 };

struct lvx_fp4_plan_t {
    int blocks, groups;  // tiles of 32 * blocks rows and 256 / groups columns, K shared by so many groups of waves; blocks 0: the kernels for few rows
};

// Tiles pay from some product of rows (in blocks of 16) and columns on, later where the rows are few or have to be widened: 64 x 5120 x 5120 15, 14 and 10 us (bf16, widened,
// mixed) against 30, 19 and 19 of the few-row kernels, 64 x 1280 x 1280 6.7, 6.9 and 5.7 against 8.7, 6.5 and 6.5; but 40 x 2568 x 1184 7.0, 7.1 and 5.9 against 6.0,
// 5.3 and 5.3, and 24 x 5120 x 13824 36 and 34 against 34 and 25 (bf16, widened; mixed products are taken where the caller asks for them).
// Of the tiles the one that takes the least time: rounds of one workgroup a compute unit, of a start and a time per step of 128 channels that were measured in one round.  Four
// groups over K have half the columns and half the steps one after the other: where two leave units idle they are faster (64 x 5120 x 13824 54 -> 38 us and, mixed, 35 -> 22).
static inline lvx_fp4_plan_t lvx_fp4_plan(int mode, int M, int N, int K) {
    const int64_t row_blocks = ((int64_t)M + 15) / 16;
    const int64_t from = mode == LVX_FP4_A_WIDEN ? (row_blocks >= 3 ? 15000 : 30000) : row_blocks >= 4 ? 5000 : mode == LVX_FP4_A_NATIVE ? 10000 : 15000;
    if (row_blocks < 2 || row_blocks * N < from) return {0, 0};
    static const struct {
        int blocks, groups;
        double start, step;
    } tiles[3][5] = {{{2, 2, 4.7, .57}, {1, 2, 4.4, .454}, {1, 4, 2.0, .33}},
                     {{3, 2, 5.4, .71}, {2, 2, 4.6, .585}, {1, 2, 4.6, .444}, {2, 4, 2.8, .37}, {1, 4, 2.1, .304}},
                     {{3, 2, 5.2, .41}, {2, 2, 4.6, .356}, {1, 2, 4.5, .278}, {2, 4, 3.5, .204}, {1, 4, 3.1, .171}}};
    const double steps = (double)(((int64_t)K + 127) / 128);
    lvx_fp4_plan_t best = {0, 0};
    double least = 0;
    for (const auto &t : tiles[mode]) {
        if (t.blocks == 0) break;
        const int64_t cols = 256 / t.groups, n = ((N + cols - 1) / cols) * (((int64_t)M + 32 * t.blocks - 1) / (32 * t.blocks));
        const double time = (double)((n + 255) / 256) * (t.start + t.step * steps);
        if (least == 0 || time < least) least = time, best = {t.blocks, t.groups};
    }
    return best;
}

// Tiles reach their rows (96 at most) and columns (128) with 32-bit offsets in bytes: below 2^24 bytes a row these stay below 2^31.
static inline bool lvx_fp4_tiles_reach(int64_t lda, int64_t ldw) { return lda < 1 << 24 && ldw < 1 << 24; }

// The kernel of a call with rows lda and weights ldw bytes apart; further apart, any number of rows goes through the kernels for few.
static inline lvx_fp4_plan_t lvx_fp4_call_plan(int mode, int M, int N, int K, int64_t lda, int64_t ldw) {
    return lvx_fp4_tiles_reach(lda, ldw) ? lvx_fp4_plan(mode, M, N, K) : lvx_fp4_plan_t{0, 0};
}

// Rows that lie in LDS whole, of K values of `bytes` bytes, beside the scales of 16 nb columns.
static inline int64_t lvx_fp4_resident_bytes(int bytes, int M, int K, int nb) { return (int64_t)M * ((int64_t)K * bytes + 16) + 16 * nb * (((K / 32 + 15) & ~15) + 4); }

// Blocks of 16 columns of such a workgroup, 0 where the rows are better loaded as they are multiplied.  Rows have to be long enough to pay for the way to LDS (1 x 1280 x 1280
// 3.9 us against 3.2).  The fewest columns with which all workgroups stay at once, two a compute unit or, where there are few enough, one of all its LDS: one row x 5120 x 5120
// 6.7 us against 8.2, 12 bf16 rows 9.8 (two blocks, one workgroup a unit) against 10.4, 14 8-bit rows x 13824 x 5120 13.0 against 13.7, 12 x 27648 x 5120 22.3 (four blocks)
// against 25.3; but 12 bf16 rows x 13824 x 5120 16.2 in four blocks with a unit's LDS each against 15.0.  Columns for fewer than half the units leave the rows' way bare: 14 8-bit
// rows x 1280 x 5120 6.7 against 5.9.  Where all columns take several rounds anyway, many small workgroups hide each other's starts: 1 x 27648 x 5120 17.8 in single blocks, 19.9
// in four.
static inline int lvx_fp4_resident(int bytes, int M, int N, int K) {
    if (M > 16 || K < 4096) return 0;
    const int64_t all = 160 * 1024, one = ((int64_t)N + 15) / 16, two = ((int64_t)N + 31) / 32;
    const int64_t need = lvx_fp4_resident_bytes(bytes, M, K, 1), need2 = lvx_fp4_resident_bytes(bytes, M, K, 2);
    if (one < 128) return (int64_t)M * K * bytes <= 56 * 1024 && need <= all ? 1 : 0;
    if (one > 1024 && need <= all / 6) return 1;
    if ((one <= 512 && need <= all / 2) || (one <= 256 && need <= all)) return 1;
    if ((two <= 512 && need2 <= all / 2) || (two <= 256 && need2 <= all)) return 2;
    return lvx_fp4_resident_bytes(bytes, M, K, 4) <= all / 2 ? 4 : 0;
}
