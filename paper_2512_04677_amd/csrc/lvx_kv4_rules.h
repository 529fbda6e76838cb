// Which form of the attention over the 4-bit cache a call takes: a rule on sizes only, in plain host C++ with no GPU types, so that it can be evaluated for any size
// without a GPU.
#pragma once
#include <stdint.h>

constexpr int LVX_KV4_MAX_SPLITS = 64;   // ranges of keys of a row: the joining wave has a lane for each
constexpr int LVX_KV4_MAX_GROUPS = 512;  // workgroups (ranges counted) up to which keys are split: two a compute unit

struct lvx_kv4_plan_t {
    int rows, row_tiles, splits;  // rows of a workgroup (tokens x heads of a group): 16, 32, 64 or 128; workgroups a sequence and kv head; ranges of keys
};

// The form and the ranges with the least time by the measured time of an iteration (head_dim 128; 64 takes the same constants, unmeasured): a workgroup goes through its range of keys `waves` tiles of 64 at a time,
// in 0.1 us `alone` on its compute unit or `beside` a second one, and 512 of them take `full`.  Few rows to a workgroup fill the chip from fewer rows, many read the keys
// less often: 64 tokens of 40 heads against 1560 keys 9.6 us in blocks of 16 rows, 51 of 128 (a cache of as many places: the rule knows those, not the keys that there
// are, and with 24960 places takes another form, 14.0 us); 1560 tokens against 24960 keys 734 us in 128.  A causal prompt's
// workgroups see fewer keys the earlier their rows: where there are more than stay at once, they cost the average, the longest bounds the others.  Ranges cost the launch
// that joins them, 5 us and the partial outputs' way out and in: one token of 40 heads against 4680 keys 9.3 us in twelve, 18.6 in one; 512 tokens of 8 heads against
// 4096 keys 18.0 in one, 25.9 in two.
static inline lvx_kv4_plan_t lvx_kv4_plan(int n_seqs, int kv_heads, int max_keys, int n_heads, int max_tokens) {
    static const struct {
        int rows, waves;
        double alone, beside, full, start;
    } forms[4] = {{16, 8, 14, 14, 24, 0}, {32, 8, 22, 22, 44, 10}, {64, 2, 13, 22, 22, 0}, {128, 1, 19, 20, 20, 0}};
    static const int ranges[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    const int64_t rows = (int64_t)max_tokens * (n_heads / kv_heads), tiles = ((int64_t)max_keys + 63) / 64;
    const int64_t half = (tiles + 1) / 2, mean = tiles - max_tokens / 128 > half ? tiles - max_tokens / 128 : half;
    lvx_kv4_plan_t best = {16, 1, 1};
    double least = 0;
    for (const auto &f : forms) {
        if (f.rows > 16 && 2 * rows <= f.rows) break;
        const int64_t row_tiles = (rows + f.rows - 1) / f.rows, blocks = row_tiles * kv_heads * n_seqs;
        for (const int splits : ranges) {
            const int64_t groups = blocks * splits;
            if (splits > 1 && (groups > LVX_KV4_MAX_GROUPS || splits > tiles)) break;
            const int64_t range = (tiles + splits - 1) / splits, mean_range = (mean + splits - 1) / splits;
            const double longest = (double)((range + f.waves - 1) / f.waves) * (groups <= 256 ? f.alone : f.beside);
            const double rounds = (double)(groups / 512) * f.full + (groups % 512 > 256 ? f.full : groups % 512 > 0 ? f.alone : 0);
            const double all = rounds * (double)((mean_range + f.waves - 1) / f.waves);
            const double join = splits > 1 ? 50 + (double)rows * kv_heads * n_seqs * splits / 410 : 0;
            const double time = (longest > all ? longest : all) + f.start + join;
            if (least == 0 || time < least) least = time, best = {f.rows, (int)row_tiles, splits};
        }
    }
    return best;
}

// Rows times ranges of any call of up to max_tokens tokens a sequence, a bound that grows with them: splits * rows of a sequence and kv head * kv_heads * n_seqs <= 512 * 128.
static inline uint64_t lvx_kv4_partial_rows(int n_seqs, int max_keys, int n_heads, int max_tokens) {
    const uint64_t tiles = ((uint64_t)max_keys + 63) / 64;
    if (tiles == 1) return 0;
    const uint64_t most = (uint64_t)max_tokens * n_heads * n_seqs * (tiles < LVX_KV4_MAX_SPLITS ? tiles : LVX_KV4_MAX_SPLITS);
    return most < LVX_KV4_MAX_GROUPS * 128 ? most : LVX_KV4_MAX_GROUPS * 128;
}
