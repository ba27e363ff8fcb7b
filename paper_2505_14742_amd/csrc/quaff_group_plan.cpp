// Choice of the tile, and of the workgroups that share a contraction, for the rows products (quaff_group_gemm.h).  Host code only.
#include "quaff_internal.h"

namespace quaff {

namespace {

// What a launch of one tile shape takes, fitted to launches of 64 to 2048 tiles at two contraction lengths: microseconds per stage of the
// contraction while every compute unit has at most one workgroup, while all fit at once (`slots`), and per round beyond that, and what comes on top
// (launch, first operands, results; a round's results).  4-bit at 4096 / 16384: 64 x 64 0.55 / 1.1 / 1.05 us a stage of 256 values,
// 128 x 128 0.80 / 1.2 / 1.2, 256 x 256 1.9; bf16 at 2048 / 4096: 0.62 / 0.71 / 0.72 a stage of 64, 0.50 (plain B) or 0.76 / 0.95 / 0.95, 1.5.
struct Shape { int tile, slots; double one, all, round, fixed, fixed_round; };
constexpr Shape kMx4Shapes[] = {{64, 1024, 0.55, 1.10, 1.05, 2, 5.5}, {128, 512, 0.80, 1.20, 1.20, 4, 8}, {256, 256, 1.90, 1.90, 1.85, 12, 12}};
constexpr Shape kNkShapes[] = {{64, 1024, 0.62, 0.71, 0.72, 2, 6}, {128, 512, 0.50, 0.95, 0.95, 6, 8}, {256, 256, 1.50, 1.50, 1.48, 11, 12}};
constexpr Shape kKnShapes[] = {{64, 1024, 0.66, 0.71, 0.74, 2, 6}, {128, 512, 0.76, 0.92, 0.95, 7, 8}, {256, 256, 1.60, 1.60, 1.55, 9, 12}};

double shape_time(const Shape& s, double tiles, double stages) {
    // few large tiles have the caches to themselves
    if (s.tile == 256 && tiles <= 256) return stages * s.one * (tiles <= 64 ? 0.5 : tiles <= 128 ? 0.75 : 1.0) + s.fixed;
    if (tiles <= 256) return stages * s.one + s.fixed;
    if (s.tile == 64 && tiles <= 512) return stages * s.one + s.fixed;
    if (tiles <= s.slots) return stages * s.all + s.fixed + 3;
    // rounds: tiles are dealt out as units get free, so a part of a round costs less than a whole one
    const double exact = tiles / s.slots;
    const int64_t whole = (int64_t)exact;
    const double rounds = 0.5 * (exact + (double)(exact > (double)whole ? whole + 1 : whole));
    return rounds * (stages * s.round + s.fixed_round);
}

}  // namespace

GroupPlan group_rows_plan(int kind, int64_t t, int64_t N, int64_t K, int32_t n_groups) {
    const int64_t groups = n_groups > 0 ? n_groups : 1;
    GroupPlan best{16, 1};
    // Few rows per group (quaff_group_few.h).  With a plain B its workgroups, 16 columns each, become too many where many groups have rows: 2048 -> 1408, 64
    // groups, 4-bit, 24 rows 14.9 us and 64 x 64 tiles 15.2, 150 rows 31.6 and 21.4; bf16 input gradient 24 rows 25.5 and 27.5, 700 rows 98 and 70.  [K x N] takes
    // 64 columns: forward 24 rows 24 and 32, 700 rows 76 and 83, 1024 -> 4096 200 rows in 100 groups 99 and 117; but its wavefronts share the contraction, which has to be long (512 -> 512, 600 rows in
    // 128 groups: 15.4 and 13.3; 64 -> 3776, 586 in 243: 109 and 67).
    const double rows = (double)t / 16 + (n_groups > 0 ? 0.5 * (double)(groups < t ? groups : t) : 0.5);
    const double few = rows * (double)(kind == kGroupKN ? (N + 63) / 64 : N / 16);
    if (t <= 16 * groups && (kind == kGroupKN ? K >= 1024 || few <= 512 : few <= 2400)) return best;
    const Shape* shapes = kind == kGroupMx4 ? kMx4Shapes : kind == kGroupNK ? kNkShapes : kKnShapes;
    const int64_t stages = kind == kGroupMx4 ? (K + 255) / 256 : (K + 63) / 64;
    double least = 0;
    for (int i = 0; i < 3; ++i) {
        const Shape& s = shapes[i];
        // half a tile of every group is expected to be empty
        const double rows = n_groups > 0 ? (double)t / s.tile + 0.5 * (double)(groups < t ? groups : t) : (double)((t + s.tile - 1) / s.tile);
        const double tiles = rows * (double)((N + s.tile - 1) / s.tile);
        for (int64_t parts = 1; parts <= (s.tile == 256 ? 1 : 8); ++parts) {
            if (parts > 1 && stages / parts < 4) break;
            const int64_t per = (stages + parts - 1) / parts;
            if ((stages + per - 1) / per != parts) continue;                    // (no part is empty)
            double us = shape_time(s, tiles * (double)parts, (double)per);
            // partial results: written and read, and a launch
            if (parts > 1) us += 5 + (double)parts * (double)t * (double)N * 8 / 3e6;
            if (least == 0 || us < least) {
                least = us;
                best = GroupPlan{s.tile, (int32_t)parts};
            }
        }
    }
    return best;
}

size_t group_rows_partial_bytes(int kind, int64_t t, int64_t N, int64_t K, int32_t n_groups) {
    const int64_t parts = group_rows_plan(kind, t, N, K, n_groups).parts;
    return parts > 1 ? (size_t)parts * t * N * sizeof(float) : 0;
}

// Tile of the weight gradients: 128 x 128, narrow results in one tile of their width, 256 x 256 where that is a workgroup per compute unit and the groups have
// rows enough (2048 x 5632, 16 groups: 128 rows in each 231 us with the small tile, 195 with the large; 512 rows 352 and 303).
void group_ragged_tile(int64_t t, int64_t M, int64_t N, int32_t n_groups, int* bm, int* bn) {
    *bm = *bn = 128;
    if (N <= 64) *bn = N <= 32 ? 32 : 64;
    else if (M <= 64) *bm = M <= 32 ? 32 : 64;
    else if (group_slab_rows(t, M, N, n_groups) == 0 && t >= 64 * (int64_t)n_groups && ((M + 255) / 256) * ((N + 255) / 256) * n_groups >= 256)
        *bm = *bn = 256;
}

// Slabs of rows where the tiles alone are too few workgroups, or one busy group would keep a few of them for long.  Small results (an
// adapter's factor) can afford three workgroups per compute unit, for larger ones the partial results cost more than that gives.
int32_t group_slab_rows(int64_t t, int64_t M, int64_t N, int32_t n_groups) {
    const int64_t bm = M <= 64 && N > 64 ? (M <= 32 ? 32 : 64) : 128, bn = N <= 32 ? 32 : N <= 64 ? 64 : 128;
    const int64_t tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn), want = M * N <= 131072 ? 768 : 320;
    int64_t slab = (t * tiles / want + 63) / 64 * 64;
    if (slab < 256) slab = 256;
    return slab * n_groups >= 4 * t || slab >= t ? 0 : (int32_t)slab;
}

size_t group_partial_bytes(int64_t t, int64_t M, int64_t N, int32_t n_groups) {
    const int64_t slab = group_slab_rows(t, M, N, n_groups);
    return slab ? (size_t)(t / slab + (n_groups < t ? n_groups : t)) * M * N * sizeof(float) : 0;
}

}  // namespace quaff
