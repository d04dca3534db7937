// Which kernel of the projection a call gets.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "qlinear_internal.h"

namespace qconv {

// The kernels, and a model of their times (us), its constants measured.  A workgroup
// of the few-row kernel takes `start` and `step` for each 1024 channels in its turn on
// a CU; a tile takes `steps[n]` for a step of 128 channels (of each of its groups of
// waves) with n + 1 on a CU, where `resident` fit.  E.g. 4-bit weights of 2048 channels,
// 4096 outputs: 16 rows 3.6 (16 channels and rows a workgroup; a tile of 64 with two
// groups 7.1); 64 rows 5.3 (32 x 32; tile 7.3); 160 rows 7.6 (tile of 64, two groups; with
// one 9.6, four 8.1, few-row kernel 11.8); 2048 rows 24 (tile of 128; of 64 33, of 256 38).
// Of 8192 channels, 256 rows: 19.5 (tile of 64, four groups; two 21.6, one 32, tile of
// 128 48).  8-bit, 4096 x 4096, 8192 rows: 119 (tile of 256).
enum class Kind { FEW_1x1, FEW_2x1, FEW_2x2, FEW_2x4, TILE_64x4, TILE_64x2, TILE_64, TILE_128, TILE_256 };

// row_tiles(n): how many tiles of n rows the call has.
template <class RowTiles>
Kind plan_linear(const LinearArgs &a, int w_bits, RowTiles row_tiles) {
    static const struct {
        Kind kind;
        int channels, rows;
        double start, step, adapters;
    } kFew[] = {{Kind::FEW_1x1, 16, 16, 0.9, 0.55, 2.5}, {Kind::FEW_2x1, 32, 16, 0.85, 0.8, 3.0},
                {Kind::FEW_2x2, 32, 32, 1.4, 1.15, 4.0}, {Kind::FEW_2x4, 32, 64, 3.2, 1.95, 6.0}};
    static const struct {
        Kind kind;
        int size, groups, resident;
        double start, steps8[4], steps4[4], adapters;
    } kTiles[] = {{Kind::TILE_64x4, 64, 4, 1, 4.2, {0.85}, {0.95}, 2.0},
                  {Kind::TILE_64x2, 64, 2, 2, 3.4, {0.5, 0.82}, {0.53, 0.89}, 2.0},
                  {Kind::TILE_64, 64, 1, 4, 2.9, {0.38, 0.5, 0.68, 0.82}, {0.44, 0.58, 0.72, 0.88}, 2.0},
                  {Kind::TILE_128, 128, 1, 2, 4.2, {0.7, 1.1}, {0.74, 1.17}, 4.0},
                  {Kind::TILE_256, 256, 1, 1, 6.0, {1.7}, {2.2}, 6.0}};
    const auto on_cu = [&](int64_t channels, int64_t rows) {
        return (((a.k + channels - 1) / channels) * (int64_t)row_tiles((int)rows) + 255) / 256;
    };
    Kind best = Kind::TILE_64;
    double best_us = 0;
    const auto consider = [&](Kind kind, double us) {
        if (best_us == 0 || us < best_us) best = kind, best_us = us;
    };
    for (const auto &f : kFew) {
        // (without adapters tiles of 64 are as fast wherever 64 rows a workgroup could be
        // chosen: never with 8-bit weights, within 1 % with 4-bit ones of 5700 channels)
        if (f.kind == Kind::FEW_2x4 && !a.ad.count) continue;
        consider(f.kind, 1.5 + on_cu(f.channels, f.rows) * (f.start + f.step * (w_bits == 8 ? 1.2 : 1.0) * a.c / 1024.0 +
                                                            (a.ad.count ? f.adapters : 0.0)));
    }
    for (const auto &t : kTiles) {
        const int64_t n = on_cu(t.size, t.size), rest = n % t.resident;
        const double *steps = w_bits == 8 ? t.steps8 : t.steps4;
        const double step = (n / t.resident) * steps[t.resident - 1] + (rest ? steps[rest - 1] : 0.0);
        const int64_t turns = (n + t.resident - 1) / t.resident;
        // each adapter that a tile's rows name is a step of one of its groups: few rows are
        // taken to name any, many to lie in runs of one
        const int64_t most = std::min<int64_t>(a.ad.count, a.m < t.size ? a.m : t.size);
        const int64_t named = a.m <= 256 ? most : std::min(most, (int64_t)a.ad.count * t.size / a.m + 1);
        const double adapters = a.ad.count ? t.adapters + 1.2 * (double)((named + t.groups - 1) / t.groups) : 0.0;
        consider(t.kind, t.start + (a.steps + t.groups - 1) / t.groups * step + turns * adapters);
    }
    return best;
}

// The gradients' kernels, and a model of their times (us; see plan_grad): a workgroup takes
// `start` in its turn on a CU, and step[n] for each 64 of the summed axis with n + 1 on it.
struct GradKind {
    int tile, groups, resident;
    double start, step[4];
};
constexpr GradKind kGradKinds[] = {{256, 1, 1, 10, {1.35}}, {128, 1, 2, 6, {0.83, 1.25}}, {64, 1, 4, 3.7, {0.5, 0.75, 0.95, 1.1}},
                                   {64, 2, 2, 4.3, {0.57, 1.08}}, {64, 4, 1, 5, {1.0}}};
inline double grad_time(const GradKind &k, int64_t workgroups, int64_t steps) {
    const int64_t on_cu = (workgroups + 255) / 256, rest = on_cu % k.resident;
    const double step = (on_cu / k.resident) * k.step[k.resident - 1] + (rest ? k.step[rest - 1] : 0.0);
    const int64_t turns = std::max<int64_t>((on_cu + k.resident - 1) / k.resident, 1);
    return turns * k.start + (steps + k.groups - 1) / k.groups * step;
}

// ------------------------------------------------------------------ experts
//
// How m rows are dealt to the experts is not known on the host: the plans take every
// expert to be as likely as another for each row.

// Experts that have rows, the rows of each of them, and their tiles of `size` rows.
inline int64_t expected_experts(int64_t m, int64_t experts) {
    const double none = std::pow(1.0 - 1.0 / (double)experts, (double)m);
    return std::max<int64_t>((int64_t)((double)experts * (1.0 - none) + 0.5), 1);
}
inline int64_t expected_rows(int64_t m, int64_t experts) {
    const int64_t used = expected_experts(m, experts);
    return (m + used - 1) / used;
}
// (a tile of an expert with more rows than one holds is half empty at the end)
inline int64_t expected_tiles(int64_t m, int64_t experts, int64_t size) {
    const int64_t used = expected_experts(m, experts), rows = expected_rows(m, experts);
    return rows <= size / 2 ? used : used * rows / size + (used + 1) / 2;
}
template <class Tiles>
GradPlan plan_expert_grad(Tiles tiles, int64_t steps) {
    GradPlan best{64, 1, 1, (int)steps, (int)steps};
    double best_us = 0;
    for (const auto &k : kGradKinds) {
        const double us = grad_time(k, (int64_t)tiles(k.tile), steps);
        if (best_us == 0 || us < best_us) best_us = us, best.tile = k.tile, best.groups = k.groups;
    }
    return best;
}

}  // namespace qconv
