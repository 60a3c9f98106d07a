// How the products grouped by expert are cut into workgroups, by sizes and types alone: host code, which knows nothing of what it launches.
#ifndef DEAR_EXPERTS_CUT_H
#define DEAR_EXPERTS_CUT_H

#include <cmath>
#include <cstdint>

#include "dear_ops.h"
#include "ops_sizes.h"

namespace dear_ops {

enum product { LINEAR, INPUT_GRAD, WEIGHT_GRAD };

constexpr int THREADS = 256;  // of a workgroup
constexpr int BB = 128;       // outputs' columns of a workgroup, but of tiles of 256
constexpr int WS = 64;        // summed index of a step
constexpr int CUS = 256;

// How a call's outputs are cut: tiles of 256 (WIDE), tiles of 32 or 128 rows that memory fills directly, with two steps under way (RING32, RING128) or
// with one and two workgroups a CU (FEW128), or tiles whose operands go through registers (ANY32, ANY64, ANY128); and the splits of the
// summed index.
enum cut { WIDE, RING32, RING128, FEW128, ANY32, ANY64, ANY128 };
struct choice {
    cut how;
    int splits;
    double us;
};

// Tiles of 256 that are left behind whole rounds go in quarters up to so many and, but of weight gradients, in tiles of 32 x 128 up to so many.
constexpr int MOST_IN_QUARTERS = CUS / 2, MOST_SMALL = CUS / 16;

// Tiles of n rows that the experts are expected to have: half of each one's last is empty.
inline double row_tiles(const dear_experts_t &x, int n) {
    const double used = (double)(x.experts < x.rows ? x.experts : x.rows), tiles = (double)x.rows / n + used / 2;
    return tiles < used ? used : tiles;
}

// The cut and splits of the least time by this estimate, in microseconds.  A CU takes `resident` workgroups at a time; a step of 64 of the summed
// index takes each `alone` as long as loads are what it waits for, and a `share` of the CU, or of what the caches give it, when there are more;
// all weights take their way from memory, a part of which tiles of 256 and those that begin and end at other times leave unused.  Several
// splits' sums are written, read, eight at a time, and added, 4 TB/s, in another launch.  Tiles of 256 fill the chip once each and are not
// split; their last round goes in smaller ones where it is no more than half full.  Measured, microseconds, over 8 experts, 4096 x 1024, tiles
// of 256, and RING32, RING128 and FEW128: 32 rows 34, 15, 16 and 20, 1024 rows 37, 32, 21 and 25, 2048 rows -, 53, 32 and 39, 4096 rows 36,
// 95, 55 and 50; over 64, 1024 x 1024, 4096 rows 41, 53, 37 and 33.  The input gradient's in one split and four: 32 rows RING32 33 and 19,
// RING128 41 and 20, 1024 rows 40 and 47, 45 and 29, 4096 rows in one, tiles of 256 64 and RING128 54.
inline choice choose(const dear_experts_t &x, bool is_direct, int64_t sum, int64_t columns) {
    const double steps = (double)ceil_div(sum, WS), size = x.dtype == DEAR_F32 ? 4 : 2;
    const double weights = (double)(x.experts < x.rows ? x.experts : x.rows) * (double)sum * (double)columns * size / 5.8e6;
    choice best = {ANY128, 1, 0};
    auto take = [&](cut how, int n, double us, bool at_once) {
        const double least = weights * (how == WIDE ? 1.5 : at_once && how <= RING128 ? 1 : 1.2);
        us = us > least ? us : least;
        us += 4 + (n == 1 ? 0 : 1.5 + 1.5 * (double)ceil_div(n, 8) + (double)(n + 1) * (double)x.rows * (double)columns * 4 / 4e6);
        if (best.us == 0 || us < best.us) best = {how, n, us};
    };
    auto splits = [&](cut how, int ba, double resident, double begin, double alone, double share) {
        const double tiles = row_tiles(x, ba) * (double)ceil_div(columns, BB);
        const int64_t upper = (x.rows / ba + x.experts + 1) * ceil_div(columns, BB);
        for (int64_t n = 1; n <= 32 && (n == 1 || (n * 2 * WS <= sum && upper * n * THREADS <= MAX_THREADS && x.rows * columns <= MAX_THREADS)); ++n) {
            const double a_cu = std::ceil(tiles * n / CUS), each = std::ceil(steps / n);
            const double wait = std::ceil(a_cu / resident) * (begin + each * alone), work = a_cu * each * share;
            take(how, (int)n, wait > work ? wait : work, a_cu <= 1);
        }
    };
    const bool f32 = x.dtype == DEAR_F32;
    if (is_direct) {
        splits(RING32, 32, 2, 1, 0.45, 0.42);
        splits(FEW128, 128, 2, 3, 0.85, 0.6);
        splits(RING128, 128, 1, 1, 0.7, 0.7);
        const double tiles = std::ceil(row_tiles(x, 256)) * (double)ceil_div(columns, 256), rounds = std::floor(tiles / CUS), over = tiles - rounds * CUS;
        take(WIDE, 1, 3 + steps * 1.5 * (rounds + (over > MOST_IN_QUARTERS ? 1 : over > MOST_SMALL ? 0.5 * std::ceil(4 * over / CUS) : over > 0 ? 0.3 : 0)), false);
    } else {
        splits(ANY32, 32, f32 ? 3 : 6, 3, f32 ? 2.6 : 1.4, f32 ? 1.2 : 0.7);
        splits(ANY64, 64, f32 ? 4 : 5, 3, f32 ? 3.2 : 1.4, f32 ? 2.0 : 0.7);
        splits(ANY128, 128, 3, 3, f32 ? 4.6 : 1.4, f32 ? 3.6 : 0.7);
    }
    return best;
}

// Of a weight gradient, by a like estimate, with the rows shared out evenly: tiles of 256 where an expert has more than a few steps, or of 128
// in splits of each expert's rows.  Measured, microseconds, tiles of 256, and of 128 in one, four and sixteen splits: 16384 rows, 4096 x 1024 over
// 8 123, 208, 405 and 1074, 1024 x 1024 over 8 50, 53, 99 and 275; 30000 rows, 1024 x 1024 over 2 146, 255, 102 and 132; 16000 rows, 512 x 512
// of one 140, 269, 73 and 30, 100 x 100 over 4 -, 81, 26 and 13; 500 rows, 4096 x 1024 over 8 33 and 28; fp32 16384 rows, 128 x 64 over 8 -, 157,
// 45 and 18.
inline choice choose_weight_grad(const dear_experts_t &x, bool is_direct) {
    const bool f32 = x.dtype == DEAR_F32;
    const int64_t rows = ceil_div(x.rows, x.experts);
    const double steps = (double)ceil_div(rows, WS), outputs = (double)x.experts * x.outs * x.ins, written = outputs * 4 / 4e6;
    auto tiles = [&](int n) { return (double)x.experts * (double)(ceil_div(x.outs, n) * ceil_div(x.ins, n)); };
    choice best = {ANY128, 1, 0};
    for (int64_t n = 1; n <= 32 && (n == 1 || (n * 2 * WS <= rows && tiles(128) * n * THREADS <= MAX_THREADS && outputs <= MAX_THREADS)); ++n) {
        const double a_cu = std::ceil(tiles(128) * n / CUS), each = std::ceil(steps / n), resident = f32 ? 2 : 3;
        const double wait = std::ceil(a_cu / resident) * (3 + each * (f32 ? 4.6 : 1.3)), work = a_cu * each * (f32 ? 3.6 : 0.7);
        const double us = (wait > work ? wait : work) + (n == 1 ? written : 3 + (2 * n + 1) * written);
        if (n == 1 || us < best.us) best = {ANY128, (int)n, us};
    }
    if (is_direct && rows >= 2 * WS) {
        const double rounds = std::floor(tiles(256) / CUS), over = tiles(256) - rounds * CUS;
        const double us = 3 + steps * 1.5 * (rounds + (over > MOST_IN_QUARTERS ? 1 : 0.45 * std::ceil(4 * over / CUS))) + written / 2;
        if (us <= best.us) best = {WIDE, 1, us};
    }
    return best;
}

template <int KIND> choice choose_cut(const dear_experts_t &x, bool is_direct) {
    if (KIND == WEIGHT_GRAD) return choose_weight_grad(x, is_direct);
    return KIND == LINEAR ? choose(x, is_direct, x.ins, x.outs) : choose(x, is_direct, x.outs, x.ins);
}

}  // namespace dear_ops
#endif
