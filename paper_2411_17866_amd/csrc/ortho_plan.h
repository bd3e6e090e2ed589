// The rules by which the orthogonalisation (ortho.hip) picks its kernels, from sizes
// alone; host code without HIP.
#pragma once

#include <stdint.h>

namespace dsm {

// ---- Small matrices: the whole iteration in one work-group's LDS ----

constexpr int kSmallLds = 144 << 10;
constexpr int kSmallWaves = 8;
constexpr int kSmallSquare = 5;   // fragments of A that a wave has, at most (96 x 96)
constexpr int kSmallWide = 18;    // fragments of X

// It has to fit, and to be little: a wave's products of 16 x 16 x 32 in an iteration
// take it about 0.2 us each here, five iterations 12 us + 1 us each: 64 x 64, 12 of
// them, 30 us (68 us by the products' kernels); 128 x 128, 96, 107 us (70-85 us).
inline bool is_small(int m, int n) {
    const int64_t mp = (m + 31) / 32 * 32, np = (n + 31) / 32 * 32, mi = mp / 16;
    const int64_t products = mi * mi * (np / 32 + mp / 32) + mi * (np / 16) * (mp / 32);
    return mp * (mp + np) * 4 <= kSmallLds && mi * mi <= kSmallSquare * kSmallWaves &&
           mi * (np / 16) <= kSmallWide * kSmallWaves && products <= 50 * kSmallWaves;
}

// ---- The others: tiles of the products ----

// Work-groups of a product of `count` m x n matrices by tiles of bm.
inline unsigned ortho_groups(int count, int m, int n, int bm, bool symmetric) {
    const unsigned ti = (m + bm - 1) / bm, tj = (n + bm - 1) / bm;
    return (symmetric ? ti * (ti + 1) / 2 : ti * tj) * count;
}

// The tile a product takes: the one whose turns over the CUs take least.  A CU
// holds one work-group of 256, two of 128 or of 64; a turn of 128 takes 0.62, of 64
// 0.40 (0.28 where a CU has one of them) of what a turn of 256 does, measured over
// batches from 1 x 64 x 64 to 8 x 1600 x 6400.  One 512 x 1536 fp32 matrix: A in
// 18 us by 36 tiles of 64, 41 us by 10 of 128; twelve of 768 x 2304: 68, 63 and
// 124 us by 936, 252 and 72 tiles of 64, 128 and 256.
inline int ortho_tile(int count, int m, int n, bool symmetric) {
    const auto turns = [](unsigned groups, unsigned slots) { return (groups + slots - 1) / slots; };
    const unsigned small = ortho_groups(count, m, n, 64, symmetric);
    const float t64 = small <= 256 ? 0.28f : 0.40f * turns(small, 512);
    const float t128 = 0.62f * turns(ortho_groups(count, m, n, 128, symmetric), 512);
    const float t256 = 1.0f * turns(ortho_groups(count, m, n, 256, symmetric), 256);
    return t64 <= t128 && t64 <= t256 ? 64 : t128 <= t256 ? 128 : 256;
}

}  // namespace dsm
