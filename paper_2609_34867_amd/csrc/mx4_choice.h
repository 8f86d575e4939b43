// Which kernel takes an MXFP4 product (mx4_gemm.hip): plain arithmetic.
//
// Each kernel's time is estimated and the least taken.  What decides is how the
// tiles fall into rounds and what a tile loads: one of 256 x 256 needs half of what
// four of 128 x 128 load, and the last round may leave most CUs idle.  The numbers
// are fitted to measurements on 256 CUs at M = 48 .. 11264 and (N, K) from (4096, 4096)
// to (15360, 5120) and gated (13824, 5120); they rank the kernels and are no forecast of
// a call's time, where k is short least of all.  Every kernel timed at 24 .. 11264 rows of
// the widths 1280 to 5120 (483 sizes): the one taken is within 3% of the best at 93% of
// them, and at worst 29% behind it, in small linear products (256 x 2048 x 2048 7.2 us by
// 64 x 64 tiles, 5.6 as few rows).
// For example N = 12288, K = 4096: 64 rows 10.8 us by 64 x 64 tiles (13.1 as few rows,
// 14.3 by 128 x 128); 384 rows 18.0 by 128 x 192 (20.6 by 128 x 128); 704 rows 24.8 by
// 192 x 192 (31.9 by 128 x 128); 4096 rows 104 by 256 x 256 (125 by 128 x 128).
#pragma once

#include <stdint.h>

namespace p4q {

struct Mx4TileCost {
    double idle, busy;                           // us a stage, of the first tile on the device and with every CU at work
    double epilogue;                             // us a round
    int per_cu;                                  // work-groups
    int parts = 1;                               // that share k
};
inline double mx4_tile_cost(int M, int N, int K, int bm, int bn, const Mx4TileCost &c, int cus) {
    const int64_t tiles = (((int64_t)M + bm - 1) / bm) * (((int64_t)N + bn - 1) / bn);
    const int64_t slots = (int64_t)cus * c.per_cu, whole = tiles / slots;
    const int stages = ((K / 32 + 7) / 8 + c.parts - 1) / c.parts;
    double us = 2.5 + (double)whole * (c.epilogue + stages * c.busy);
    if (const int64_t left = tiles % slots) {
        // two on a CU take nearly twice as long as one, whether or not every CU has two
        const bool paired = left > cus;
        us += c.epilogue + stages * (paired ? c.busy - 0.2 * (double)(slots - left) / cus
                                            : c.idle + (c.busy / c.per_cu - c.idle) * (double)left / cus);
    }
    return us;
}

// few rows: what its work-groups load, 15 MB a microsecond
inline double mx4_rows_cost(int M, int N, int K, int mb, int frags, int outputs) {
    const double groups = ((N + outputs - 1) / outputs) * (double)((M + 16 * mb - 1) / (16 * mb));
    return 3.5 + groups * ((K / 32 + 7) / 8) * (frags + mb) * 2176.0 / 15e6;
}

// what becomes of the sums
enum Epilogue { kLinear, kGated, kGatedQuant };

// few rows at a time, or tiles of rows by rows of the weight (gated: half as many outputs);
// Parts: two parts of a work-group share k
enum Mx4Kernel {
    kRows16,
    kRows32,
    kTile64x64,
    kTile64x64Parts,
    kTile64x128,
    kTile64x128Parts,
    kTile128x128,
    kTile128x192,
    kTile192x192,
    kTile192x256,
    kTile256x256
};

inline Mx4Kernel mx4_kernel(Epilogue form, int M, int N, int K, int cus) {
    if (M <= 16) return kRows16;
    const bool linear = form == kLinear;
    const int W = linear ? 64 : 32;                        // outputs of 64 weight rows
    const int NO = form == kGatedQuant ? 32 : 16, F = linear ? 1 : form == kGated ? 2 : 4;
    double least = M <= 1024 ? mx4_rows_cost(M, N, K, 2, F, NO) : 1e30;
    Mx4Kernel best = kRows32;
    auto offer = [&](Mx4Kernel which, int bm, int bn, const Mx4TileCost &c) {
        const double us = mx4_tile_cost(M, N, K, bm, bn, c, cus);
        if (us < least) least = us, best = which;
    };
    if (linear) {
        offer(kTile64x64, 64, 64, {0.38, 0.42, 1.0, 1});
        offer(kTile64x64Parts, 64, 64, {0.57, 0.70, 2.0, 1, 2});
        offer(kTile64x128Parts, 64, 128, {0.79, 0.86, 1.5, 1, 2});
        offer(kTile64x128, 64, 128, {0.54, 0.95, 1.0, 2});
    } else {
        offer(kTile64x128, 64, 64, {0.5, 0.55, 1.0, 1});
    }
    offer(kTile128x128, 128, 2 * W, {0.55, 1.2, 1.5, 2});
    if (linear) {
        offer(kTile128x192, 128, 192, {0.7, 0.87, 2.3, 1});
        offer(kTile192x192, 192, 192, {0.85, 1.18, 2.8, 1});
    }
    offer(kTile192x256, 192, 4 * W, {1.02, 1.42, linear ? 2.2 : 2.7, 1});
    offer(kTile256x256, 256, 4 * W, {1.18, 1.73, 4.0, 1});
    return best;
}

// Wavefronts of a few-rows work-group: two where there are two work-groups for each CU or
// more, else four.  Linear, 32 rows at N = 12288, K = 4096 (768 work-groups) 7.4 against
// 9.8 us, one row at N = 5120, K = 13824 (320) 11.5 against 8.5; gated, 16 rows at N =
// 11008, K = 4096 (688) 9.7 against 12.1.  Gated and quantized, whose four take 100 KB of
// LDS, two would be the better at N = 11008, K = 4096 (344) too: 10.4 against 11.9.
inline int mx4_rows_waves(int64_t groups, int cus) { return groups >= 2 * cus ? 2 : 4; }

}  // namespace p4q
