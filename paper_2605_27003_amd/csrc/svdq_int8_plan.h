// Which tiles a product of the 8-bit layer takes, and in which order (host only).  All give the same sums, exact integers.
#pragma once
#include <cstdint>

namespace svdq {

enum class Int8Tiles { FEW_16x16, FEW_16x32, FEW_32x16, FEW_32x32, T64x32, T64x64, T64x128, T128x128, T256x128, T256x160, T256x256 };
constexpr int INT8_TILES = 11;
struct Int8TileShape {
    int bm, bn;
    double stage;                // us of a block alone on its CU for 128 k; 0: the few-token kernel
    int per_cu;                  // blocks that fit a CU's LDS
};
// A block's time goes by the bytes that it brings to LDS, about 75 a ns where some come from its XCD's L2 and some from behind it (135 where all
// come from L2, 50 where none do), whatever is in flight; 256 x 256 comes near the matrix pipes' time.
inline Int8TileShape int8_tile_shape(Int8Tiles t) {
    switch (t) {
        case Int8Tiles::FEW_16x16: return {16, 16, 0.0, 2};
        case Int8Tiles::FEW_16x32: return {16, 32, 0.0, 2};
        case Int8Tiles::FEW_32x16: return {32, 16, 0.0, 1};
        case Int8Tiles::FEW_32x32: return {32, 32, 0.0, 1};
        case Int8Tiles::T64x32: return {64, 32, 0.22, 2};
        case Int8Tiles::T64x64: return {64, 64, 0.235, 2};
        case Int8Tiles::T64x128: return {64, 128, 0.31, 2};
        case Int8Tiles::T128x128: return {128, 128, 0.415, 2};
        case Int8Tiles::T256x128: return {256, 128, 0.58, 1};
        case Int8Tiles::T256x160: return {256, 160, 0.84, 1};
        default: return {256, 256, 0.97, 1};
    }
}

struct Int8Plan {
    Int8Tiles tiles;
    double cost;                 // estimate, us; negative: the tiles cannot be numbered in 32 bits
};

// rows: of the call.  experts: 0 where it is not grouped.
// Estimate for one choice: a launch and its first bytes 2, and the longest of
//   rounds     a block's stages and its end, for as many rounds as there are tiles for each of 256 CUs (two blocks that share a CU take 1.75 times as
//              long as one)
//   fabric     what the XCDs' L2s fetch at 9 TB/s: 256 tiles at a time, each XCD the rows and channels of its share of them
//   memory     weights and codes at 5.5 TB/s, outputs at 4.4 where their rows are whole memory lines and at 3.3 where tiles share lines (8318 x 28896 of
//              binary32 at K = 176: 240 us; 28884 channels: 436)
// and a little of each, which decides where choices share their bound.  A tile that has its CU alone has nothing to overlap its stores with.
// The figures are fitted to 900 calls of 1 to 75600 rows, each timed with every tile (beyond 4000 rows with those of 64 rows and more), before there were kernels that
// fetch whole lines, which the estimate does not know.  On the calls that it was fitted to the choice is 1.9 % slower than the best tile timed in the mean,
// a third at worst; six of them, more than 5000 rows by 10 to 25 channels, take few-token tiles, which were not timed there.
inline Int8Plan int8_cost(Int8Tiles t, int64_t rows, int N, int K, int experts, bool out_f32) {
    const Int8TileShape s = int8_tile_shape(t);
    const int64_t with_rows = experts ? (rows < experts ? rows : experts) : 1, nt = ((int64_t)N + s.bn - 1) / s.bn;
    const int64_t most = experts ? rows / s.bm + with_rows : (rows + s.bm - 1) / s.bm;                // row tiles that there can be
    const double mt = experts ? (double)rows / s.bm + 0.5 * with_rows : (double)most;                 // and that there are, on average
    Int8Plan p{t, -1.0};
    if ((most + 8) * (nt + 8) + 512 >= INT32_MAX) return p;
    const double weights = (double)with_rows * N * K, codes = (double)rows * K, tiles = mt * nt;
    const double across = mt / with_rows < 8 ? (mt / with_rows < 1 ? 1 : mt / with_rows) : 8, share = tiles < 256 ? tiles / 8 : 32;    // an XCD's tiles: row tiles, all
    const double shared = share / across < 1 ? share : across, channels = share / across < 1 ? 1 : share / across;
    double fabric = tiles / share * (shared * s.bm + channels * s.bn) * K;
    if (fabric < weights + codes) fabric = weights + codes;
    fabric /= 9.0e6;
    const int64_t row = (int64_t)N * (out_f32 ? 4 : 2);
    const double outputs = (double)rows * row / (row % 128 ? 3.3e6 : 4.4e6), memory = (weights + codes) / 5.5e6 + outputs;
    // rounds of blocks, in the time of one block alone on its CU
    const double n = tiles / 256.0, whole = experts ? n + 0.375 : (double)(int64_t)(n + 0.999);
    const double rounds = n <= 1.0 ? 1.0 : s.per_cu == 2 ? (n <= 2.0 ? 1.75 : 1.03 * n) : whole;
    double time;
    if (s.stage == 0.0) {
        const double used = experts ? (rows < 2 * experts ? 2.0 : (double)s.bm) : (double)(rows < s.bm ? rows : s.bm);      // rows past the last are in L1 already
        time = (s.per_cu == 2 && n > 1.0 ? n : rounds) * ((used + s.bn) * K / 58.0e3 + 0.7);   // walking blocks share their CU evenly
    } else {
        time = rounds * (((K + 127) / 128) * s.stage + 0.7 + 4.35 * s.bm * s.bn / 65536.0);
    }
    if (s.stage > 0.0 && s.per_cu == 1) time += 0.6 * outputs;
    double most_time = time;
    if (fabric > most_time) most_time = fabric;
    if (memory > most_time) most_time = memory;
    p.cost = 2.0 + most_time + 0.125 * (time + fabric) + 0.15 * memory;
    return p;
}

inline Int8Plan int8_plan(int64_t rows, int N, int K, int experts, bool out_f32) {
    Int8Plan best{Int8Tiles::T256x256, -1.0};
    for (int i = 0; i < INT8_TILES; ++i) {
        const Int8Plan p = int8_cost((Int8Tiles)i, rows, N, K, experts, out_f32);
        if (p.cost >= 0.0 && (best.cost < 0.0 || p.cost < 0.995 * best.cost)) best = p;
    }
    return best;
}

// Row tiles by channel tiles that there can be: every expert with rows adds at most one row tile that is not full.
inline int64_t int8_tiles(int64_t rows, int N, int experts, int bm, int bn) {
    const int64_t mt = experts ? rows / bm + (rows < experts ? rows : experts) : (rows + bm - 1) / bm;
    return mt * (((int64_t)N + bn - 1) / bn);
}

// The kernel for tiles: how many stages ahead it requests, and whether it fetches rows by whole memory lines.
struct Int8Kernel {
    Int8Tiles tiles;
    int depth;
    bool lines;
};
inline Int8Kernel int8_kernel(Int8Tiles t, int64_t rows, int N, int K, int experts) {
    const Int8TileShape s = int8_tile_shape(t);
    const int64_t tiles = int8_tiles(rows, N, experts, s.bm, s.bn);
    // rows fetched by whole lines, a block alone on its CU: where enough blocks share what L2 gives.  (Few wait for latency, and have less under way so:
    // one tile of 128 x 128 takes up to 1.29 times as long, 48 to 256 tiles 0.7 to 1.1 times, 0.94 in the mean of 80 products.)
    const bool lines = K % 128 && tiles > 48 && tiles <= 256;
    switch (t) {
        case Int8Tiles::T64x32:
        case Int8Tiles::T64x64: return {t, 4, false};
        case Int8Tiles::T64x128: return {t, lines ? 4 : 3, lines};
        // a block alone on its CU, or two.  (Up to 48 tiles the estimate takes smaller ones.)
        case Int8Tiles::T128x128: return {t, tiles <= 256 && (lines || K % 128 == 0) ? 4 : 2, lines};
        default: return {t, 2, false};
    }
}

}  // namespace svdq
