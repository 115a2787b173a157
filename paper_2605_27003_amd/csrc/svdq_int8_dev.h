// Device side that the kernels of the 8-bit layer share: which expert a row or a tile of rows belongs to.
#pragma once
#include "svdq_int8.h"
#include "svdq_lds.h"
#include "svdq_tiles.h"

namespace svdq {

constexpr int BK = 128;          // k (and bytes) of a row per stage of a product: one memory line
constexpr float QMAX8 = 127.0f;  // codes are symmetric: -128 is not used

// Expert of a row, or -1 for a row that no expert owns.  The running maximum of the offsets passes `row` where the first
// offset does.  Wave-uniform; all lanes take part.
__device__ __forceinline__ int expert_of_row(const Groups& g, const int64_t row, const int lane) {
    for (int j0 = 0; j0 <= g.E; j0 += 64) {
        const int j = j0 + lane;
        const uint64_t past = __ballot(j <= g.E && g.offsets[j < g.E ? j : g.E] > row);
        if (past) return j0 + __builtin_ctzll(past) - 1;
    }
    return -1;
}

// A tile of rows of one expert and a tile of its channels.
struct GroupTile {
    int e, row0, row_end, mt, nt;    // rows [row0, row_end) are the expert's; the tile is its mt-th by its nt-th
};

// Tile `id` of a grouped grid whose blocks take bm rows: false where there are fewer.  Tiles are numbered expert by expert, within one
// in groups of eight row tiles across the channel tiles; XCD id % 8 takes a run of them (its L2 then holds few experts'
// weights).  Every wave finds it alone, a lane for every 64th part of the experts: two passes over the offsets (their running
// maximum, then the tiles), no LDS, no barrier; about 1 us.
__device__ __forceinline__ bool group_tile(const Groups& g, const int M, const int bm, const int ntiles, const int id, const int lane, GroupTile& t) {
    const int per = (g.E + 63) >> 6, e0 = lane * per;
    auto offset = [&](const int e) {
        const int o = g.offsets[e < g.E ? e : g.E];
        return o < 0 ? 0 : o > M ? M : o;
    };
    int top = 0;                                                      // largest offset up to the lane's first expert's start
    for (int j = 0; j < per; ++j) {
        const int o = offset(e0 + j);
        top = o > top ? o : top;
    }
    int before = top;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(before, d);
        if (lane >= d && o > before) before = o;
    }
    before = __shfl_up(before, 1);
    if (lane == 0) before = 0;
    auto walk = [&](auto&& each) {                                    // the lane's experts: start, end, tiles
        int start = before;
        {
            const int o = offset(e0);
            start = o > start ? o : start;
        }
        for (int j = 0; j < per && e0 + j < g.E; ++j) {
            const int o = offset(e0 + j + 1), end = o > start ? o : start;
            each(e0 + j, start, end, (end - start + bm - 1) / bm);
            start = end;
        }
    };
    int mine = 0;
    walk([&](int, int, int, const int n) { mine += n; });
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    const int total = __builtin_amdgcn_readlane(upto, 63) * ntiles;
    const int chunk = (total + 7) >> 3, n = (id & 7) * chunk + (id >> 3);
    if ((id >> 3) >= chunk || n >= total) return false;
    // row tiles in front of tile n, counted in whole row tiles: its expert is the one whose tiles hold number n
    const int first = upto - mine;
    const uint64_t reach = __ballot(first * ntiles <= n);
    const int owner = 63 - __builtin_clzll(reach);
    int at = first, e = 0, row0 = 0, row_end = 0, at_e = 0, tiles_e = 1;
    walk([&](const int ex, const int s, const int en, const int k) {
        if (at * ntiles <= n && n < (at + k) * ntiles) e = ex, row0 = s, row_end = en, at_e = at, tiles_e = k;
        at += k;
    });
    t.e = __builtin_amdgcn_readlane(e, owner);
    t.row0 = __builtin_amdgcn_readlane(row0, owner);
    t.row_end = __builtin_amdgcn_readlane(row_end, owner);
    const int local = n - __builtin_amdgcn_readlane(at_e, owner) * ntiles, mtiles = __builtin_amdgcn_readlane(tiles_e, owner);
    const int sm = local / (8 * ntiles), rem = local - sm * (8 * ntiles);
    const int width = mtiles - 8 * sm < 8 ? mtiles - 8 * sm : 8;
    t.nt = rem / width;
    t.mt = 8 * sm + rem - t.nt * width;
    return true;
}

// Where a block's tile lies, and its expert's weights.
struct TilePlace {
    int m0, m_end, n0;
    const int8_t* qw;
    const float *sw, *bias;
};
template <int BM, int BN, bool GROUPED>
__device__ __forceinline__ bool tile_place(const GemmInt8& g, const TileGrid& tg, const int id, const int lane, TilePlace& p) {
    int mt, nt;
    p.qw = g.qw;
    p.sw = g.sw;
    p.bias = g.bias;
    if constexpr (GROUPED) {
        GroupTile t;
        if (!group_tile(g.groups, (int)g.M, BM, tg.ntiles, id, lane, t)) return false;
        p.m0 = t.row0 + t.mt * BM;
        p.m_end = t.row_end;
        nt = t.nt;
        p.qw += (int64_t)t.e * g.N * g.K;
        p.sw += (int64_t)t.e * g.N;
        if (p.bias) p.bias += (int64_t)t.e * g.N;
    } else {
        if (!tile_of(tg, id, mt, nt)) return false;
        p.m0 = mt * BM;
        p.m_end = (int)g.M;
    }
    p.n0 = nt * BN;
    return true;
}

// As many blocks as there can be tiles: every expert with rows adds at most one row tile that is not full.
inline int grouped_blocks(const GemmInt8& g, const int bm, const int bn) {
    const int64_t mt = g.M / bm + (g.M < g.groups.E ? g.M : g.groups.E);
    return (int)((mt * ((g.N + bn - 1) / bn) + 7) / 8 * 8);
}

}  // namespace svdq
