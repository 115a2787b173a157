// Device side that the kernels of the 8-bit layer share: which expert a row or a tile of rows belongs to.
#pragma once
#include "svdq.h"
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

// Numbers the tiles of a grouped product whose tiles have bm rows.  Every wave does so alone, a lane for every 64th part of the experts (up to
// sixteen), from one reading of the offsets that then stay in registers: no LDS, no barrier, and no memory access when a tile is looked up.
struct GroupScan {
    static constexpr int MOST = SVDQ_MAX_EXPERTS / 64;
    int at[MOST + 1];                // offsets of the lane's experts, as their running maximum
    int first, total;                // row tiles in front of the lane's; all of them
    int per, bm, e0;

    __device__ __forceinline__ GroupScan(const Groups& g, const int M, const int bm_, const int lane) : per((g.E + 63) >> 6), bm(bm_), e0(lane * ((g.E + 63) >> 6)) {
        int top = 0;
#pragma unroll
        for (int j = 0; j <= MOST; ++j)
            if (j <= per) {
                const int o = g.offsets[e0 + j < g.E ? e0 + j : g.E];
                at[j] = o < 0 ? 0 : o > M ? M : o;
            }
#pragma unroll
        for (int j = 0; j < MOST; ++j)
            if (j < per && at[j] > top) top = at[j];
        int before = top;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(before, d);
            if (lane >= d && o > before) before = o;
        }
        before = __shfl_up(before, 1);
        if (lane == 0) before = 0;
        int mine = 0;
#pragma unroll
        for (int j = 0; j <= MOST; ++j)
            if (j <= per) {
                at[j] = at[j] > before ? at[j] : before;
                if (j > 0) mine += (at[j] - before + bm - 1) / bm;    // (experts past the last have no rows)
                before = at[j];
            }
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        first = upto - mine;
        total = __builtin_amdgcn_readlane(upto, 63);
    }

    // Tile `id`: false where there are fewer.  Tiles are numbered expert by expert, within one in groups of eight row tiles across the channel
    // tiles; XCD id % 8 takes a run of them (its L2 then holds few experts' weights).
    __device__ __forceinline__ bool tile(const int id, const int ntiles, GroupTile& t) const {
        const int chunk = (total * ntiles + 7) >> 3, n = (id & 7) * chunk + (id >> 3);
        if ((id >> 3) >= chunk || n >= total * ntiles) return false;
        const int owner = 63 - __builtin_clzll(__ballot(first * ntiles <= n));
        int k = first, e = 0, row0 = 0, row_end = 0, k_e = 0, tiles_e = 1;
#pragma unroll
        for (int j = 0; j < MOST; ++j)
            if (j < per) {
                const int tiles = (at[j + 1] - at[j] + bm - 1) / bm;
                if (k * ntiles <= n && n < (k + tiles) * ntiles) e = e0 + j, row0 = at[j], row_end = at[j + 1], k_e = k, tiles_e = tiles;
                k += tiles;
            }
        t.e = __builtin_amdgcn_readlane(e, owner);
        t.row0 = __builtin_amdgcn_readlane(row0, owner);
        t.row_end = __builtin_amdgcn_readlane(row_end, owner);
        const int local = n - __builtin_amdgcn_readlane(k_e, owner) * ntiles, mtiles = __builtin_amdgcn_readlane(tiles_e, owner);
        const int sm = local / (8 * ntiles), rem = local - sm * (8 * ntiles);
        const int width = mtiles - 8 * sm < 8 ? mtiles - 8 * sm : 8;
        t.nt = rem / width;
        t.mt = 8 * sm + rem - t.nt * width;
        return true;
    }
};

// Where a block's tile lies, and its expert's weights.
struct TilePlace {
    int m0, m_end, n0;
    const int8_t* qw;
    const float *sw, *bias;
};
template <int BM, int BN>
__device__ __forceinline__ bool tile_place(const GemmInt8& g, const TileGrid& tg, const int id, TilePlace& p) {
    int mt, nt;
    if (!tile_of(tg, id, mt, nt)) return false;
    p = TilePlace{mt * BM, (int)g.M, nt * BN, g.qw, g.sw, g.bias};
    return true;
}
template <int BM, int BN>
__device__ __forceinline__ bool tile_place(const GemmInt8& g, const TileGrid& tg, const GroupScan& scan, const int id, TilePlace& p) {
    GroupTile t;
    if (!scan.tile(id, tg.ntiles, t)) return false;
    p = TilePlace{t.row0 + t.mt * BM, t.row_end, t.nt * BN, g.qw + (int64_t)t.e * g.N * g.K, g.sw + (int64_t)t.e * g.N, g.bias ? g.bias + (int64_t)t.e * g.N : nullptr};
    return true;
}

// As many blocks as there can be tiles: every expert with rows adds at most one row tile that is not full.
inline int grouped_blocks(const GemmInt8& g, const int bm, const int bn) {
    const int64_t mt = g.M / bm + (g.M < g.groups.E ? g.M : g.groups.E);
    return (int)((mt * ((g.N + bn - 1) / bn) + 7) / 8 * 8);
}

}  // namespace svdq
