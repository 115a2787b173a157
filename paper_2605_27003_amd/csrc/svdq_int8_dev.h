// Device side that the kernels of the 8-bit layer share: which expert a row or a tile of rows belongs to.
#pragma once
#include "svdq.h"
#include "svdq_int8.h"
#include "svdq_int8_plan.h"
#include "svdq_lds.h"

namespace svdq {

constexpr int BK = 128;          // k (and bytes) of a row per stage of a product: one memory line
constexpr float QMAX8 = 127.0f;  // codes are symmetric: -128 is not used

// A row's scale from the bit pattern of its largest magnitude (a NaN's or an infinity's is past every finite one's), and what its values are
// multiplied with; false: codes 0, the scale NaN where the row or its ratio is none, 0 where it would not be a normal number (an infinite one comes of a
// row's own ratio, which nobody checks).
__device__ __forceinline__ bool row_scale(const uint32_t top, const float rho, float& s, float& inv) {
    const bool finite = top < 0x7f800000u;
    s = __fdiv_rn(__fmul_rn(rho, bits_f(top)), QMAX8);
    const bool fine = finite && s >= 1.17549435e-38f && s <= 3.40282347e38f;
    inv = fine ? __fdiv_rn(1.0f, s) : 0.0f;
    if (!fine) s = finite && s == s ? 0.0f : bits_f(0x7fc00000u);
    return fine;
}
// eight codes: clamped first, so that adding 1.5 2^23 rounds to the nearest whole number (ties to even) in the low bits
__device__ __forceinline__ uint2 codes8(const float (&x)[8], const float inv, const bool fine) {
    uint32_t b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = f_bits(__fadd_rn(__builtin_amdgcn_fmed3f(__fmul_rn(x[j], inv), -QMAX8, QMAX8), 12582912.0f));
    uint2 o;
    o.x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
    o.y = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[7], b[6], 0x0c0c0400u), __builtin_amdgcn_perm(b[5], b[4], 0x0c0c0400u), 0x05040100u);
    return fine ? o : uint2{0, 0};
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}

// An output from its exact sum: rounded to binary32, times the token's scale, then one multiplication and addition that round once, in every kernel alike.
__device__ __forceinline__ float output(const int sum, const float sx, const float sw, const float bias) {
    return __builtin_fmaf(__fmul_rn((float)sum, sx), sw, bias);
}

// Number of the first offset past a row, E + 1 if there is none: the row is the expert's before it (the running maximum of the offsets passes
// the row where the first offset does).  Wave-uniform; all lanes take part.
__device__ __forceinline__ int first_offset_past(const Groups& g, const int64_t row, const int lane) {
    for (int j0 = 0; j0 <= g.E; j0 += 256) {                          // four loads under way at a time
        int o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = g.offsets[j0 + 64 * k + lane < g.E ? j0 + 64 * k + lane : g.E];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint64_t past = __ballot(j0 + 64 * k + lane <= g.E && o[k] > row);
            if (past) return j0 + 64 * k + __builtin_ctzll(past);
        }
    }
    return g.E + 1;
}

// How blocks (id, id + 256, ...: XCD id % 8) take the `total` tiles of a product: 256 consecutive ones at a time, an eighth of them, 32, consecutive
// on every XCD (of what is left at the end, too).  -1: none.
__device__ __forceinline__ int tile_number(const int id, const int total) {
    const int base = id & ~255, left = total - base, run = left >= 256 ? 32 : (left + 7) >> 3, j = (id & 255) >> 3;
    const int n = base + (id & 7) * run + j;
    return j < run && n < total ? n : -1;
}
// Tiles are numbered in groups of eight row tiles across the channel tiles: an XCD's 32 are eight by four, and with fewer row tiles than
// eight it has channel tiles that no other XCD reads (512 rows, 64 x 64 tiles, N = K = 5120: 23 us; 36 where XCDs own row tiles).
__device__ __forceinline__ void tile_split(const int n, const int mtiles, const int ntiles, int& mt, int& nt) {
    const int sm = n / (8 * ntiles), rem = n - sm * (8 * ntiles), width = mtiles - 8 * sm < 8 ? mtiles - 8 * sm : 8;
    nt = rem / width;
    mt = 8 * sm + rem - nt * width;
}

// Where a block's tile lies, and its expert's weights.
struct TilePlace {
    int m0, m_end, n0;               // rows [.., m_end) are the expert's
    const int8_t* qw;
    const float *sw, *bias;
};

// The tiles of a product that is not grouped.
template <int BM, int BN>
struct DenseTiles {
    int mtiles, ntiles, total;
    __device__ __forceinline__ DenseTiles(const GemmInt8& g, int) : mtiles((int)((g.M + BM - 1) / BM)), ntiles((g.N + BN - 1) / BN), total(mtiles * ntiles) {}
    __device__ __forceinline__ bool place(const GemmInt8& g, const int id, TilePlace& p) const {
        const int n = tile_number(id, total);
        if (n < 0) return false;
        int mt, nt;
        tile_split(n, mtiles, ntiles, mt, nt);
        p = TilePlace{mt * BM, (int)g.M, nt * BN, g.qw, g.sw, g.bias};
        return true;
    }
};

// The tiles of a grouped one, expert by expert.  Every wave numbers them alone, a lane for every 64th part of the experts (up to sixteen), from one
// reading of the offsets that then stay in registers: no LDS, no barrier, and no memory access when a tile is looked up.
template <int BM, int BN>
struct GroupTiles {
    static constexpr int MOST = SVDQ_MAX_EXPERTS / 64;
    int at[MOST + 1];                // offsets of the lane's experts, as their running maximum
    int first, total;                // row tiles in front of the lane's; all tiles
    int per, e0, ntiles;

    __device__ __forceinline__ GroupTiles(const GemmInt8& g, const int lane) : per((g.groups.E + 63) >> 6), e0(lane * ((g.groups.E + 63) >> 6)), ntiles((g.N + BN - 1) / BN) {
        const int E = g.groups.E, M = (int)g.M;
        int top = 0;
#pragma unroll
        for (int j = 0; j <= MOST; ++j)
            if (j <= per) {
                const int o = g.groups.offsets[e0 + j < E ? e0 + j : E];
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
                if (j > 0) mine += (at[j] - before + BM - 1) / BM;    // (experts past the last have no rows)
                before = at[j];
            }
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        first = upto - mine;
        total = __builtin_amdgcn_readlane(upto, 63) * ntiles;
    }

    __device__ __forceinline__ bool place(const GemmInt8& g, const int id, TilePlace& p) const {
        const int n = tile_number(id, total);
        if (n < 0) return false;
        const int owner = 63 - __builtin_clzll(__ballot(first * ntiles <= n));
        int k = first, e = 0, row0 = 0, row_end = 0, k_e = 0, tiles_e = 1;
#pragma unroll
        for (int j = 0; j < MOST; ++j)
            if (j < per) {
                const int tiles = (at[j + 1] - at[j] + BM - 1) / BM;
                if (k * ntiles <= n && n < (k + tiles) * ntiles) e = e0 + j, row0 = at[j], row_end = at[j + 1], k_e = k, tiles_e = tiles;
                k += tiles;
            }
        int mt, nt;
        e = __builtin_amdgcn_readlane(e, owner);
        tile_split(n - __builtin_amdgcn_readlane(k_e, owner) * ntiles, __builtin_amdgcn_readlane(tiles_e, owner), ntiles, mt, nt);
        p = TilePlace{__builtin_amdgcn_readlane(row0, owner) + mt * BM, __builtin_amdgcn_readlane(row_end, owner), nt * BN,
                      g.qw + (int64_t)e * g.N * g.K, g.sw + (int64_t)e * g.N, g.bias ? g.bias + (int64_t)e * g.N : nullptr};
        return true;
    }
};

template <bool GROUPED, int BM, int BN> struct TilesOf { using type = DenseTiles<BM, BN>; };
template <int BM, int BN> struct TilesOf<true, BM, BN> { using type = GroupTiles<BM, BN>; };

// As many blocks as there can be tiles, in whole rounds of the numbering.
inline int most_tiles(const GemmInt8& g, const int bm, const int bn) {
    return (int)((int8_tiles(g.M, g.N, g.groups.offsets ? g.groups.E : 0, bm, bn) + 255) / 256 * 256);
}

}  // namespace svdq
