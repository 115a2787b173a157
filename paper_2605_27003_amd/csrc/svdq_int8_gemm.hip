// The product of the 8-bit layer on the int8 matrix cores: y = (qx qw^T) sx sw + bias, 32-bit integer sums over all of K (exact
// for every K the interface takes: K 127^2 < 2^31), then three binary32 operations and one rounding to the output's type.
//
// v_mfma_i32_32x32x32_i8: lane l holds row l % 32 of its operand and the 16 consecutive k [16 (l / 32), +16) as 16 bytes.  As in the
// 4-bit kernels the transposed tile D[n][m] is computed (weights are the A operand), so that a lane owns one token and, per
// register quad, four consecutive channels.
//
// Both operands lie in memory as they come, rows of K bytes.  A stage is 128 k of every row of the tile, one full memory line per
// row: eight lanes of a direct global->LDS transfer move a row's line, and since lane i's 16 bytes land at LDS place i the
// lanes pick their pieces in rotated order: piece c of row r stands at place c ^ ((r / 2) % 8) of its 128 bytes.  The 32 rows
// that an operand read covers then meet all banks evenly.
#include "svdq_int8_dev.h"
#include "svdq_kernels.h"
#include "svdq_tiles.h"

namespace svdq {

namespace {

constexpr int BK = 128;                                   // k (and bytes) of a row per stage

template <int BM_, int BN_, int WM_, int WN_, int NS_>
struct Int8Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NS = NS_, NW = WM * WN, THREADS = 64 * NW;
    static constexpr int MT = BM / WM / 32, NT = BN / WN / 32;        // 32 x 32 blocks of a wave
    static constexpr int ND = (BM + BN) / 8 / NW;                     // transfers of a wave per stage, eight rows each
    static constexpr uint32_t STAGE = (BM + BN) * BK;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "a transfer is of one operand");
};

// A wave's finished block row: 32 tokens x 32 NT channels, transposed through the wave's own LDS and stored 16 bytes a lane.
// value(ni, i) is the lane's token's value of channel 32 ni + 8 (i / 4) + 4 (lane / 32) + i % 4.  `vec`: whole pieces can be stored
// as 16 bytes; the pieces at N's end, and all of them otherwise, go element by element.
template <class T, int NT, class Value>
__device__ __forceinline__ void store_rows(Value value, const uint32_t region, const int lane, T* __restrict__ y, const int64_t ldy,
                                           const int rows, const int cols, const bool vec) {
    constexpr int ROW = NT * 32 * (int)sizeof(T), PITCH = ROW + 16, LANES = ROW / 16, STEP = 64 / LANES, EL = 16 / (int)sizeof(T);
    const int l32 = lane & 31, kh = lane >> 5;
#pragma unroll
    for (int ni = 0; ni < NT; ++ni)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t at = region + l32 * PITCH + (ni * 32 + 8 * q + 4 * kh) * (int)sizeof(T);
            const float v0 = value(ni, 4 * q), v1 = value(ni, 4 * q + 1), v2 = value(ni, 4 * q + 2), v3 = value(ni, 4 * q + 3);
            if constexpr (sizeof(T) == 2) {
                lds_write8_pinned(at, uint2{f2_bf16_rne(v0, v1), f2_bf16_rne(v2, v3)});
            } else {
                lds_write8_pinned(at, uint2{f_bits(v0), f_bits(v1)});
                lds_write8_pinned(at + 8, uint2{f_bits(v2), f_bits(v3)});
            }
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int r0 = lane / LANES, c = lane % LANES;
#pragma unroll
    for (int it = 0; it < 32 / STEP; ++it) {
        const int row = it * STEP + r0;
        const uint4 v = lds_read16_pinned(region + row * PITCH + c * 16);
        if (row >= rows) continue;
        T* const p = y + (int64_t)row * ldy + c * EL;
        if (vec && (c + 1) * EL <= cols) {
            *reinterpret_cast<uint4*>(p) = v;
        } else {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < EL; ++i)
                if (c * EL + i < cols) {
                    if constexpr (sizeof(T) == 2) p[i] = (T)(w[i >> 1] >> (16 * (i & 1)));
                    else p[i] = w[i];
                }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// TAIL: K is no multiple of a stage.  The last stage's pieces beyond K repeat the row's last piece, and count as zeros in the
// weights' operand.
template <class G, bool TAIL, bool GROUPED, class T>
__global__ __launch_bounds__(G::THREADS, 1)
void gemm_int8_kernel(const GemmInt8 g, const TileGrid tg) {
    constexpr int BM = G::BM, BN = G::BN, MT = G::MT, NT = G::NT, NS = G::NS, ND = G::ND, NW = G::NW;
    constexpr int STORE = 32 * (NT * 32 * 4 + 16);                    // of a wave, the wider type's
    constexpr uint32_t RING = NS * G::STAGE, BYTES = RING > NW * STORE ? RING : NW * STORE;
    __shared__ __attribute__((aligned(16))) uint8_t ring[BYTES];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % G::WM, wn = wave / G::WM;
    const int l32 = lane & 31, kh = lane >> 5;
    const int K = g.K, N = g.N;
    const uint32_t ring0 = (uint32_t)(uintptr_t)(lds_byte*)ring;

    int m0, m_end, n0;
    const int8_t* qw = g.qw;
    const float *sw = g.sw, *bias = g.bias;
    if constexpr (GROUPED) {
        GroupTile t;
        if (!group_tile(g.groups, (int)g.M, BM, tg.ntiles, blockIdx.x, lane, t)) return;
        m0 = t.row0 + t.mt * BM;
        m_end = t.row_end;
        n0 = t.nt * BN;
        qw += (int64_t)t.e * N * K;
        sw += (int64_t)t.e * N;
        if (bias) bias += (int64_t)t.e * N;
    } else {
        int mt, nt;
        if (!tile_of(tg, blockIdx.x, mt, nt)) return;
        m0 = mt * BM;
        m_end = (int)g.M;
        n0 = nt * BN;
    }
    const int nstages = (K + BK - 1) / BK;

    // ---- transfers: number j of this wave covers rows 8 j .. 8 j + 7 of the tile's tokens, then of its channels
    const int8_t* const abase = g.qx + (int64_t)m0 * K;
    const int8_t* const wbase = qw + (int64_t)n0 * K;
    const int place = lane & 7;
    uint32_t voff[ND], piece[2];
    piece[0] = place ^ (lane >> 4);
    piece[1] = place ^ (4 + (lane >> 4));
#pragma unroll
    for (int p = 0; p < ND; ++p) {
        const int j = wave * ND + p;
        const bool w = 8 * j >= BM;
        const int left = (w ? N - 1 - n0 : m_end - 1 - m0);           // rows past the end repeat the last one
        int row = 8 * j - (w ? BM : 0) + (lane >> 3);
        row = row < left ? row : left;
        voff[p] = (uint32_t)row * (uint32_t)K + piece[j & 1] * 16;
    }
    auto request = [&](const int s, const uint32_t slot, const int p) {
        const int j = wave * ND + p;
        const int8_t* const base = (8 * j >= BM ? wbase : abase) + (int64_t)s * BK;
        uint32_t v = voff[p];
        if constexpr (TAIL) {
            const int left = (K >> 4) - 8 * s - 1, over = (int)piece[j & 1] - left;
            if (over > 0) v -= over * 16;
        }
        dma16(base, v, slot + j * 1024);
    };

    // ---- operands: piece 2 kk + kh of a row for k step kk
    const uint32_t turn = (kh ^ (l32 >> 1)) & 7;
    const uint32_t rd_a = (wm * MT * 32 + l32) * BK, rd_w = (BM + wn * NT * 32 + l32) * BK;
    struct Operands {
        uint4 w[NT], x[MT];
    };
    auto read_w = [&](Operands& o, const uint32_t slot, const int s, const int kk, const int ni) {
        uint4 v = lds_read16_pinned(slot + rd_w + ni * 32 * BK + ((turn ^ (2 * kk)) << 4));
        if constexpr (TAIL) {
            if (8 * s + 2 * kk + kh >= (K >> 4)) v = uint4{0, 0, 0, 0};
        }
        o.w[ni] = v;
    };
    auto read_x = [&](Operands& o, const uint32_t slot, const int kk, const int mi) {
        o.x[mi] = lds_read16_pinned(slot + rd_a + mi * 32 * BK + ((turn ^ (2 * kk)) << 4));
    };
    auto next_slot = [&](const uint32_t c) { return (c == ring0 + (NS - 1) * G::STAGE) ? ring0 : c + G::STAGE; };

    int16v acc[NT][MT];
#pragma unroll
    for (int ni = 0; ni < NT; ++ni)
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) acc[ni][mi] = (int16v)(0);

    uint32_t cur = ring0;
    {
        uint32_t sl = ring0;
        for (int s = 0; s < NS; ++s) {
            if (s < nstages)
#pragma unroll
                for (int p = 0; p < ND; ++p) request(s, sl, p);
            sl = next_slot(sl);
        }
        if (nstages >= NS) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 1) * ND) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    Operands op0, op1;
#pragma unroll
    for (int ni = 0; ni < NT; ++ni) read_w(op0, cur, 0, 0, ni);
#pragma unroll
    for (int mi = 0; mi < MT; ++mi) read_x(op0, cur, 0, mi);

    // One k step: the products of `o`, and between them the reads of the next step's operands into `on` and, where the stage's slot
    // has become free, the requests that fill it again.
    auto step = [&](const Operands& o, Operands& on, const uint32_t slot, const int s, const int kk, const bool fetch, const bool refill,
                    const int rs, const uint32_t rslot) {
        constexpr int T_ = MT * NT, READS = MT + NT, RP = (READS + T_ - 1) / T_, DP = (ND + T_ - 1) / T_;
#pragma unroll
        for (int t = 0; t < T_; ++t) {
            const int ni = t / MT, mi = t % MT;
            const int4v a = {(int)o.w[ni].x, (int)o.w[ni].y, (int)o.w[ni].z, (int)o.w[ni].w};
            const int4v b = {(int)o.x[mi].x, (int)o.x[mi].y, (int)o.x[mi].z, (int)o.x[mi].w};
            acc[ni][mi] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc[ni][mi], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (fetch)
#pragma unroll
                for (int r = t * RP; r < (t + 1) * RP && r < READS; ++r) {
                    if (r == 0) read_w(on, slot, s, kk, 0);           // in the order of their use
                    else if (r <= MT) read_x(on, slot, kk, r - 1);
                    else read_w(on, slot, s, kk, r - MT);
                }
            if (refill)
#pragma unroll
                for (int p = t * DP; p < (t + 1) * DP && p < ND; ++p) request(rs, rslot, p);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // A stage: the wait for the next one and the barrier stand in front of its last step, when every wave has taken its last
    // operands of this one out of LDS; that step's instructions carry the requests for stage s + NS.
    auto stage = [&](const int s, const bool refill, const bool last) {
        step(op0, op1, cur, s, 1, true, false, 0, 0);
        step(op1, op0, cur, s, 2, true, false, 0, 0);
        step(op0, op1, cur, s, 3, true, false, 0, 0);
        if (refill) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * ND) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const uint32_t nxt = next_slot(cur);
        step(op1, op0, nxt, s + 1, 0, !last, refill, s + NS, cur);
        cur = nxt;
    };
    int s = 0;
    for (; s + NS < nstages; ++s) stage(s, true, false);
    for (; s + 1 < nstages; ++s) stage(s, false, false);
    stage(s, false, true);

    // ---- y = acc sx sw + bias, one block row at a time.  The barrier of the last stage was passed when every wave had read its
    // last operands: the ring is free.
    const bool vec = ((reinterpret_cast<uintptr_t>(g.y) | (uintptr_t)(g.ldy * (int64_t)sizeof(T))) & 15) == 0;
    const int nw = n0 + wn * NT * 32;
    if (nw >= N) return;
    float cs[NT][16], cb[NT][16];
#pragma unroll
    for (int ni = 0; ni < NT; ++ni)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int n = nw + 32 * ni + 8 * (i >> 2) + 4 * kh + (i & 3), at = n < N ? n : N - 1;
            cs[ni][i] = sw[at];
            cb[ni][i] = bias ? bias[at] : 0.0f;
        }
#pragma unroll
    for (int mi = 0; mi < MT; ++mi) {
        const int m = m0 + (wm * MT + mi) * 32, rows = m_end - m;
        if (rows <= 0) break;
        const float ts = g.sx[l32 < rows ? m + l32 : m_end - 1];
        store_rows<T, NT>([&](const int ni, const int i) { return ((float)acc[ni][mi][i] * ts) * cs[ni][i] + cb[ni][i]; },
                          ring0 + wave * STORE, lane, reinterpret_cast<T*>(g.y) + (int64_t)m * g.ldy + nw, g.ldy, rows, N - nw, vec);
    }
}

template <class G, bool TAIL, bool GROUPED>
void launch_tiles_t(const GemmInt8& g, const bool out_f32, const TileGrid& tg, const int blocks, hipStream_t stream) {
    if (out_f32) hipLaunchKernelGGL((gemm_int8_kernel<G, TAIL, GROUPED, uint32_t>), dim3(blocks), dim3(G::THREADS), 0, stream, g, tg);
    else hipLaunchKernelGGL((gemm_int8_kernel<G, TAIL, GROUPED, uint16_t>), dim3(blocks), dim3(G::THREADS), 0, stream, g, tg);
}

// As many blocks as there can be tiles: every expert with rows adds at most one row tile that is not full.
template <class G>
int64_t grouped_blocks(const GemmInt8& g) {
    const int64_t mt = g.M / G::BM + (g.M < g.groups.E ? g.M : g.groups.E);
    return (mt * ((g.N + G::BN - 1) / G::BN) + 7) / 8 * 8;
}

template <class G>
hipError_t launch_tiles(const GemmInt8& g, const bool out_f32, hipStream_t stream) {
    const int ntiles = (g.N + G::BN - 1) / G::BN;
    const bool tail = g.K % BK != 0;
    if (g.groups.offsets) {
        const int blocks = (int)grouped_blocks<G>(g);
        const TileGrid tg{0, ntiles, 0, 0};
        if (tail) launch_tiles_t<G, true, true>(g, out_f32, tg, blocks, stream);
        else launch_tiles_t<G, false, true>(g, out_f32, tg, blocks, stream);
        return hipGetLastError();
    }
    const TileGrid tg = make_tile_grid((int)((g.M + G::BM - 1) / G::BM), ntiles);
    if (tail) launch_tiles_t<G, true, false>(g, out_f32, tg, tile_ids(tg), stream);
    else launch_tiles_t<G, false, false>(g, out_f32, tg, tile_ids(tg), stream);
    return hipGetLastError();
}

using T128 = Int8Tile<128, 128, 2, 2, 2>;

}  // namespace

// Block ids and tile numbers are 32-bit: rounded up to the eight XCDs, fewer than 2^31 / 8 row tiles of eight by channel tiles.
bool gemm_int8_fits(const GemmInt8& g) {
    const int64_t mt = (g.M + 127) / 128 + (g.groups.offsets ? g.groups.E : 0), nt = ((int64_t)g.N + 127) / 128;
    return (mt + 8) * (nt + 8) < INT32_MAX;
}

hipError_t launch_gemm_int8(const GemmInt8& g, bool out_f32, hipStream_t stream) { return launch_tiles<T128>(g, out_f32, stream); }

}  // namespace svdq
