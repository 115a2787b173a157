// The product of the 8-bit layer on the int8 matrix cores: y = (qx qw^T) sx sw + bias, 32-bit integer sums over all of K (exact
// for every K the interface takes: K 128^2 < 2^31), then three binary32 roundings and one to the output's type (svdq_int8_dev.h, output).
//
// v_mfma_i32_16x16x64_i8: lane l holds row l % 16 of its operand and the 16 consecutive k [16 (l / 16), +16) as 16 bytes.  As in the
// 4-bit kernels the transposed tile D[n][m] is computed (weights are the A operand), so that a lane owns token l % 16 and the four
// consecutive channels from 4 (l / 16) on.  (The 32 x 32 x 32 instruction halves the operand reads, but
// 32760 x 5120 x 13824 ran at 2.62 POP/s with it against 2.83.)
//
// Both operands lie in memory as they come, rows of K bytes.  A stage is 128 k of every row of the tile, one full memory line per
// row: eight lanes of a direct global->LDS transfer move a row's line, and since lane i's 16 bytes land at LDS place i the
// lanes pick their pieces in rotated order: piece c of row r stands at place c ^ ((r / 2) % 8) of its 128 bytes.  The 16 rows
// that an operand read covers then meet all banks evenly.
#include "svdq_int8_dev.h"
#include "svdq_int8_plan.h"

namespace svdq {

namespace {

constexpr int I = 16;            // tokens, and channels, of a matrix instruction

// The end of a tile whose scales and biases stand in LDS (binary32: the tokens', the channels', the channels' biases): y = acc sx sw + bias,
// up to MOST tokens at a time in column groups whose rows are one memory line (128 bytes) where the wave has as many channels, each
// transposed through the wave's own LDS and stored `unit` bytes a lane, as the rows' alignment allows: 16 (a piece over the last channel goes
// element by element), 4, or an element.
template <class T, int MT, int NT, int MOST>
struct TileStore {
    static constexpr int EL = 16 / (int)sizeof(T), LINE = 8 * EL / I;  // blocks of a line
    static constexpr int CB = NT % LINE == 0 ? LINE : NT % 2 == 0 && LINE > 2 ? 2 : 1, COLS = CB * I, ROWS = MT * I <= MOST ? MT * I : MOST;
    static constexpr int PITCH = COLS * (int)sizeof(T) + 16, BYTES = ROWS * PITCH;
    static constexpr int MP = ROWS / I, LANES = COLS / EL, STEP = 64 / LANES;
    static_assert(NT % CB == 0 && MT % MP == 0, "whole groups");
    // region: BYTES of the wave's own.  tokens, channels, biases: LDS addresses of the wave's first.
    static __device__ __forceinline__ void run(const int4v (&acc)[NT][MT], const uint32_t region, const uint32_t tokens, const uint32_t channels, const uint32_t biases,
                                               const bool has_bias, const int lane, T* __restrict__ y, const int64_t ldy, const int rows, const int cols, const int unit) {
        const int li = lane % I, lk = lane / I;
#pragma unroll
        for (int m0 = 0; m0 < MT; m0 += MP) {
            float ts[MP];
#pragma unroll
            for (int mi = 0; mi < MP; ++mi) ts[mi] = bits_f(lds_read4(tokens + ((m0 + mi) * I + li) * 4));
#pragma unroll
            for (int g = 0; g < NT / CB; ++g) {
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    const int ni = g * CB + cb, at = 4 * lk;
                    const uint32_t c = (ni * I + at) * 4;
                    const uint4 s4 = lds_read16(channels + c), b4 = has_bias ? lds_read16(biases + c) : uint4{0, 0, 0, 0};
                    const float s[4] = {bits_f(s4.x), bits_f(s4.y), bits_f(s4.z), bits_f(s4.w)};
                    const float b[4] = {bits_f(b4.x), bits_f(b4.y), bits_f(b4.z), bits_f(b4.w)};
#pragma unroll
                    for (int mi = 0; mi < MP; ++mi) {
                        float v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = output(acc[ni][m0 + mi][i], ts[mi], s[i], b[i]);
                        const uint32_t to = region + (mi * I + li) * PITCH + (cb * I + at) * (int)sizeof(T);
                        if constexpr (sizeof(T) == 2) {
                            lds_write8_pinned(to, uint2{f2_bf16_rne(v[0], v[1]), f2_bf16_rne(v[2], v[3])});
                        } else {
                            lds_write8_pinned(to, uint2{f_bits(v[0]), f_bits(v[1])});
                            lds_write8_pinned(to + 8, uint2{f_bits(v[2]), f_bits(v[3])});
                        }
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                const int left = cols - g * COLS;
                T* const y0 = y + g * COLS;
                if (unit == 16) {
                    const int r0 = lane / LANES, c = lane % LANES;
#pragma unroll
                    for (int it = 0; it < (ROWS + STEP - 1) / STEP; ++it) {
                        const int row = it * STEP + r0;
                        if (ROWS % STEP && row >= ROWS) continue;
                        const uint4 v = lds_read16_pinned(region + row * PITCH + c * 16);
                        if (m0 * I + row >= rows) continue;
                        T* const p = y0 + (int64_t)(m0 * I + row) * ldy + c * EL;
                        if ((c + 1) * EL <= left) {
                            *reinterpret_cast<uint4*>(p) = v;
                        } else {
                            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int i = 0; i < EL; ++i)
                                if (c * EL + i < left) {
                                    if constexpr (sizeof(T) == 2) p[i] = (T)(w[i >> 1] >> (16 * (i & 1)));
                                    else p[i] = w[i];
                                }
                        }
                    }
                } else {
                    // four bytes a lane, or two: consecutive lanes store consecutive elements
                    auto by = [&](auto PERC) {
                        constexpr int PER = decltype(PERC)::value, E = COLS / PER;       // stores a row, elements each
#pragma unroll 4
                        for (int i = lane; i < ROWS * PER; i += 64) {
                            const int row = i / PER, c = i % PER;
                            if (m0 * I + row >= rows) break;
                            T* const p = y0 + (int64_t)(m0 * I + row) * ldy + c * E;
                            const uint32_t v = lds_read4(region + row * PITCH + (c * E * (int)sizeof(T) & ~3));
                            if constexpr (E * sizeof(T) == 2) {
                                if (c < left) *p = (T)(v >> (16 * (c & 1)));
                            } else if constexpr (E == 2) {
                                if (2 * c + 1 < left) *reinterpret_cast<uint32_t*>(p) = v;
                                else if (2 * c < left) *p = (T)v;
                            } else {
                                if (c < left) *p = (T)v;
                            }
                        }
                    };
                    if (sizeof(T) == 4 || unit == 2) by(IC<COLS>{});
                    else by(IC<COLS / 2>{});
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            }
        }
    }
};

// A tile of BM tokens by BN channels for WM x WN waves; its operands stand in LDS from DEPTH stages ahead on.
template <int BM_, int BN_, int WM_, int WN_, int DEPTH_, bool LINES_ = false>
struct Int8Tile {
    static constexpr bool LINES = LINES_;                             // fetched by whole lines: of a K that is no multiple of a stage
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, DEPTH = DEPTH_, NW = WM * WN, THREADS = 64 * NW, MT = BM / WM / I, NT = BN / WN / I;
    static constexpr int NA = (BM / 8 + NW - 1) / NW, NB = (BN / 8 + NW - 1) / NW;                    // transfers of a wave a stage, eight rows each
    static constexpr uint32_t A = BM * BK, W = BN * BK, RING = (DEPTH + 1) * A + DEPTH * W;
    static constexpr int TOKENS = (BM + 63) / 64 * 64, CHANNELS = (BN + 63) / 64 * 64;                // scales and biases come 64 at a time
    static constexpr uint32_t SCALES = (TOKENS + 2 * CHANNELS) * 4;
    static_assert(BM % (WM * I) == 0 && BN % (WN * I) == 0 && MT * NT % 2 == 0 && DEPTH >= 2, "whole blocks, and quarters of a stage's instructions");
};

// The tokens' rows of a stage, A(s), stand in a ring of DEPTH + 1 places, the channels', W(s), in one of DEPTH.  Stage s requests
// A(s + DEPTH) during its first three quarters (its place has been free since the barrier of stage s - 1) and W(s + DEPTH) during its
// last, where W(s) stood: requests that come all at once behind the barrier take longer than the instructions that they stand between
// (with a place less and all of them there, 256 x 256 tiles took 6 % longer at K = 13824).
// TAIL: K is no multiple of a stage.  The last stage's pieces beyond K repeat the row's last piece, and count as zeros in the weights' operand.
//
// LINES: rows of such a K begin anywhere in a memory line, so that 128 bytes from where a row begins are parts of two lines and a stage's transfers
// fetch every line twice.  Here they fetch whole lines: window j of a row is the j-th line that the row has a part of, its k begin `phase`
// pieces into window 0, and stage s reads windows s and s + 1, each lane the one that its piece is in.  (The phase of a row goes by its number modulo
// 16, so that a lane has one for all its rows; the rotation above still spreads 16 rows over all banks, for every K.)  A stage more has to have
// arrived, and the channels' ring has a place more: tiles of up to 128 tokens have the LDS.  512 x 5120, K = 5136: 21.2 us, 27.5 without.
template <class G, bool TAIL, bool GROUPED, class T>
__global__ __launch_bounds__(G::THREADS, 1)
void gemm_int8_kernel(const GemmInt8 g) {
    constexpr int BM = G::BM, BN = G::BN, MT = G::MT, NT = G::NT, NA = G::NA, NB = G::NB, DEPTH = G::DEPTH;
    constexpr bool LINES = TAIL && G::LINES;
    constexpr uint32_t RING = G::RING + (LINES ? G::W : 0);
    using Store = TileStore<T, MT, NT, (RING >= (G::NW + 1) * 64 * 144 + G::SCALES ? 64 : 32)>;
    static_assert(RING >= (G::NW + 1) * Store::BYTES + G::SCALES && G::A >= G::SCALES, "the store transposes in the ring, beside the scales");
    __shared__ __attribute__((aligned(16))) uint8_t ring[RING];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % G::WM, wn = wave / G::WM;
    const int li = lane % I, lk = lane / I;
    const int K = g.K, N = g.N;
    const uint32_t ring_a = (uint32_t)(uintptr_t)(lds_byte*)ring, ring_w = ring_a + (DEPTH + 1) * G::A;
    TilePlace at;
    if (!typename TilesOf<GROUPED, BM, BN>::type(g, lane).place(g, blockIdx.x, at)) return;
    const int m0 = at.m0, m_end = at.m_end, n0 = at.n0;
    const int nstages = (K + BK - 1) / BK;

    // ---- transfers: j of this wave covers rows 8 (wave NA + j) .. + 7 (where that is past the tile: its last eight rows again)
    const int a0 = wave * NA, w0 = wave * NB;
    auto block_a = [&](const int j) { return BM / 8 % G::NW == 0 || a0 + j < BM / 8 ? a0 + j : BM / 8 - 1; };
    auto block_w = [&](const int j) { return BN / 8 % G::NW == 0 || w0 + j < BN / 8 ? w0 + j : BN / 8 - 1; };
    const int8_t* const abase = g.qx + (int64_t)m0 * K;
    const int8_t* const wbase = at.qw + (int64_t)n0 * K;
    const int place = lane & 7;
    const uint32_t first_a = (uint32_t)((uintptr_t)abase >> 4), first_w = (uint32_t)((uintptr_t)wbase >> 4);
    auto phase = [&](const uint32_t first, const int row) { return LINES ? (int)((first + (uint32_t)row * (uint32_t)(K >> 4)) & 7) : 0; };
    uint32_t va[NA], vw[NB];
    int pa[NA], pw[NB];                                               // piece of a row in stage 0: negative ones are the row's before
    auto rows_of = [&](uint32_t& v, int& piece, const uint32_t first, const int block, const int last) {      // rows past the end repeat the last one
        const int row = 8 * block + (lane >> 3), from = row < last ? row : last;
        piece = (place ^ ((row >> 1) & 7)) - phase(first, from);
        v = (uint32_t)from * (uint32_t)K + (uint32_t)(piece + (LINES ? 8 : 0)) * 16;
    };
#pragma unroll
    for (int j = 0; j < NA; ++j) rows_of(va[j], pa[j], first_a, block_a(j), m_end - 1 - m0);
#pragma unroll
    for (int j = 0; j < NB; ++j) rows_of(vw[j], pw[j], first_w, block_w(j), N - 1 - n0);
    // EDGE: of what may be the last stage (with LINES, one of the last two windows or the first), whose pieces can lie beyond K (or before the row)
    auto request = [&](auto EDGEC, const int8_t* base, uint32_t v, const int piece, const int s, const uint32_t to) {
        if constexpr (TAIL && decltype(EDGEC)::value) {
            const int k16 = 8 * s + piece, last = (K >> 4) - 1;
            if (k16 > last) v -= (k16 - last) * 16;
            if (LINES && k16 < 0) v -= k16 * 16;
        }
        dma16(base + (int64_t)(s - (LINES ? 1 : 0)) * BK, v, to);
    };
    auto request_a = [&](auto EDGEC, const int s, const uint32_t to, const int j) { request(EDGEC, abase, va[j], pa[j], s, to + block_a(j) * 1024); };
    auto request_w = [&](auto EDGEC, const int s, const uint32_t to, const int j) { request(EDGEC, wbase, vw[j], pw[j], s, to + block_w(j) * 1024); };
    auto next_a = [&](const uint32_t c) { return c == ring_a + DEPTH * G::A ? ring_a : c + G::A; };
    constexpr int PLACES_W = LINES ? DEPTH + 1 : DEPTH;
    auto next_w = [&](const uint32_t c) { return c == ring_w + (PLACES_W - 1) * G::W ? ring_w : c + G::W; };

    // ---- operands: piece PS kk + lk of a row, for k step kk, stands at that place ^ (row / 2) % 8
    constexpr int PS = 64 / I, STEPS = 8 / PS;
    const int turn = (li >> 1) & 7;
    uint32_t rd_a[STEPS], rd_w[STEPS];
    bool on_a[STEPS], on_w[STEPS];                                    // the lane's piece is in the window behind
#pragma unroll
    for (int kk = 0; kk < STEPS; ++kk) {
        const int qa = PS * kk + lk + phase(first_a, li), qw = PS * kk + lk + phase(first_w, li);
        rd_a[kk] = (wm * MT * I + li) * BK + (((qa & 7) ^ turn) << 4);
        rd_w[kk] = (wn * NT * I + li) * BK + (((qw & 7) ^ turn) << 4);
        on_a[kk] = LINES && qa > 7, on_w[kk] = LINES && qw > 7;
    }
    struct Operands {
        int4v w[NT], x[MT];
    };
    typedef const volatile __attribute__((address_space(3))) int4v lds_i4;
    auto fetch = [&](const uint32_t from, const int block) { return *reinterpret_cast<lds_i4*>((lds_byte*)(uintptr_t)from + block * I * BK); };
    auto read = [&](auto EDGEC, Operands& o, const uint32_t fa, const uint32_t fw, const int s, const int kk, const int r) {
        if (r >= 1 && r <= MT) {                                      // in the order of their use
            o.x[r - 1] = fetch(fa, r - 1);
            return;
        }
        const int ni = r == 0 ? 0 : r - MT;
        o.w[ni] = fetch(fw, ni);
        if constexpr (TAIL && decltype(EDGEC)::value) {
            if (8 * s + PS * kk + lk >= (K >> 4)) o.w[ni] = int4v{0, 0, 0, 0};
        }
    };

    int4v acc[NT][MT];
#pragma unroll
    for (int ni = 0; ni < NT; ++ni)
#pragma unroll
        for (int mi = 0; mi < MT; ++mi) acc[ni][mi] = int4v{0, 0, 0, 0};

    uint32_t cur_a = ring_a, cur_w = ring_w;
    const int windows = nstages + (LINES ? 1 : 0);                    // of the transfers
#pragma unroll
    for (int s = 0; s < DEPTH; ++s)
        if (s < windows) {
#pragma unroll
            for (int j = 0; j < NA; ++j) request_a(IC<1>{}, s, ring_a + s * G::A, j);
#pragma unroll
            for (int j = 0; j < NB; ++j) request_w(IC<1>{}, s, ring_w + s * G::W, j);
        }
    // wait for a stage with `behind` whole ones, at most DEPTH - 1, requested after it
    auto wait_for = [&](const int behind) {
        if (DEPTH > 3 && behind >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * (NA + NB)) : "memory");
        else if (DEPTH > 2 && behind == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (NA + NB)) : "memory");
        else if (behind == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NA + NB) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    static_assert(DEPTH <= 4 && (!LINES || DEPTH >= 3), "the waits");
    wait_for((windows < DEPTH ? windows : DEPTH) - (LINES ? 2 : 1));
    __syncthreads();
    constexpr int T_ = MT * NT, READS = MT + NT, QUARTER = STEPS * T_ / 4;
    Operands op[2];
#pragma unroll
    for (int r = 0; r < READS; ++r) read(IC<1>{}, op[0], (on_a[0] ? ring_a + G::A : ring_a) + rd_a[0], (on_w[0] ? ring_w + G::W : ring_w) + rd_w[0], 0, 0, r);

    // A stage is STEPS k steps, of T_ instructions each; between those the reads of the next step's operands and the stage's requests.
    // Before its last quarter (when every wave has all of its operands) stand the wait for the next stage's rows and the barrier.
    // EDGE: its requests may be the last stage's, or its reads.
    auto stage = [&](const int s, auto FILLC, auto EDGEC, auto LASTC) {
        constexpr bool fill = decltype(FILLC)::value, last = decltype(LASTC)::value;
        const uint32_t na = next_a(cur_a), nw = next_w(cur_w), free_a = cur_a == ring_a ? ring_a + DEPTH * G::A : cur_a - G::A;
        const uint32_t free_w = !LINES ? cur_w : cur_w == ring_w ? ring_w + DEPTH * G::W : cur_w - G::W;
        auto instructions = [&](auto FROM, auto TO) {
            constexpr int from = decltype(FROM)::value, until = decltype(TO)::value, kk = from / T_, rk = (kk + 1) % STEPS;
            constexpr bool next = kk + 1 == STEPS;                    // its reads are of the next stage, behind the barrier
            constexpr int r0 = next ? 3 * QUARTER : kk * T_, span = next ? QUARTER : T_, RP = (READS + span - 1) / span;
            uint32_t fa = next ? na : cur_a, fw = next ? nw : cur_w;
            if constexpr (LINES) fa = on_a[rk] ? next_a(fa) : fa, fw = on_w[rk] ? next_w(fw) : fw;
            fa += rd_a[rk];
            fw += rd_w[rk];
            asm volatile("" : "+v"(fa), "+v"(fw));
#pragma unroll
            for (int n = from; n < until; ++n) {
                const int t = n % T_, ni = t / MT, mi = t % MT;
                acc[ni][mi] = __builtin_amdgcn_mfma_i32_16x16x64_i8(op[kk & 1].w[ni], op[kk & 1].x[mi], acc[ni][mi], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if (!(next && last) && n >= r0)
#pragma unroll
                    for (int r = (n - r0) * RP; r < (n - r0 + 1) * RP && r < READS; ++r)
                        read(EDGEC, op[rk & 1], fa, fw, next ? s + 1 : s, rk, r);
                if constexpr (fill) {                                 // request i of n stands behind instruction (i + 1/2) / n of its part
#pragma unroll
                    for (int j = 0; j < NA; ++j)
                        if (n == (2 * j + 1) * 3 * QUARTER / (2 * NA)) request_a(EDGEC, s + DEPTH, free_a, j);
#pragma unroll
                    for (int j = 0; j < NB; ++j)
                        if (n == 3 * QUARTER + j * QUARTER / NB) request_w(EDGEC, s + DEPTH, free_w, j);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        instructions(IC<0>{}, IC<T_>{});
        instructions(IC<T_>{}, IC<3 * QUARTER>{});
        if constexpr (fill) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - (LINES ? 3 : 2)) * (NA + NB) + NA) : "memory");
        else wait_for(nstages - 2 - s);
        __syncthreads();
        instructions(IC<3 * QUARTER>{}, IC<4 * QUARTER>{});
        cur_a = na;
        cur_w = nw;
    };
    int s = 0;
    for (; s + DEPTH + (LINES ? 2 : TAIL ? 1 : 0) < windows; ++s) stage(s, IC<1>{}, IC<0>{}, IC<0>{});
    if constexpr (TAIL)
        for (; s + DEPTH < windows; ++s) stage(s, IC<1>{}, IC<1>{}, IC<0>{});
    for (; s + 1 < nstages; ++s) stage(s, IC<0>{}, IC<1>{}, IC<0>{});
    // the last stage's requests are the tile's scales and biases, 64 values each, into a free place of the tokens'
    const uint32_t scales = LINES ? (cur_a == ring_a ? ring_a + DEPTH * G::A : cur_a - G::A) : next_a(cur_a);
    for (int j = wave; j < (int)G::SCALES / 256; j += G::NW) {
        constexpr int CHANNEL0 = G::TOKENS / 64, BIAS0 = CHANNEL0 + G::CHANNELS / 64;
        const bool tok = j < CHANNEL0, bia = j >= BIAS0;
        const int i = (j - (tok ? 0 : bia ? BIAS0 : CHANNEL0)) * 64 + lane, end = tok ? m_end - 1 - m0 : N - 1 - n0;
        if (!bia || at.bias) dma4(tok ? g.sx + m0 : bia ? at.bias + n0 : at.sw + n0, (uint32_t)(i < end ? i : end) * 4, scales + j * 256);
    }
    stage(s, IC<0>{}, IC<1>{}, IC<1>{});

    const int own_lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)) & 63;      // no register through the K loop for it
    const uintptr_t ends = reinterpret_cast<uintptr_t>(g.y) | (uintptr_t)(g.ldy * (int64_t)sizeof(T));
    const int unit = (ends & 15) == 0 ? 16 : (ends & 3) == 0 ? 4 : 2;
    const int mw = m0 + wm * MT * I, nw = n0 + wn * NT * I;
    if (nw >= N || mw >= m_end) return;
    const int below = (int)(scales - ring_a) / Store::BYTES;          // waves whose store area fits below the scales
    const uint32_t region = wave < below ? ring_a + wave * Store::BYTES : scales + G::SCALES + (wave - below) * Store::BYTES;
    Store::run(acc, region, scales + wm * MT * I * 4, scales + (G::TOKENS + wn * NT * I) * 4, scales + (G::TOKENS + G::CHANNELS + wn * NT * I) * 4,
               at.bias != nullptr, own_lane, reinterpret_cast<T*>(g.y) + (int64_t)mw * g.ldy + nw, g.ldy, m_end - mw, N - nw, unit);
}

// WHOLE: of a K of whole stages only.
template <class G, bool WHOLE = false>
hipError_t launch_tiles(const GemmInt8& g, const bool out_f32, hipStream_t stream) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(most_tiles(g, G::BM, G::BN)), dim3(G::THREADS), 0, stream, g); };
    auto typed = [&](auto TAILC, auto GROUPEDC) {
        constexpr bool TAIL = decltype(TAILC)::value, GROUPED = decltype(GROUPEDC)::value;
        if (out_f32) go(gemm_int8_kernel<G, TAIL, GROUPED, uint32_t>);
        else go(gemm_int8_kernel<G, TAIL, GROUPED, uint16_t>);
    };
    const bool grouped = g.groups.offsets != nullptr;
    if constexpr (!WHOLE) {
        if (G::LINES || g.K % BK) {
            grouped ? typed(IC<1>{}, IC<1>{}) : typed(IC<1>{}, IC<0>{});
            return hipGetLastError();
        }
    }
    if constexpr (!G::LINES) grouped ? typed(IC<0>{}, IC<1>{}) : typed(IC<0>{}, IC<0>{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_int8(const GemmInt8& g, const Int8Plan& p, bool out_f32, hipStream_t stream) {
    const Int8Kernel k = int8_kernel(p.tiles, g.M, g.N, g.K, g.groups.offsets ? g.groups.E : 0);
    switch (p.tiles) {
        case Int8Tiles::T64x32: return launch_tiles<Int8Tile<64, 32, 2, 2, 4>>(g, out_f32, stream);
        case Int8Tiles::T64x64: return launch_tiles<Int8Tile<64, 64, 2, 2, 4>>(g, out_f32, stream);
        case Int8Tiles::T64x128:
            if (k.lines) return launch_tiles<Int8Tile<64, 128, 2, 4, 4, true>>(g, out_f32, stream);
            return launch_tiles<Int8Tile<64, 128, 2, 4, 3>>(g, out_f32, stream);
        case Int8Tiles::T128x128:
            if (k.lines) return launch_tiles<Int8Tile<128, 128, 2, 4, 4, true>>(g, out_f32, stream);
            if (k.depth == 4) return launch_tiles<Int8Tile<128, 128, 2, 4, 4>, true>(g, out_f32, stream);
            return launch_tiles<Int8Tile<128, 128, 2, 4, 2>>(g, out_f32, stream);
        case Int8Tiles::T256x128: return launch_tiles<Int8Tile<256, 128, 4, 2, 2>>(g, out_f32, stream);
        case Int8Tiles::T256x160: return launch_tiles<Int8Tile<256, 160, 4, 2, 2>>(g, out_f32, stream);
        case Int8Tiles::T256x256: return launch_tiles<Int8Tile<256, 256, 2, 4, 2>>(g, out_f32, stream);
        default: return launch_gemm_int8_few(g, k, out_f32, stream);
    }
}

}  // namespace svdq
