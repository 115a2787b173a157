// Activations of the 8-bit layer: one pass over x that smooths (eq. 5), finds every token's largest magnitude, derives its clipped
// scale s = (rho a) / 127 (eq. 8-9) and rounds its codes (eq. 3), K + 4 bytes written for 2 K read.
//
// A token's scale needs the whole row, so the row stays in registers between the maximum and the rounding: a wave, two, four
// or sixteen of them share a row, eight consecutive k a lane and chunk.  The block walks a run of rows with the smoothing vector in
// registers (it is twice a row's bytes) and the next row's x under way; one barrier a row where waves share it, on
// two alternating sets of partial maxima.
//
// A row with a NaN or an infinity gets scale NaN and codes 0, so its outputs are NaN and no other row's are; a row whose
// scale would not be a normal number gets scale 0 and codes 0.
#include "svdq_act.h"
#include "svdq_int8_dev.h"

namespace svdq {

namespace {

// GELU costs 20 vector instructions' time a value (75600 x 13824: 1026 us for what memory gives in 665), but it is a function of 65 536
// values: one block per CU computes them all once, in 128 KB of LDS, and then looks its values up (BY_TABLE; the same function, the same bits).
enum Activation { NO_GELU, GELU, GELU_BY_TABLE };

// W waves share a row of up to 512 W C values; a block has four waves, or sixteen (W = 16, and with the table).
template <int W, int C, int ACT, bool GROUPED>
__global__ __launch_bounds__(W <= 4 && ACT != GELU_BY_TABLE ? 256 : 1024)
void quantize_int8_kernel(const QuantInt8 q, const int run) {
    constexpr int NW = W <= 4 && ACT != GELU_BY_TABLE ? 4 : 16, TEAMS = NW / W;          // teams of W waves, each with rows of its own
    __shared__ uint32_t part[2][NW];
    __shared__ uint32_t table[ACT == GELU_BY_TABLE ? 32768 : 1];      // bf16(gelu(.)) of every bf16 value, two a word
    static_assert(ACT != GELU_BY_TABLE || !GROUPED, "the table's blocks take longer runs than have a lane a row");
    if constexpr (ACT == GELU_BY_TABLE) {
        for (uint32_t i = threadIdx.x; i < 32768; i += 64 * NW) table[i] = gelu_tanh_bf16x2(2 * i | (2 * i + 1) << 16);
        __syncthreads();
    }
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = wave / W, tw = wave % W;
    const int chunks = q.K >> 3;
    int at[C];                                                       // the lane's chunks; those past K repeat the last one
    bool in[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int i = (c * W + tw) * 64 + lane;
        in[c] = i < chunks;
        at[c] = in[c] ? i : chunks - 1;
    }
    const int64_t begin = ((int64_t)blockIdx.x * TEAMS + team) * run;
    const uint16_t* const x = reinterpret_cast<const uint16_t*>(q.x);
    // the run's rows of x and ratios, a lane each
    const int64_t ahead = begin + lane < q.M ? begin + lane : q.M - 1;
    const int tokens = q.rows ? q.rows[ahead] : 0;
    const float ratios = q.row_rho ? q.row_rho[ahead] : q.rho;

    auto load = [&](uint4 (&v)[C], const int i) {                    // the run's i-th row
        int64_t r = begin + i;
        bool none = r >= q.M;
        if (q.rows) {
            r = __builtin_amdgcn_readlane(tokens, i);
            none = none || r < 0 || r >= q.x_rows;                   // no such token: zeros
        }
        if (none) {
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = uint4{0, 0, 0, 0};
            return;
        }
        const uint4* const p = reinterpret_cast<const uint4*>(x + r * q.ldx);
#pragma unroll
        for (int c = 0; c < C; ++c) v[c] = p[at[c]];
    };
    float il[C][8];
    auto load_il = [&](const int e) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const float4v* const p = reinterpret_cast<const float4v*>(q.inv_lambda + (int64_t)e * q.K) + 2 * at[c];
            const float4v a = p[0], b = p[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) il[c][i] = a[i], il[c][4 + i] = b[i];
        }
    };
    uint4 next[C];
    load(next, 0);
    // number of the first offset past the row: it only grows along the run
    int expert = -1, past = 0, past_offset = 0;
    if constexpr (GROUPED) {
        past = first_offset_past(q.groups, begin, lane);
        past_offset = past <= q.groups.E ? q.groups.offsets[past] : 0;
    }
    if (!GROUPED && q.inv_lambda) load_il(0);

    for (int i = 0; i < run; ++i) {
        const int64_t row = begin + i;
        if (W == 1 && row >= q.M) return;                            // teams of one wave have no barrier to keep
        uint4 v[C];
#pragma unroll
        for (int c = 0; c < C; ++c) v[c] = next[c];
        if (i + 1 < run) load(next, i + 1);
        bool owned = row < q.M;
        if constexpr (GROUPED) {
            while (past <= q.groups.E && past_offset <= row)
                if (++past <= q.groups.E) past_offset = q.groups.offsets[past];
            const int e = past - 1;
            owned = owned && e >= 0 && past <= q.groups.E;
            if (owned && e != expert && q.inv_lambda) load_il(e);
            if (owned) expert = e;
        }
        float xs[C][8];
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (ACT == GELU) w[j] = gelu_tanh_bf16x2(w[j]);
                if constexpr (ACT == GELU_BY_TABLE) {
                    const uint16_t* const t = reinterpret_cast<const uint16_t*>(table);
                    w[j] = t[w[j] & 0xffff] | (uint32_t)t[w[j] >> 16] << 16;
                }
                xs[c][2 * j] = bf16lo_f(w[j]);
                xs[c][2 * j + 1] = bf16hi_f(w[j]);
            }
            if (q.inv_lambda)
#pragma unroll
                for (int j = 0; j < 8; ++j) xs[c][j] = __fmul_rn(xs[c][j], il[c][j]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {                            // magnitudes as bit patterns: a NaN is the largest
                const uint32_t m = f_bits(xs[c][j]) & 0x7fffffffu;
                top = m > top ? m : top;
            }
        }
        top = wave_max(top);
        if constexpr (W > 1) {
            if (lane == 0) part[i & 1][wave] = top;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const uint32_t o = part[i & 1][team * W + k];
                top = o > top ? o : top;
            }
        }
        if (!owned) continue;
        float s, inv;
        const bool fine = row_scale(top, q.row_rho ? bits_f((uint32_t)__builtin_amdgcn_readlane((int)f_bits(ratios), i)) : q.rho, s, inv);
        if (lane == 0 && tw == 0) q.sx[row] = s;
        int8_t* const out = q.qx + row * q.K;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const uint2 o = codes8(xs[c], inv, fine);
            if (in[c]) reinterpret_cast<uint2*>(out)[at[c]] = o;
        }
    }
}

template <int W, int C>
hipError_t launch_rows(const QuantInt8& q, const bool gelu, hipStream_t stream) {
    constexpr int TEAMS = W <= 4 ? 4 / W : 1, THREADS = W <= 4 ? 256 : 64 * W;
    // Up to 2048 blocks, eight a CU, then longer runs of rows, of 16 at most (a lane holds each row's token and ratio); beyond those, more blocks.  Eight
    // are there at once where a lane has one chunk or two.  The registers of three leave room for five, of four for four, of five (32760 x 5120) for three and
    // of seven for two, and sixteen waves have a CU to themselves: there blocks wait for a place.  Rounded up, since a few blocks more than places are a
    // round more (grouped 25786 x 2832 in 1075 blocks of a place for 1024 50.6 us, in 992 39.3).  Grouped, a block begins with its expert, token and
    // smoothing vector one after the other: with few rows an expert 1024 blocks (128 rows each of K = 2048: 17.3 us, with 2048 19.3; 16380 of K = 5120: 113.7
    // and 105.2).
    const bool four = q.groups.offsets && q.M / q.groups.E < 1024;
    const int64_t teams = (int64_t)TEAMS * (four ? 1024 : 2048);
    int64_t run = (q.M + teams - 1) / teams;
    run = run > 16 ? 16 : run;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)((q.M + TEAMS * run - 1) / (TEAMS * run))), dim3(THREADS), 0, stream, q, (int)run);
        return hipGetLastError();
    };
    if (q.groups.offsets) return gelu ? go(quantize_int8_kernel<W, C, GELU, true>) : go(quantize_int8_kernel<W, C, NO_GELU, true>);
    return gelu ? go(quantize_int8_kernel<W, C, GELU, false>) : go(quantize_int8_kernel<W, C, NO_GELU, false>);
}

template <int W, int C>
hipError_t launch_by_table(const QuantInt8& q, hipStream_t stream) {
    constexpr int TEAMS = 16 / W;
    const int64_t run = (q.M + TEAMS * 256 - 1) / (TEAMS * 256);
    hipLaunchKernelGGL((quantize_int8_kernel<W, C, GELU_BY_TABLE, false>), dim3((uint32_t)((q.M + TEAMS * run - 1) / (TEAMS * run))), dim3(1024), 0, stream, q, (int)run);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_int8(const QuantInt8& q, bool gelu, hipStream_t stream) {
    const int chunks = q.K >> 3;
    if (gelu && !q.groups.offsets && q.M * q.K >= (int64_t)1 << 27) {        // the table takes a block 10 us
        if (chunks <= 64) return launch_by_table<1, 1>(q, stream);
        if (chunks <= 128) return launch_by_table<1, 2>(q, stream);
        if (chunks <= 256) return launch_by_table<1, 4>(q, stream);
        if (chunks <= 512) return launch_by_table<4, 2>(q, stream);
        if (chunks <= 768) return launch_by_table<4, 3>(q, stream);
        if (chunks <= 1024) return launch_by_table<4, 4>(q, stream);
        if (chunks <= 2048) return launch_by_table<16, 2>(q, stream);
        return launch_by_table<16, 4>(q, stream);
    }
    if (chunks <= 64) return launch_rows<1, 1>(q, gelu, stream);
    if (chunks <= 128) return launch_rows<1, 2>(q, gelu, stream);
    if (q.M >= 2048) {
        // A row costs each of its waves the maximum's exchange and two divisions, as much as sixteen values a lane: few waves, many values.
        if (chunks <= 192) return launch_rows<1, 3>(q, gelu, stream);
        if (chunks <= 256) return launch_rows<1, 4>(q, gelu, stream);
        if (chunks <= 512) return launch_rows<2, 4>(q, gelu, stream);
        if (chunks <= 640) return launch_rows<2, 5>(q, gelu, stream);
        if (chunks <= 1024) return launch_rows<4, 4>(q, gelu, stream);
        if (chunks <= 1280) return launch_rows<4, 5>(q, gelu, stream);
        if (chunks <= 1792) return launch_rows<4, 7>(q, gelu, stream);
    }
    // few rows: what counts is one row's time
    if (chunks <= 256) return launch_rows<4, 1>(q, gelu, stream);
    if (chunks <= 512) return launch_rows<4, 2>(q, gelu, stream);
    if (chunks <= 768) return launch_rows<4, 3>(q, gelu, stream);
    if (chunks <= 2048) return launch_rows<16, 2>(q, gelu, stream);
    return launch_rows<16, 4>(q, gelu, stream);
}

}  // namespace svdq
