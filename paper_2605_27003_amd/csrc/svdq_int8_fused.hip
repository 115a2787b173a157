// A whole 8-bit layer in one launch, where it is so small that the host's launches are what it takes: few tiles and a short K.
//
// A block owns 16 tokens by 32 channels, as in the few-token kernel, and makes its tokens' codes itself, for all of K, into LDS (a row a wave, the
// quantise pass's arithmetic); the first stages of its weights are on their way meanwhile.  The work done again by every channel tile's block (16 K
// values from L2) costs what the second kernel's start did (replayed from a graph 256 tokens, K = N = 512 take 5.9 us, and 5.7 in two
// kernels), and the host, which such layers wait for, 6.9 us a call instead of 10.6.  The codes stay on the chip, unless the caller has memory
// for them: then the blocks of the first channel tile write the codes and scales that the two launches leave (8.3 us a call, since torch's allocator takes
// 1.4 to find the memory).
#include "svdq_act.h"
#include "svdq_int8_dev.h"

namespace svdq {

namespace {

constexpr int TOK = 16, BN = 32, NW = 4, DEPTH = 3, CT = BN / 16;

template <int KMAX, bool GELU, bool GROUPED>
__global__ __launch_bounds__(64 * NW)
void layer_int8_kernel(const QuantInt8 q, const GemmInt8 g) {
    constexpr int NB = BN / 8, C = (KMAX + 511) / 512;
    constexpr uint32_t STAGE = BN * BK, CODES = TOK * KMAX, SUMS = CT * 64 * 16;
    constexpr uint32_t OFF_RING = CODES, OFF_SUMS = OFF_RING + NW * DEPTH * STAGE, OFF_SCALES = OFF_SUMS + NW * SUMS;
    __shared__ __attribute__((aligned(16))) uint8_t lds[OFF_SCALES + 3 * 256];           // tokens', channels' scales, biases

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane & 15, lk = lane >> 4;
    const int K = g.K, N = g.N;
    TilePlace at;
    if (!typename TilesOf<GROUPED, TOK, BN>::type(g, lane).place(g, blockIdx.x, at)) return;
    const int m0 = at.m0, rows = at.m_end - m0 < TOK ? at.m_end - m0 : TOK, cols = N - at.n0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)lds, mine = lds0 + OFF_RING + wave * DEPTH * STAGE;
    const int nstages = (K + BK - 1) / BK, count = (nstages - wave + NW - 1) / NW;       // of this wave

    // ---- weights: eight rows a transfer; rows past the end repeat the last one, the last stage's pieces beyond K the row's last piece
    const int8_t* const wbase = at.qw + (int64_t)at.n0 * K;
    auto request = [&](const int i, const uint32_t slot) {            // this wave's i-th stage
        const int s = wave + i * NW, left = (K >> 4) - 8 * s - 1;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int row = 8 * j + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);  // piece c of row r stands at place c ^ (r / 2) % 8
            dma16(wbase + (int64_t)s * BK, (uint32_t)(row < cols - 1 ? row : cols - 1) * (uint32_t)K + (piece < left ? piece : left) * 16, slot + j * 1024);
        }
    };
    if (wave == 0) {
        const uint32_t ch = lane < cols ? lane : cols - 1;
        dma4(at.sw + at.n0, ch * 4, lds0 + OFF_SCALES + 256);
        if (at.bias) dma4(at.bias + at.n0, ch * 4, lds0 + OFF_SCALES + 512);
    }
    for (int i = 0; i < DEPTH; ++i)
        if (i < count) request(i, mine + i * STAGE);

    // ---- codes of the tile's tokens: rows wave, wave + 4, ...
    {
        const bool keep = q.qx && at.n0 == 0;
        const int chunks = K >> 3;
        const float* const il = q.inv_lambda ? q.inv_lambda + (at.qw - g.qw) / N : nullptr;           // its expert's: e N K / N
        int at_c[C];
        bool in[C];
        float lam[C][8];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            in[c] = c * 64 + lane < chunks;
            at_c[c] = in[c] ? c * 64 + lane : chunks - 1;
            if (il) {
                const float4v a = reinterpret_cast<const float4v*>(il)[2 * at_c[c]], b = reinterpret_cast<const float4v*>(il)[2 * at_c[c] + 1];
#pragma unroll
                for (int j = 0; j < 4; ++j) lam[c][j] = a[j], lam[c][4 + j] = b[j];
            }
        }
        auto load = [&](uint4 (&v)[C], const int r) {
            int64_t row = m0 + r;
            bool none = r >= rows;
            if (!none && q.rows) {
                row = q.rows[row];
                none = row < 0 || row >= q.x_rows;                    // no such token: zeros
            }
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = none ? uint4{0, 0, 0, 0} : reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(q.x) + row * q.ldx)[at_c[c]];
        };
        uint4 next[C];
        load(next, wave);
        for (int r = wave; r < rows; r += NW) {
            uint4 v[C];
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = next[c];
            load(next, r + NW);
            float xs[C][8];
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (GELU) w[j] = gelu_tanh_bf16x2(w[j]);
                    xs[c][2 * j] = bf16lo_f(w[j]);
                    xs[c][2 * j + 1] = bf16hi_f(w[j]);
                }
                if (il)
#pragma unroll
                    for (int j = 0; j < 8; ++j) xs[c][j] = __fmul_rn(xs[c][j], lam[c][j]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t m = f_bits(xs[c][j]) & 0x7fffffffu;
                    top = m > top ? m : top;
                }
            }
            float s, inv;
            const bool fine = row_scale(wave_max(top), q.row_rho ? q.row_rho[m0 + r] : q.rho, s, inv);
            if (lane == 0) *reinterpret_cast<__attribute__((address_space(3))) float*>((lds_byte*)(uintptr_t)(lds0 + OFF_SCALES + r * 4)) = s;
            if (lane == 0 && keep) q.sx[m0 + r] = s;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint2 o = codes8(xs[c], inv, fine);
                if (!in[c]) continue;
                const int k8 = at_c[c], stage = k8 >> 4, piece = (k8 >> 1) & 7;          // eight k each: stages of sixteen, pieces of two
                lds_write8_pinned(lds0 + (stage * TOK + r) * BK + ((piece ^ ((r >> 1) & 7)) << 4) + (k8 & 1) * 8, o);
                if (keep) reinterpret_cast<uint2*>(q.qx + (int64_t)(m0 + r) * K)[k8] = o;
            }
        }
    }
    // Everything so far has arrived, whatever waits the loads above came with; from here on the waits count transfers.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    // ---- the products: as in the few-token kernel, the tokens' operands from the codes.  (Rows past the last, and pieces beyond K, hold anything:
    // the former's results are not stored, the latter meet zeros.)
    const uint32_t turn = (lk ^ (li >> 1)) & 7;
    int4v acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = int4v{0, 0, 0, 0};
    uint32_t slot = mine;
    typedef const volatile __attribute__((address_space(3))) int4v lds_i4;
    for (int i = 0; i < count; ++i) {
        const int s = wave + i * NW;
        if (i >= DEPTH) {                                             // the first ones are there
            const int behind = count - 1 - i < DEPTH - 1 ? count - 1 - i : DEPTH - 1;
            if (behind == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NB) : "memory");
            else if (behind == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NB) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        static_assert(DEPTH == 3, "the waits above");
        int4v w[2][CT], x[2];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const uint32_t from = li * BK + ((turn ^ (4 * kk)) << 4);
            const bool past = 8 * s + 4 * kk + lk >= (K >> 4);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                w[kk][c] = *reinterpret_cast<lds_i4*>((lds_byte*)(uintptr_t)(slot + from) + c * 16 * BK);
                if (past) w[kk][c] = int4v{0, 0, 0, 0};
            }
            x[kk] = *reinterpret_cast<lds_i4*>((lds_byte*)(uintptr_t)(lds0 + s * TOK * BK + from));
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[kk][c], x[kk], acc[c], 0, 0, 0);
        if (i + DEPTH < count) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // the operands are out of the place that the request fills
            request(i + DEPTH, slot);
        }
        slot = slot == mine + (DEPTH - 1) * STAGE ? mine : slot + STAGE;
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
        *reinterpret_cast<__attribute__((address_space(3))) int4v*>((lds_byte*)(uintptr_t)(lds0 + OFF_SUMS + wave * SUMS + (c * 64 + lane) * 16)) = acc[c];
    __syncthreads();
    const int n = tid % BN;
    const uint32_t scales = lds0 + OFF_SCALES;
    const float cs = bits_f(lds_read4(scales + 256 + n * 4)), cb = at.bias ? bits_f(lds_read4(scales + 512 + n * 4)) : 0.0f;
    uint16_t* const y = reinterpret_cast<uint16_t*>(g.y) + (int64_t)m0 * g.ldy + at.n0 + n;
#pragma unroll
    for (int i = 0; i < TOK * BN / (64 * NW); ++i) {
        const int m = tid / BN + i * (64 * NW / BN);
        const uint32_t from = lds0 + OFF_SUMS + (((n >> 4) * 64 + m + 16 * ((n & 15) >> 2)) * 4 + (n & 3)) * 4;
        int sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += (int)lds_read4(from + w * SUMS);
        const float r = output(sum, bits_f(lds_read4(scales + m * 4)), cs, cb);
        if (m < rows && n < cols) y[(int64_t)m * g.ldy] = (uint16_t)f_bf16_rne(r);
    }
}

template <int KMAX>
void launch(const QuantInt8& q, const GemmInt8& g, const bool gelu, const int blocks, hipStream_t stream) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * NW), 0, stream, q, g); };
    if (g.groups.offsets) gelu ? go(layer_int8_kernel<KMAX, true, true>) : go(layer_int8_kernel<KMAX, false, true>);
    else gelu ? go(layer_int8_kernel<KMAX, true, false>) : go(layer_int8_kernel<KMAX, false, false>);
}

}  // namespace

// Up to two blocks for every CU, with a K that lets two of them have one's LDS (16 tokens, N = 5120, K = 1024: 7.5 us, 10.5 in two launches); a longer
// one with a row for each wave (one token, K = N = 4096: 7.1 and 10.1; but 16 tokens 13.8 and 10.1).
bool layer_int8_fits(const GemmInt8& g) {
    return (g.K <= 1408 || (g.K <= 4096 && g.M <= NW)) && int8_tiles(g.M, g.N, g.groups.offsets ? g.groups.E : 0, TOK, BN) <= 512;
}

hipError_t launch_layer_int8(const QuantInt8& q, const GemmInt8& g, const bool gelu, hipStream_t stream) {
    const int blocks = most_tiles(g, TOK, BN);
    // two blocks fit a CU's LDS up to K = 1408
    if (g.K <= 512) launch<512>(q, g, gelu, blocks, stream);
    else if (g.K <= 1408) launch<1408>(q, g, gelu, blocks, stream);
    else launch<4096>(q, g, gelu, blocks, stream);
    return hipGetLastError();
}

}  // namespace svdq
