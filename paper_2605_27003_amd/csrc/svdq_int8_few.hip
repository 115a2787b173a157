// The product of the 8-bit layer for few tokens, where what counts is how fast the weights come from memory.
//
// A block owns a tile of 16 or 32 tokens by 16 or 32 channels (D[n][m], as in the tile kernels), and its waves split K: wave w takes the
// 128-byte stages w, w + NW, ... of every row, so that the waves together read runs of each weight row.  Every wave has a ring of its own in
// LDS, filled by direct transfers DEPTH stages ahead, and waits for nobody: no barrier stands between stages, and what is in flight costs no
// registers.  (Operands straight to registers would be sixteen rows' pieces a load: 38 bytes a ns a CU from L2 where transfers of
// whole lines, eight lanes a row, reach 135.)  Blocks walk the tiles: a wave's requests run on into its next tiles while sums are added up and
// stored, since with a short K a tile is little more than its start.  The partial sums, exact integers in any order, meet in LDS.
//
// Times here are of calls that find their weights in the 256 MB memory-side cache, left there by the call before.  Where every call has weights of its
// own, as the layers of a model have: 157 MB for one token 28.1 us for 23.2 (5.6 TB/s), 26 MB for 24 tokens 10.1 for 6.8, replayed from a graph.
#include "svdq_int8_dev.h"
#include "svdq_int8_plan.h"

namespace svdq {

namespace {

constexpr int CUS = 256;

template <int TOK, int BN, int NW, int DEPTH, bool TAIL, bool GROUPED, class T>
__global__ __launch_bounds__(64 * NW)
void gemm_int8_few_kernel(const GemmInt8 g, const int walkers) {
    constexpr int TT = TOK / 16, CT = BN / 16, NA = TOK / 8, NB = BN / 8, ND = NA + NB, OUT = (TOK * BN + 64 * NW - 1) / (64 * NW), ROWS = 64 * NW / BN;
    constexpr uint32_t STAGE = (TOK + BN) * BK, SUMS = CT * TT * 64 * 16, SCALES = 3 * 256;
    // rings; then every wave's sums; then the scales and biases of a tile, of the DEPTH that requests can be ahead, and of the one before, which
    // other waves may still be storing
    constexpr uint32_t OFF_SUMS = NW * DEPTH * STAGE, OFF_SCALES = OFF_SUMS + NW * SUMS;
    __shared__ __attribute__((aligned(16))) uint8_t lds[OFF_SCALES + (DEPTH + 2) * SCALES];
    static_assert(DEPTH >= 2 && DEPTH <= 4, "the waits below");

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane & 15, lk = lane >> 4;
    const int K = g.K, N = g.N;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)lds, mine = lds0 + wave * DEPTH * STAGE;
    const int nstages = (K + BK - 1) / BK, count = (nstages - wave + NW - 1) / NW;       // a tile's stages of this wave

    const typename TilesOf<GROUPED, TOK, BN>::type tiles(g, lane);

    // ---- requests: eight rows each, the tokens' first; rows past the end repeat the last one.  Ahead of a tile's first, wave 0 asks for its scales.
    int rid = blockIdx.x, rstage = 0, rtile = 0;                      // what is requested next
    const int8_t *abase = nullptr, *wbase = nullptr;
    uint32_t v[ND], rslot = mine;
    const uint32_t piece[2] = {(uint32_t)((lane & 7) ^ (lane >> 4)), (uint32_t)((lane & 7) ^ (4 + (lane >> 4)))};    // piece c of row r stands at place c ^ (r / 2) % 8
    bool more = true;
    auto request = [&] {
        if (rstage == 0) {
            TilePlace p;
            more = more && tiles.place(g, rid, p);                    // (where a block has no tile it has none behind it)
            if (!more) return;
            const int rows = p.m_end - p.m0, cols = N - p.n0;
            abase = g.qx + (int64_t)p.m0 * K;
            wbase = p.qw + (int64_t)p.n0 * K;
#pragma unroll
            for (int j = 0; j < ND; ++j) {
                const int row = 8 * (j < NA ? j : j - NA) + (lane >> 3), last = (j < NA ? rows : cols) - 1;
                v[j] = (uint32_t)(row < last ? row : last) * (uint32_t)K + piece[j & 1] * 16;
            }
            if (wave == 0) {
                const uint32_t to = lds0 + OFF_SCALES + rtile * SCALES;
                const uint32_t tok = lane < rows ? lane : rows - 1, ch = lane < cols ? lane : cols - 1;
                dma4(g.sx + p.m0, tok * 4, to);
                dma4(p.sw + p.n0, ch * 4, to + 256);
                if (p.bias) dma4(p.bias + p.n0, ch * 4, to + 512);
            }
        }
        const int s = wave + rstage * NW;
#pragma unroll
        for (int j = 0; j < ND; ++j) {
            uint32_t o = v[j];
            if constexpr (TAIL) {
                const int left = (K >> 4) - 8 * s - 1, over = (int)piece[j & 1] - left;
                if (over > 0) o -= over * 16;
            }
            dma16((j < NA ? abase : wbase) + (int64_t)s * BK, o, rslot + j * 1024);
        }
        rslot = rslot == mine + (DEPTH - 1) * STAGE ? mine : rslot + STAGE;
        if (++rstage == count) {
            rstage = 0;
            rid += walkers;
            rtile = rtile == DEPTH + 1 ? 0 : rtile + 1;
        }
    };
    static_assert(NA % 2 == 0 && NB % 2 == 0, "a transfer's rotation goes by its number's parity");

    int ahead = 0;                                                    // stages requested and not yet read
    if (count > 0)
        for (int i = 0; i < DEPTH; ++i) {
            request();
            ahead += more;
        }
    const uint32_t turn = (lk ^ (li >> 1)) & 7;
    uint32_t slot = mine;
    typedef const volatile __attribute__((address_space(3))) int4v lds_i4;
    TilePlace p;
    int tile = 0;
    for (int id = blockIdx.x; tiles.place(g, id, p); id += walkers) {
        int4v acc[CT][TT];
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[c][t] = int4v{0, 0, 0, 0};
        for (int i = 0; i < count; ++i) {
            // transfers of `ahead` - 1 stages stand behind the awaited one's (and stores and scales: the waits hold for at least what they name)
            if (ahead >= 4) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * ND) : "memory");
            else if (ahead == 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * ND) : "memory");
            else if (ahead == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            int4v w[2][CT], x[2][TT];
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const uint32_t from = slot + li * BK + ((turn ^ (4 * kk)) << 4);
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    w[kk][c] = *reinterpret_cast<lds_i4*>((lds_byte*)(uintptr_t)from + (TOK + c * 16) * BK);
                    if constexpr (TAIL) {
                        if (8 * (wave + i * NW) + 4 * kk + lk >= (K >> 4)) w[kk][c] = int4v{0, 0, 0, 0};
                    }
                }
#pragma unroll
                for (int t = 0; t < TT; ++t) x[kk][t] = *reinterpret_cast<lds_i4*>((lds_byte*)(uintptr_t)from + t * 16 * BK);
            }
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int t = 0; t < TT; ++t)
#pragma unroll
                    for (int c = 0; c < CT; ++c) acc[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[kk][c], x[kk][t], acc[c][t], 0, 0, 0);
            slot = slot == mine + (DEPTH - 1) * STAGE ? mine : slot + STAGE;
            --ahead;
            if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // the operands are out of the place that the request fills
                request();
                ahead += more;
            }
        }
        // ---- every wave's sums, lane by lane; then one thread an output.  Wave 0 has waited for transfers behind the tile's scales.
        __syncthreads();                                              // the previous tile's sums are read
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int t = 0; t < TT; ++t)
                *reinterpret_cast<__attribute__((address_space(3))) int4v*>((lds_byte*)(uintptr_t)(lds0 + OFF_SUMS + wave * SUMS + ((c * TT + t) * 64 + lane) * 16)) = acc[c][t];
        __syncthreads();
        const int rows = p.m_end - p.m0, cols = N - p.n0, n = tid % BN;
        const uint32_t scales = lds0 + OFF_SCALES + tile * SCALES;
        const float cs = bits_f(lds_read4(scales + 256 + n * 4)), cb = p.bias ? bits_f(lds_read4(scales + 512 + n * 4)) : 0.0f;
        T* const y = reinterpret_cast<T*>(g.y) + (int64_t)p.m0 * g.ldy + p.n0 + n;
#pragma unroll
        for (int i = 0; i < OUT; ++i) {
            const int m = tid / BN + i * ROWS;
            if (m >= TOK) break;                                      // more threads than outputs
            const uint32_t from = lds0 + OFF_SUMS + ((((n >> 4) * TT + (m >> 4)) * 64 + (m & 15) + 16 * ((n & 15) >> 2)) * 4 + (n & 3)) * 4;
            int sum = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) sum += (int)lds_read4(from + w * SUMS);
            const float r = output(sum, bits_f(lds_read4(scales + m * 4)), cs, cb);
            if (m < rows && n < cols) {
                if constexpr (sizeof(T) == 2) y[(int64_t)m * g.ldy] = (T)f_bf16_rne(r);
                else y[(int64_t)m * g.ldy] = f_bits(r);
            }
        }
        tile = tile == DEPTH + 1 ? 0 : tile + 1;
    }
}

template <int TOK, int BN, int NW, int DEPTH>
hipError_t launch(const GemmInt8& g, const bool out_f32, hipStream_t stream) {
    const bool grouped = g.groups.offsets != nullptr;
    const int most = most_tiles(g, TOK, BN), walkers = most < 2 * CUS ? most : 2 * CUS;  // multiples of 256, as tile_number asks
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(walkers), dim3(64 * NW), 0, stream, g, walkers); };
    auto typed = [&](auto TAILC, auto GROUPEDC) {
        constexpr bool TAIL = decltype(TAILC)::value, GROUPED = decltype(GROUPEDC)::value;
        if (out_f32) go(gemm_int8_few_kernel<TOK, BN, NW, DEPTH, TAIL, GROUPED, uint32_t>);
        else go(gemm_int8_few_kernel<TOK, BN, NW, DEPTH, TAIL, GROUPED, uint16_t>);
    };
    if (g.K % BK) grouped ? typed(IC<1>{}, IC<1>{}) : typed(IC<1>{}, IC<0>{});
    else grouped ? typed(IC<0>{}, IC<1>{}) : typed(IC<0>{}, IC<0>{});
    return hipGetLastError();
}

}  // namespace

// Thirty-two channels a block halve the tokens' transfers (24 tokens, 5120 x 5120: 7.8 against 9.2 us); sixteen, on eight waves, where there
// are few blocks (one token, N = 1024, K = 13824: 5.6 against 7.4 us).
hipError_t launch_gemm_int8_few(const GemmInt8& g, const Int8Kernel& k, bool out_f32, hipStream_t stream) {
    switch (k.tiles) {
        case Int8Tiles::FEW_16x16: return launch<16, 16, 8, 2>(g, out_f32, stream);
        case Int8Tiles::FEW_16x32: return launch<16, 32, 4, 2>(g, out_f32, stream);
        case Int8Tiles::FEW_32x16: return launch<32, 16, 8, 2>(g, out_f32, stream);
        default: return launch<32, 32, 4, 2>(g, out_f32, stream);
    }
}

}  // namespace svdq
