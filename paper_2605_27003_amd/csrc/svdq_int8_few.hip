// The product of the 8-bit layer for few tokens, where what counts is how fast the weights come from memory.
//
// A block owns 16 channels by 16, 32 or 64 tokens (D[n][m], as in the tile kernels), and its waves split K: wave w takes the 128-byte stages w,
// w + waves, ... of every row, so that the waves together read runs of each weight row.  Every wave has a ring of its own in LDS, filled by
// direct transfers DEPTH stages ahead, and waits for nobody: no barrier stands in the loop, and what is in flight costs no registers.
// (Operands straight to registers would be sixteen rows' pieces a load, a line for every lane; transfers move whole lines, eight lanes a row.)
// The partial sums, exact integers in any order, meet in LDS at the end.
#include "svdq_int8_dev.h"

namespace svdq {

namespace {

template <int TOK, int NW, int DEPTH, bool TAIL, bool GROUPED, class T>
__global__ __launch_bounds__(64 * NW)
void gemm_int8_few_kernel(const GemmInt8 g, const TileGrid tg) {
    constexpr int BN = 16, TT = TOK / 16, NA = TOK / 8, NB = BN / 8, ND = NA + NB, OUT = TOK * BN / (64 * NW);
    constexpr uint32_t STAGE = (TOK + BN) * BK, SUMS = TT * 64 * 16;  // of a wave
    static_assert(DEPTH * STAGE >= SUMS && OUT >= 1, "the sums meet where the rings stood");
    __shared__ __attribute__((aligned(16))) uint8_t ring[NW * DEPTH * STAGE];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane & 15, lk = lane >> 4;
    const int K = g.K, N = g.N;
    TilePlace at;
    if (!tile_place<TOK, BN, GROUPED>(g, tg, blockIdx.x, lane, at)) return;
    const int m0 = at.m0, rows = at.m_end - at.m0, n0 = at.n0, cols = N - n0;
    const uint32_t mine = (uint32_t)(uintptr_t)(lds_byte*)ring + wave * DEPTH * STAGE;
    const int nstages = (K + BK - 1) / BK, count = (nstages - wave + NW - 1) / NW;       // of this wave

    // this thread's outputs: token o / 16, channel o % 16 of the tile for o = tid + i 64 NW
    float ts[OUT], cs, cb;
    {
        const int n = tid & 15, c = n < cols ? n : cols - 1;
        cs = at.sw[n0 + c];
        cb = at.bias ? at.bias[n0 + c] : 0.0f;
#pragma unroll
        for (int i = 0; i < OUT; ++i) {
            const int m = (tid >> 4) + i * 4 * NW;
            ts[i] = g.sx[m0 + (m < rows ? m : rows - 1)];
        }
    }

    // ---- transfers: eight rows each, the tokens' first; rows past the end repeat the last one
    const int8_t* const abase = g.qx + (int64_t)m0 * K;
    const int8_t* const wbase = at.qw + (int64_t)n0 * K;
    uint32_t v[ND], piece[ND];
#pragma unroll
    for (int j = 0; j < ND; ++j) {
        const int row = 8 * (j < NA ? j : j - NA) + (lane >> 3), last = (j < NA ? rows : cols) - 1;
        piece[j] = (lane & 7) ^ ((row >> 1) & 7);                     // piece c of row r stands at place c ^ (r / 2) % 8
        v[j] = (uint32_t)(row < last ? row : last) * (uint32_t)K + piece[j] * 16;
    }
    auto request = [&](const int i, const uint32_t slot) {            // this wave's i-th stage
        const int s = wave + i * NW;
#pragma unroll
        for (int j = 0; j < ND; ++j) {
            uint32_t o = v[j];
            if constexpr (TAIL) {
                const int left = (K >> 4) - 8 * s - 1, over = (int)piece[j] - left;
                if (over > 0) o -= over * 16;
            }
            dma16((j < NA ? abase : wbase) + (int64_t)s * BK, o, slot + j * 1024);
        }
    };
    const uint32_t turn = (lk ^ (li >> 1)) & 7;
    int4v acc[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t] = int4v{0, 0, 0, 0};

    // The scales above are loads too: awaited here, so that the waits below count transfers alone.
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(cs), "+v"(cb), "+v"(ts[0]) :: "memory");
    for (int i = 0; i < DEPTH; ++i)
        if (i < count) request(i, mine + i * STAGE);
    uint32_t slot = mine;
    typedef const volatile __attribute__((address_space(3))) int4v lds_i4;
    for (int i = 0; i < count; ++i) {
        const int behind = count - 1 - i < DEPTH - 1 ? count - 1 - i : DEPTH - 1;        // stages requested after this one
        if (behind >= 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * ND) : "memory");
        else if (behind == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * ND) : "memory");
        else if (behind == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        int4v w[2], x[2][TT];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const uint32_t p = slot + li * BK + ((turn ^ (4 * kk)) << 4);
            w[kk] = *reinterpret_cast<lds_i4*>((lds_byte*)(uintptr_t)p + TOK * BK);
            if constexpr (TAIL) {
                if (8 * (wave + i * NW) + 4 * kk + lk >= (K >> 4)) w[kk] = int4v{0, 0, 0, 0};
            }
#pragma unroll
            for (int t = 0; t < TT; ++t) x[kk][t] = *reinterpret_cast<lds_i4*>((lds_byte*)(uintptr_t)p + t * 16 * BK);
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[kk], x[kk][t], acc[t], 0, 0, 0);
        if (i + DEPTH < count) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // the operands are out of the place
            request(i + DEPTH, slot);
        }
        slot = slot == mine + (DEPTH - 1) * STAGE ? mine : slot + STAGE;
    }
    static_assert(DEPTH <= 4, "the waits above");

    // ---- every wave's sums, lane by lane, at the start of its ring; then one thread an output
#pragma unroll
    for (int t = 0; t < TT; ++t)
        *reinterpret_cast<__attribute__((address_space(3))) int4v*>((lds_byte*)(uintptr_t)(mine + (t * 64 + lane) * 16)) = acc[t];
    __syncthreads();
    const int n = tid & 15;
    T* const y = reinterpret_cast<T*>(g.y) + (int64_t)m0 * g.ldy + n0 + n;
#pragma unroll
    for (int i = 0; i < OUT; ++i) {
        const int m = (tid >> 4) + i * 4 * NW;
        const uint32_t from = (uint32_t)(uintptr_t)(lds_byte*)ring + (((m >> 4) * 64 + (m & 15) + 16 * (n >> 2)) * 4 + (n & 3)) * 4;
        int sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += (int)lds_read4(from + w * DEPTH * STAGE);
        const float r = ((float)sum * ts[i]) * cs + cb;
        if (m < rows && n < cols) {
            if constexpr (sizeof(T) == 2) y[(int64_t)m * g.ldy] = (T)f_bf16_rne(r);
            else y[(int64_t)m * g.ldy] = f_bits(r);
        }
    }
}

template <int TOK, int NW, int DEPTH>
hipError_t launch(const GemmInt8& g, const bool out_f32, hipStream_t stream) {
    const int ntiles = (g.N + 15) / 16;
    const bool grouped = g.groups.offsets != nullptr;
    const TileGrid tg = grouped ? TileGrid{0, ntiles, 0, 0} : make_tile_grid((int)((g.M + TOK - 1) / TOK), ntiles);
    const int blocks = grouped ? grouped_blocks(g, TOK, 16) : tile_ids(tg);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * NW), 0, stream, g, tg); };
    auto typed = [&](auto TAILC, auto GROUPEDC) {
        constexpr bool TAIL = decltype(TAILC)::value, GROUPED = decltype(GROUPEDC)::value;
        if (out_f32) go(gemm_int8_few_kernel<TOK, NW, DEPTH, TAIL, GROUPED, uint32_t>);
        else go(gemm_int8_few_kernel<TOK, NW, DEPTH, TAIL, GROUPED, uint16_t>);
    };
    if (g.K % BK) grouped ? typed(IC<1>{}, IC<1>{}) : typed(IC<1>{}, IC<0>{});
    else grouped ? typed(IC<0>{}, IC<1>{}) : typed(IC<0>{}, IC<0>{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_int8_few(const GemmInt8& g, const int tokens, bool out_f32, hipStream_t stream) {
    if (tokens <= 16) return launch<16, 4, 4>(g, out_f32, stream);
    if (tokens <= 32) return launch<32, 4, 4>(g, out_f32, stream);
    return launch<64, 4, 3>(g, out_f32, stream);
}

}  // namespace svdq
