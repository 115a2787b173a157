// The 8-bit layer: what its kernels (svdq_int8_*.hip) offer the C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace svdq {

// Rows and experts of a grouped call.  offsets: E + 1 row numbers on the device, read as their running maximum and within
// [0, M], so that whatever they hold an expert's rows are a span of [0, M] and no row has two experts.
struct Groups {
    const int32_t* offsets;      // null: one expert, all rows
    int E;
};

struct QuantInt8 {
    const void* x;               // [x_rows, ldx] bf16
    int64_t ldx;
    const int32_t* rows;         // row i of the codes is row rows[i] of x (null: row i)
    int64_t x_rows;
    const float* inv_lambda;     // [K], or [E, K] (null: ones)
    const float* row_rho;        // [M] (null: rho)
    float rho;
    int K;
    int64_t M;
    int8_t* qx;                  // [M, K]
    float* sx;                   // [M]
    Groups groups;
};
hipError_t launch_quantize_int8(const QuantInt8& q, bool gelu, hipStream_t stream);

struct GemmInt8 {
    const int8_t* qx;            // [M, K]
    const float* sx;             // [M]
    const int8_t* qw;            // [E, N, K]
    const float* sw;             // [E, N]
    const float* bias;           // [E, N] or null
    void* y;                     // [M, ldy] bf16 or binary32
    int64_t ldy, M;
    int N, K;
    Groups groups;
};
struct Int8Plan;
struct Int8Kernel;
hipError_t launch_gemm_int8(const GemmInt8& g, const Int8Plan& p, bool out_f32, hipStream_t stream);
hipError_t launch_gemm_int8_few(const GemmInt8& g, const Int8Kernel& k, bool out_f32, hipStream_t stream);     // the few-token kernel's tiles

// Both halves in one launch, for layers that fit it (bf16 outputs).  x and y share no memory.
bool layer_int8_fits(const GemmInt8& g);
hipError_t launch_layer_int8(const QuantInt8& q, const GemmInt8& g, bool gelu, hipStream_t stream);

}  // namespace svdq
