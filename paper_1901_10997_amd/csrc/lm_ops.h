// Launchers of the operators around the cells (gated linear recurrence, RMS norm, 8-bit product, sampling); lm_ops.cpp
// checks the arguments of the C entries and calls them.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace l355 {

// Records `msg` as what lstm_last_error(NULL) returns and gives back `code`; never throws (lstm355.cpp).
int op_error(int code, const char* msg) noexcept;

constexpr int kScaleCols = 128;             // columns that share a scale of an 8-bit operand
constexpr float kE4m3Max = 448.f;
constexpr float kSmallestScale = 0x1p-126f; // scale of a block of zeros, and of one whose own would be subnormal

// ---- gated linear recurrence (scan_kernels.hip)
constexpr int kScanSteps = 16;              // steps of one thread; the forward keeps the state in front of each such run
struct ScanArgs {
    int T, B, H, bf16, reverse;
    const void* P;                          // [T, B, 4H]
    int64_t P_t, P_b;
    const int* lengths;
    const float* c0;                        // forward
    void* h;
    int64_t h_t, h_b;
    float* cT;
    float* states;                          // written by the forward, read by the backward
    const void* dh;                         // backward
    int64_t dh_t, dh_b;
    const float* dcT;
    void* dP;
    int64_t dP_t, dP_b;
    float* dc0;
    float* ws;
};
size_t scan_workspace_bytes(int T, int B, int H);
bool scan_fits(int T, int B, int H);
hipError_t launch_scan_forward(const ScanArgs& a, hipStream_t s);
hipError_t launch_scan_backward(const ScanArgs& a, hipStream_t s);

// ---- RMS norm and 8-bit quantization (norm_kernels.hip)
constexpr int kNormMaxCols = 16384;
struct NormArgs {
    int M, N, bf16;
    const void* x;
    int64_t x_ld;
    const void* residual;
    int64_t residual_ld;
    const float* weight;
    float eps;
    void* sum;
    int64_t sum_ld;
    void* y;
    int64_t y_ld;
    uint8_t* y8;
    int64_t y8_ld;
    float* scale;
    int64_t scale_ld;
    float* rstd;
};
hipError_t launch_rmsnorm_forward(const NormArgs& a, hipStream_t s);
struct NormGradArgs {
    int M, N, bf16;
    const void* sum;
    int64_t sum_ld;
    const float* weight;
    const float* rstd;
    const void* dy;
    int64_t dy_ld;
    const void* dsum;
    int64_t dsum_ld;
    void* dx;
    int64_t dx_ld;
    float* dweight;
    float* ws;
};
size_t rmsnorm_workspace_bytes(int M, int N);
hipError_t launch_rmsnorm_backward(const NormGradArgs& a, hipStream_t s);
struct QuantizeArgs {
    int M, N, bf16, block_rows;
    const void* x;
    int64_t x_ld;
    uint8_t* q;
    int64_t q_ld;
    float* scale;
    int64_t scale_ld;
};
hipError_t launch_quantize_fp8(const QuantizeArgs& a, hipStream_t s);

// ---- product of 8-bit operands (matmul_fp8.hip)
struct MatmulFp8Args {
    int M, N, K, w_block_rows, out_bf16;
    const uint8_t* A;
    int64_t a_ld;
    const float* a_scale;
    int64_t a_scale_ld;
    const uint8_t* W;
    int64_t w_ld;
    const float* w_scale;
    int64_t w_scale_ld;
    const float* bias;
    void* C;
    int64_t c_ld;
};
hipError_t launch_matmul_fp8(const MatmulFp8Args& a, hipStream_t s);

// ---- sampling (sample_kernels.hip)
constexpr int kSampleMaxVocabulary = 1 << 20;
struct SampleArgs {
    int M, V, bf16;
    const void* logits;
    int64_t ld;
    const uint8_t* allowed;
    int64_t allowed_ld;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;
    int* token;
    float* prob;
    int* kept;
};
hipError_t launch_sample(const SampleArgs& a, hipStream_t s);

}  // namespace l355
