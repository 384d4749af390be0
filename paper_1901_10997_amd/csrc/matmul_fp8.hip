// Product of e4m3 operands with a scale for every 128 columns:
//
//     C[m, n] = sum over blocks kb of  a_scale[m, kb] w_scale[n or n / 128, kb]  sum over k in kb of A[m, k] W[n, k]   + bias[n]
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>

namespace l355 {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Sixteen bytes of a row at column k: zeros for what lies behind column K.  Rows are padded to sixteen bytes.
__device__ __forceinline__ u32x4v load16(const uint8_t* row, int k, int K)
{
    u32x4v v = {0u, 0u, 0u, 0u};
    if (k < K) {
        v = *(const u32x4v*)(row + k);
        if (k + 16 > K) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int left = K - k - 4 * i;         // bytes of this word inside the row
                v[i] &= left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
            }
        }
    }
    return v;
}
// eight e4m3 values as bf16, which holds them all
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi)
{
    const u32x4v w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true))};
    return __builtin_bit_cast(bf16x8, w);
}

constexpr int kRowsWaves = 4;

// Few rows: a workgroup takes 16 rows of W and 16 MT of A, its waves every fourth block of 128 columns; their sums meet in
// LDS.  Lane (r, g) of a wave holds row r's columns 32 g .. 32 g + 31 of a block for both operands, whatever order the
// instruction sums them in.  The rows of W are the instruction's first operand, so a lane ends with four neighbouring n of
// one m, and one scale of A per lane does.
template <int MT>
__global__ __launch_bounds__(64 * kRowsWaves) void matmul_fp8_rows_kernel(MatmulFp8Args a)
{
    __shared__ f32x4v sums[kRowsWaves][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int tiles_n = (a.N + 15) / 16, n0 = blockIdx.x % tiles_n * 16, m0 = blockIdx.x / tiles_n * 16 * MT;
    const uint8_t* const w_row = a.W + (int64_t)min(n0 + r, a.N - 1) * a.w_ld;
    const uint8_t* a_row[MT];
    const float* a_scale[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = min(m0 + 16 * t + r, a.M - 1);
        a_row[t] = a.A + (int64_t)m * a.a_ld;
        a_scale[t] = a.a_scale + (int64_t)m * a.a_scale_ld;
    }
    const float* w_scale[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = min(n0 + 4 * g + i, a.N - 1);
        w_scale[i] = a.w_scale + (int64_t)(a.w_block_rows == 1 ? n : n / a.w_block_rows) * a.w_scale_ld;
    }
    f32x4v acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = (f32x4v){0.f, 0.f, 0.f, 0.f};
    const int blocks = (a.K + kScaleCols - 1) / kScaleCols;
    for (int kb = wave; kb < blocks; kb += kRowsWaves) {
        const int k = kb * kScaleCols + 32 * g;
        const u32x4v w0 = load16(w_row, k, a.K), w1 = load16(w_row, k + 16, a.K);
        const bf16x8 w[4] = {widen(w0[0], w0[1]), widen(w0[2], w0[3]), widen(w1[0], w1[1]), widen(w1[2], w1[3])};
        float ws[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ws[i] = w_scale[i][kb];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const u32x4v x0 = load16(a_row[t], k, a.K), x1 = load16(a_row[t], k + 16, a.K);
            f32x4v d = {0.f, 0.f, 0.f, 0.f};
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[0], widen(x0[0], x0[1]), d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[1], widen(x0[2], x0[3]), d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[2], widen(x1[0], x1[1]), d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[3], widen(x1[2], x1[3]), d, 0, 0, 0);
            const float as = a_scale[t][kb];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(d[i] * ws[i], as, acc[t][i]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
#pragma unroll
    for (int t0 = 0; t0 < MT; t0 += kRowsWaves) {
        const int t = t0 + wave;
        if (t >= MT) continue;
        f32x4v v = sums[0][t][lane];
#pragma unroll
        for (int w = 1; w < kRowsWaves; ++w) v += sums[w][t][lane];
        const int m = m0 + 16 * t + r;
        if (m >= a.M) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = n0 + 4 * g + i;
            if (n >= a.N) continue;
            const float c = v[i] + (a.bias ? a.bias[n] : 0.f);
            if (a.out_bf16) ((uint16_t*)a.C)[(int64_t)m * a.c_ld + n] = to_bf16(c);
            else ((float*)a.C)[(int64_t)m * a.c_ld + n] = c;
        }
    }
}

}  // namespace

size_t matmul_fp8_workspace_bytes(int, int, int) { return 256; }

hipError_t launch_matmul_fp8(const MatmulFp8Args& a, hipStream_t s)
{
    const dim3 block(64 * kRowsWaves);
    const unsigned n = (a.N + 15) / 16;
    if (a.M <= 16) hipLaunchKernelGGL(matmul_fp8_rows_kernel<1>, dim3(n), block, 0, s, a);
    else hipLaunchKernelGGL(matmul_fp8_rows_kernel<4>, dim3(n * ((a.M + 63) / 64)), block, 0, s, a);
    return hipGetLastError();
}

}  // namespace l355
