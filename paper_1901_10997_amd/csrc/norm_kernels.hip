// Root-mean-square norm with the residual's addition in front and 8-bit values with scales behind, its gradient, and the
// quantization alone.
//
//     s = round(x + r)    rstd = (sum s^2 / N + eps)^-1/2    y = s rstd w
//     a block of 128 columns: scale = max |y| / 448, q = e4m3(y / scale)
//     gradient: g = dy w, xhat = s rstd, ds = rstd (g - xhat sum(g xhat) / N) + ds_in, dw = sum over rows of dy xhat
//
// Bound: HBM.  A row is held in registers between its two uses, so everything is read and written once.  Lane l of a row's
// waves holds granules of eight neighbouring columns, so that sixteen lanes - a row of the wavefront's cross-lane network -
// hold a block of 128 and its maximum takes four register moves.
#include "device_math.h"
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>
#include <cfloat>

namespace l355 {

namespace {

constexpr int kNormThreads = 256;
constexpr int kGranule = 8;

// Columns col .. col+7 of a row that has N of them; what lies behind the row is 0.  A granule inside the row is moved in 16-byte
// pieces wherever it starts (elem.h), so that rows of an odd length cost what those of an even one do: 754 rows of 7671 bf16
// columns with residual and 8-bit values 13.8 us; with such rows read column by column 31.7.
template <class E>
__device__ __forceinline__ void load_granule(const typename E::T* row, int col, int N, float* v)
{
    if (col + kGranule <= N) {
        load_n<E, kGranule, true>(row + col, v);
    } else {
#pragma unroll
        for (int i = 0; i < kGranule; ++i) v[i] = col + i < N ? E::load(row + col + i) : 0.f;
    }
}
template <class E>
__device__ __forceinline__ void store_granule(typename E::T* row, int col, int N, const float* v)
{
    if (col + kGranule <= N) {
        store_n<E, kGranule, true>(row + col, v);
    } else {
#pragma unroll
        for (int i = 0; i < kGranule; ++i)
            if (col + i < N) E::store(row + col + i, v[i]);
    }
}

// Scale of a block whose largest finite magnitude is amax (an infinity counts as the largest finite value)
__device__ __forceinline__ float block_scale(float amax) { return fmaxf(fminf(amax, FLT_MAX) / kE4m3Max, kSmallestScale); }

// v / scale, rounded to e4m3: the quotient as division rounds it (multiplied by 1 / scale and corrected by its remainder),
// so that a tie stays a tie; an infinity becomes the largest value, NaN stays NaN.
__device__ __forceinline__ float scaled(float v, float scale, float inverse)
{
    const float q = v * inverse;
    const float exact = fmaf(fmaf(-q, scale, v), inverse, q);
    return fabsf(q) > kE4m3Max ? copysignf(kE4m3Max, q) : exact;
}
__device__ __forceinline__ u32x2v pack_e4m3(const float* v)
{
    u32x2v w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], p, true);
        w[i] = (uint32_t)p;
    }
    return w;
}
__device__ __forceinline__ void store_e4m3(uint8_t* row, int col, int N, u32x2v w)
{
    if (col + kGranule <= N) {
        *(u32x2v*)(row + col) = w;
    } else {
#pragma unroll
        for (int i = 0; i < kGranule; ++i)
            if (col + i < N) row[col + i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}
// Eight columns of every lane to e4m3; lane 0 of each block of sixteen lanes stores the scale.
__device__ __forceinline__ void quantize_granule(const float* v, int col, int N, uint8_t* q_row, float* scale_row)
{
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < kGranule; ++i) amax = fmaxf(amax, fabsf(v[i]));
    const float scale = block_scale(row16_max(amax)), inverse = 1.f / scale;
    float q[kGranule];
#pragma unroll
    for (int i = 0; i < kGranule; ++i) q[i] = scaled(v[i], scale, inverse);
    store_e4m3(q_row, col, N, pack_e4m3(q));
    if ((threadIdx.x & 15) == 0 && col < N) scale_row[col / kScaleCols] = scale;
}

// Sum over the WPR waves of a row, in all of their threads; `part` is of this use alone until the next barrier but one.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* part)
{
    v = wave_sum(v);
    if constexpr (WPR > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) v += part[i];
    }
    return v;
}

// The largest of the WPR waves of a row, in all of their threads; NaN gives way
template <int WPR>
__device__ __forceinline__ float row_max(float v, float* part)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    if constexpr (WPR > 1) {
        __syncthreads();            // everybody has read what is there
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WPR; ++i) v = fmaxf(v, part[i]);
    }
    return v;
}

// Mean squares (with eps) outside these: the sum of squares is beyond fp32, or some of them are below its normal numbers.
constexpr float kSmallMean = 0x1p-100f, kLargeMean = 0x1p110f;

// WPR waves of a workgroup's four on a row, IT granules per lane: rows of up to 512 WPR IT columns.
template <class E, int WPR, int IT>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_forward_kernel(NormArgs a)
{
    __shared__ float part[4];
    using T = typename E::T;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = blockIdx.x * (4 / WPR) + wave / WPR;
    if (row >= a.M) return;                     // whole waves, and with one row per workgroup none
    const int col0 = ((wave % WPR) * 64 + lane) * kGranule;
    const T* const x = (const T*)a.x + (int64_t)row * a.x_ld;
    float v[IT][kGranule], squares = 0.f;
#pragma unroll
    for (int k = 0; k < IT; ++k) load_granule<E>(x, col0 + k * WPR * 512, a.N, v[k]);
    if (a.residual) {
        const T* const r = (const T*)a.residual + (int64_t)row * a.residual_ld;
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            float w[kGranule];
            load_granule<E>(r, col0 + k * WPR * 512, a.N, w);
            // rounded to the type it is kept in, so that the norm, the next layer's residual and the gradient see one value
#pragma unroll
            for (int i = 0; i < kGranule; ++i) v[k][i] = E::round(v[k][i] + w[i]);
        }
    }
    if (a.sum) {
        T* const s = (T*)a.sum + (int64_t)row * a.sum_ld;
#pragma unroll
        for (int k = 0; k < IT; ++k) store_granule<E>(s, col0 + k * WPR * 512, a.N, v[k]);
    }
#pragma unroll
    for (int k = 0; k < IT; ++k)
#pragma unroll
        for (int i = 0; i < kGranule; ++i) squares = fmaf(v[k][i], v[k][i], squares);
    const float mean = row_sum<WPR>(squares, part) / (float)a.N + a.eps;
    float rstd = 1.f / sqrtf(mean), power = 1.f;
    if (!(mean >= kSmallMean && mean <= kLargeMean)) {      // all of the row's threads or none
        float largest = 0.f;
#pragma unroll
        for (int k = 0; k < IT; ++k)
#pragma unroll
            for (int i = 0; i < kGranule; ++i) largest = fmaxf(largest, fabsf(v[k][i]));
        largest = fmaxf(row_max<WPR>(largest, part), sqrtf(a.eps));
        if (largest > 0.f && largest <= FLT_MAX) {          // else a row of zeros without eps, or with an infinity: as it came out
            // by the power of two that brings the larger of the row and sqrt(eps) to about one
            const int e = max(-126, min(126, 1 - __builtin_amdgcn_frexp_expf(largest)));
            power = __builtin_amdgcn_ldexpf(1.f, e);
            const float root = sqrtf(a.eps) * power;
            squares = 0.f;
#pragma unroll
            for (int k = 0; k < IT; ++k)
#pragma unroll
                for (int i = 0; i < kGranule; ++i) {
                    v[k][i] *= power;
                    squares = fmaf(v[k][i], v[k][i], squares);
                }
            if constexpr (WPR > 1) __syncthreads();
            rstd = 1.f / sqrtf(row_sum<WPR>(squares, part) / (float)a.N + root * root);
        }
    }
    if (a.rstd && col0 == 0) a.rstd[row] = rstd * power;
#pragma unroll
    for (int k = 0; k < IT; ++k) {
        const int col = col0 + k * WPR * 512;
        float w[kGranule];
        if (a.weight) {
            load_granule<F32>(a.weight, col, a.N, w);
        } else {
#pragma unroll
            for (int i = 0; i < kGranule; ++i) w[i] = 1.f;
        }
#pragma unroll
        for (int i = 0; i < kGranule; ++i) v[k][i] = v[k][i] * rstd * w[i];
#pragma unroll
        for (int i = 0; i < kGranule; ++i)      // 0 * infinity behind the row must not reach the block's maximum
            if (col + i >= a.N) v[k][i] = 0.f;
        if (a.y) store_granule<E>((T*)a.y + (int64_t)row * a.y_ld, col, a.N, v[k]);
        if (a.y8) quantize_granule(v[k], col, a.N, a.y8 + (int64_t)row * a.y8_ld, a.scale + (int64_t)row * a.scale_ld);
    }
}

// A team of WPR waves takes every teams-th row and keeps its sums of dw in registers; those of a workgroup's teams meet in LDS
// and go to ws [workgroups][N].
template <class E, int WPR, int IT>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_backward_kernel(NormGradArgs a)
{
    __shared__ float part[2][4];
    __shared__ float met[WPR == 1 ? 3 : 1][WPR == 1 ? 512 * IT : 1];
    using T = typename E::T;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int team = blockIdx.x * (4 / WPR) + wave / WPR, teams = gridDim.x * (4 / WPR);
    const int col0 = ((wave % WPR) * 64 + lane) * kGranule;
    float dw[IT][kGranule];
#pragma unroll
    for (int k = 0; k < IT; ++k)
#pragma unroll
        for (int i = 0; i < kGranule; ++i) dw[k][i] = 0.f;
    int turn = 0;
    for (int row = team; row < a.M; row += teams, turn ^= 1) {
        const T* const s = (const T*)a.sum + (int64_t)row * a.sum_ld;
        const T* const dy = (const T*)a.dy + (int64_t)row * a.dy_ld;
        const float rstd = a.rstd[row];
        float x[IT][kGranule], g[IT][kGranule], inner = 0.f;
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            load_granule<E>(s, col0 + k * WPR * 512, a.N, x[k]);
            load_granule<E>(dy, col0 + k * WPR * 512, a.N, g[k]);
        }
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            float w[kGranule];
            if (a.weight) {
                load_granule<F32>(a.weight, col0 + k * WPR * 512, a.N, w);
            } else {
#pragma unroll
                for (int i = 0; i < kGranule; ++i) w[i] = 1.f;
            }
#pragma unroll
            for (int i = 0; i < kGranule; ++i) {
                x[k][i] *= rstd;
                dw[k][i] = fmaf(g[k][i], x[k][i], dw[k][i]);
                g[k][i] *= w[i];
                if (col0 + k * WPR * 512 + i < a.N) inner = fmaf(g[k][i], x[k][i], inner);
            }
        }
        const float mean = row_sum<WPR>(inner, part[turn]) / (float)a.N;
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            float d[kGranule];
            if (a.dsum) {
                load_granule<E>((const T*)a.dsum + (int64_t)row * a.dsum_ld, col0 + k * WPR * 512, a.N, d);
            } else {
#pragma unroll
                for (int i = 0; i < kGranule; ++i) d[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < kGranule; ++i) d[i] = fmaf(rstd, fmaf(-x[k][i], mean, g[k][i]), d[i]);
            store_granule<E>((T*)a.dx + (int64_t)row * a.dx_ld, col0 + k * WPR * 512, a.N, d);
        }
    }
    if (!a.dweight) return;
    if constexpr (WPR == 1) {
        // column i of the granules of step k stands at (k * 8 + i) * 64 + lane: every wave's lanes meet different banks
        if (wave > 0)
#pragma unroll
            for (int k = 0; k < IT; ++k)
#pragma unroll
                for (int i = 0; i < kGranule; ++i) met[wave - 1][(k * kGranule + i) * 64 + lane] = dw[k][i];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int k = 0; k < IT; ++k)
#pragma unroll
                for (int i = 0; i < kGranule; ++i) dw[k][i] += met[w][(k * kGranule + i) * 64 + lane];
    }
    float* const to = a.ws + (int64_t)blockIdx.x * a.N;
#pragma unroll
    for (int k = 0; k < IT; ++k) store_granule<F32>(to, col0 + k * WPR * 512, a.N, dw[k]);
}

// dw = sum of the rows of ws, in their order: 16 columns per workgroup, sixteen threads of each column
__global__ __launch_bounds__(256) void column_sum_kernel(const float* __restrict__ ws, int rows, int N, float* __restrict__ dw)
{
    __shared__ float part[16][16];
    const int c = threadIdx.x & 15, k = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float sum = 0.f;
    if (col < N) {
        const float* const p = ws + col;
        int t = k;
        for (; t + 112 < rows; t += 128) {      // eight loads under way
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p[(int64_t)(t + 16 * i) * N];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
        for (; t < rows; t += 16) sum += p[(int64_t)t * N];
    }
    part[k][c] = sum;
    __syncthreads();
    if (k == 0 && col < N) {
#pragma unroll
        for (int i = 1; i < 16; ++i) sum += part[i][c];
        dw[col] = sum;
    }
}

// A scale for every row and 128 columns: a wave takes 512 columns of a row.
template <class E>
__global__ __launch_bounds__(kNormThreads) void quantize_rows_kernel(QuantizeArgs a, int parts)
{
    const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row = task / parts;
    if (row >= a.M) return;
    const int col = ((int)(task % parts) * 64 + (threadIdx.x & 63)) * kGranule;
    float v[kGranule];
    load_granule<E>((const typename E::T*)a.x + row * a.x_ld, col, a.N, v);
    quantize_granule(v, col, a.N, a.q + row * a.q_ld, a.scale + row * a.scale_ld);
}

// A scale for 128 rows and 128 columns: a workgroup each, sixteen rows at a time.
template <class E>
__global__ __launch_bounds__(kNormThreads) void quantize_blocks_kernel(QuantizeArgs a, int parts)
{
    __shared__ float part[4];
    const int br = blockIdx.x / parts, bc = blockIdx.x % parts;
    const int col = bc * kScaleCols + (threadIdx.x & 15) * kGranule;
    const int row0 = br * 128 + (threadIdx.x >> 4);
    float v[8][kGranule], amax = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int row = row0 + 16 * k;
        // rows behind the matrix have no columns
        load_granule<E>((const typename E::T*)a.x + (int64_t)min(row, a.M - 1) * a.x_ld, col, row < a.M ? a.N : 0, v[k]);
#pragma unroll
        for (int i = 0; i < kGranule; ++i) amax = fmaxf(amax, fabsf(v[k][i]));
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = amax;
    __syncthreads();
    const float scale = block_scale(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]))), inverse = 1.f / scale;
    if (threadIdx.x == 0) a.scale[(int64_t)br * a.scale_ld + bc] = scale;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int row = row0 + 16 * k;
        float q[kGranule];
#pragma unroll
        for (int i = 0; i < kGranule; ++i) q[i] = scaled(v[k][i], scale, inverse);
        if (row < a.M) store_e4m3(a.q + (int64_t)row * a.q_ld, col, a.N, pack_e4m3(q));
    }
}

// The number of waves on a row and of granules per lane: a wave alone needs no barrier, four together take wide rows, and a
// few rows faster (kFewRows of them leave compute units idle otherwise).
constexpr int kFewRows = 1024;
template <class F>
void with_row_shape(int M, int N, F f)
{
    using std::integral_constant;
    if (N <= 2048 && M > kFewRows) {
        if (N <= 512) f(integral_constant<int, 1>(), integral_constant<int, 1>());
        else if (N <= 1024) f(integral_constant<int, 1>(), integral_constant<int, 2>());
        else f(integral_constant<int, 1>(), integral_constant<int, 4>());
    } else if (N <= 2048) {
        f(integral_constant<int, 4>(), integral_constant<int, 1>());
    } else if (N <= 4096) {
        f(integral_constant<int, 4>(), integral_constant<int, 2>());
    } else if (N <= 8192) {
        f(integral_constant<int, 4>(), integral_constant<int, 4>());
    } else {
        f(integral_constant<int, 4>(), integral_constant<int, 8>());
    }
}
template <class F>
void with_elements(bool bf16, F f)
{
    if (bf16) f(Bf16());
    else f(F32());
}

// Workgroups of the gradient for `rows` rows at a time in each: at most kGradGroups, and all with the same number of turns
constexpr int kGradGroups = 512;
int grad_groups(int M, int rows)
{
    const int all = (M + rows - 1) / rows, turns = (all + kGradGroups - 1) / kGradGroups;
    return turns < 1 ? 0 : (all + turns - 1) / turns;
}

}  // namespace

hipError_t launch_rmsnorm_forward(const NormArgs& a, hipStream_t s)
{
    with_elements(a.bf16, [&](auto e) {
        with_row_shape(a.M, a.N, [&](auto wpr, auto it) {
            constexpr int kWaves = decltype(wpr)::value;
            const dim3 grid((a.M + 4 / kWaves - 1) / (4 / kWaves)), block(kNormThreads);
            hipLaunchKernelGGL((rmsnorm_forward_kernel<decltype(e), kWaves, decltype(it)::value>), grid, block, 0, s, a);
        });
    });
    return hipGetLastError();
}

size_t rmsnorm_workspace_bytes(int M, int N) { return (size_t)std::min(M, kGradGroups) * N * sizeof(float); }

hipError_t launch_rmsnorm_backward(const NormGradArgs& a, hipStream_t s)
{
    int groups = 0;
    if (a.M > 0) with_elements(a.bf16, [&](auto e) {
        with_row_shape(a.M, a.N, [&](auto wpr, auto it) {
            constexpr int kWaves = decltype(wpr)::value;
            groups = grad_groups(a.M, 4 / kWaves);
            hipLaunchKernelGGL((rmsnorm_backward_kernel<decltype(e), kWaves, decltype(it)::value>), dim3(groups), dim3(kNormThreads), 0, s, a);
        });
    });
    if (a.dweight) hipLaunchKernelGGL(column_sum_kernel, dim3((a.N + 15) / 16), dim3(256), 0, s, a.ws, groups, a.N, a.dweight);
    return hipGetLastError();
}

hipError_t launch_quantize_fp8(const QuantizeArgs& a, hipStream_t s)
{
    with_elements(a.bf16, [&](auto e) {
        if (a.block_rows == 1) {
            const int parts = (a.N + 511) / 512;
            const dim3 grid((unsigned)(((int64_t)a.M * parts + 3) / 4));
            hipLaunchKernelGGL((quantize_rows_kernel<decltype(e)>), grid, dim3(kNormThreads), 0, s, a, parts);
        } else {
            const int parts = (a.N + kScaleCols - 1) / kScaleCols;
            const dim3 grid((unsigned)((int64_t)((a.M + 127) / 128) * parts));
            hipLaunchKernelGGL((quantize_blocks_kernel<decltype(e)>), grid, dim3(kNormThreads), 0, s, a, parts);
        }
    });
    return hipGetLastError();
}

}  // namespace l355
