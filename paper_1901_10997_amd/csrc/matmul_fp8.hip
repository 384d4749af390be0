// Product of e4m3 operands with a scale for every 128 columns:
//
//     C[m, n] = sum over blocks kb of  a_scale[m, kb] w_scale[n or n / 128, kb]  sum over k in kb of A[m, k] W[n, k]   + bias[n]
#include "common.h"
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>
#include <cfloat>
#include <type_traits>

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
// eight e4m3 values times a power of two (up to 2^60 either way) as bf16, which holds them all
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float power = 1.f)
{
    const u32x4v w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, true))};
    return __builtin_bit_cast(bf16x8, w);
}

// A block's sum is multiplied by two scales, each of which may be anything from 2^-126 to 2^119: their product may leave the
// range of fp32, and so may the sum times either, where the result does not.  So the power of two of a row's scale of A, up to 2^60
// of it, comes first - in the tiles with its values, as they are widened - and the sum is multiplied by W's scale and what is left
// after that: nothing on the way is out of range then unless the result is.  (16384 x 8192 x 2048 511 us with one product of
// the scales instead, 535 so; 128 x 2000 x 4000 18.8 and 19.4.)
struct RowScale {
    float power, rest;
};
__device__ __forceinline__ RowScale split_scale(float scale)
{
    const int e = max(-60, min(60, __builtin_amdgcn_frexp_expf(scale) - 1));
    return {__builtin_amdgcn_ldexpf(1.f, e), __builtin_amdgcn_ldexpf(scale, -e)};
}
// a b; where two finite numbers give an infinity the largest finite value, so that zero times it is zero
__device__ __forceinline__ float within(float a, float b)
{
    const float p = a * b;
    return fabsf(p) == __builtin_inff() && fabsf(a) <= FLT_MAX && fabsf(b) <= FLT_MAX ? copysignf(FLT_MAX, p) : p;
}

// COUNT neighbouring results of a row, those of them that it has
template <class E, int COUNT>
__device__ __forceinline__ void store_row(const MatmulFp8Args& a, int m, int n, const float* v)
{
    typename E::T* const c = (typename E::T*)a.C + (int64_t)m * a.c_ld + n;
    if (n + COUNT <= a.N) {
        constexpr int kPiece = E::kBytes == 2 && COUNT >= 8 ? 8 : 4;
#pragma unroll
        for (int i = 0; i < COUNT; i += kPiece) store_n<E, kPiece, true>(c + i, v + i);
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (n + i < a.N) E::store(c + i, v[i]);
    }
}

constexpr int kRowsWaves = 4;

// Few rows, or few tiles: a workgroup takes 16 rows of W and 16 MT of A, its waves every fourth block of 128 columns; their sums meet in
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
            const RowScale as = split_scale(a_scale[t][kb]);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(d[i] * as.power * ws[i], as.rest, acc[t][i]);
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
        const int n = n0 + 4 * g;
        float c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = v[i] + (a.bias ? a.bias[min(n + i, a.N - 1)] : 0.f);
        if (a.out_bf16) store_row<Bf16, 4>(a, m, n, c);
        else store_row<F32, 4>(a, m, n, c);
    }
}

// Many rows.  A workgroup of four waves takes a tile of 128 rows of W by 32 TM of A, each wave 64 by 16 TM of it.  The rows
// of a block of 128 columns are copied to LDS without passing through registers while the block before is multiplied, and a
// wave reads its fragments of a block at once; two to three workgroups on a compute unit fill each other's waits.
// Sixteen-byte chunk c of row r stands at chunk c ^ key(r), and lanes (r, g) read chunks g and g + 4, so that the lanes that
// are served together meet different banks (chunks 2 g and 2 g + 1 cost twice the reads).
//
// The instruction is that of bf16 operands, which hold every e4m3 value: its sums are good to fp32 (2^-21 of the magnitudes
// at worst over random codes, one block of 128).  The instructions of 8-bit operands drop what is 2^-13 below the largest
// product of a sum: with one large pair that cancels, nothing of the others is left.  They would take 331 us in place of 535 for
// 16384 x 8192 x 2048 to bf16.
//
// Bound: what a wave has to issue, and the clock.  16384 x 8192 x 2048 to bf16 takes 535 us, 1.03 PFLOP/s, where a large library
// product of bf16 operands sustains 1.14 (up to 690 where the card has lowered its clock under launches in a row).  For 64
// matrix instructions of a block a wave of the large tiles issues 128 conversions and 64 multiplications by scales: the matrix unit is
// busy for half of the cycles.  The next block's copies are issued in between the products: in front of the reads
// 4096 x 4096 x 4096 takes a twenty-fifth longer, 700 x 6000 x 1500 a fortieth.
//
// The instruction's rows are rows of W in an order that leaves a lane with sixteen neighbouring n of one m (n_of), so that C
// is written in wide pieces; one scale per lane and 16 rows of A covers them where W's scales are those of 128 rows.
typedef void __attribute__((address_space(3)))* InLds;
constexpr int kBufferWord3 = 4 << 15 | 7 << 12;     // of a buffer descriptor: 32-bit elements
constexpr int kTN = 4;                              // fragments of W per wave
__device__ __forceinline__ int key_a(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int key_w(int row) { return ((row >> 1) & 1) | ((row >> 4) & 3) << 1; }
// A wave's fragments and scales of a block, all of them there when it returns.  (Written out because in front of a read that
// it knows of the compiler waits until every copy to LDS under way has ended.)  w, a: addresses of the lower chunks, w1, a1: of
// the upper ones; ws, as: of the scales.
#define L355_READ_W(w, w1)                                                                                                       \
    "ds_read_b128 %0, " w "\n\tds_read_b128 %1, " w1 "\n\tds_read_b128 %2, " w " offset:512\n\tds_read_b128 %3, " w1 " offset:512\n\t" \
    "ds_read_b128 %4, " w " offset:1024\n\tds_read_b128 %5, " w1 " offset:1024\n\t"                                                  \
    "ds_read_b128 %6, " w " offset:1536\n\tds_read_b128 %7, " w1 " offset:1536\n\t"
#define L355_W_OUT "=&v"(fw[0][0]), "=&v"(fw[0][1]), "=&v"(fw[1][0]), "=&v"(fw[1][1]), "=&v"(fw[2][0]), "=&v"(fw[2][1]), "=&v"(fw[3][0]), "=&v"(fw[3][1])
struct Addresses {
    unsigned w, w1, a, a1, ws, as;
};
__device__ __forceinline__ void read_block(u32x4v (&fw)[4][2], u32x4v (&fa)[4][2], float (&ws)[1][4], f32x4v& as, const Addresses& at)
{
    asm volatile("ds_read_b32 %16, %22\n\tds_read_b128 %17, %23\n\tds_read_b128 %8, %20\n\tds_read_b128 %9, %21\n\t"
                 "ds_read_b128 %10, %20 offset:2048\n\tds_read_b128 %11, %21 offset:2048\n\t"
                 "ds_read_b128 %12, %20 offset:4096\n\tds_read_b128 %13, %21 offset:4096\n\t"
                 "ds_read_b128 %14, %20 offset:6144\n\tds_read_b128 %15, %21 offset:6144\n\t" L355_READ_W("%18", "%19")
                 "s_waitcnt lgkmcnt(0)"
                 : L355_W_OUT, "=&v"(fa[0][0]), "=&v"(fa[0][1]), "=&v"(fa[1][0]), "=&v"(fa[1][1]), "=&v"(fa[2][0]), "=&v"(fa[2][1]), "=&v"(fa[3][0]), "=&v"(fa[3][1]),
                   "=&v"(ws[0][0]), "=&v"(as)
                 : "v"(at.w), "v"(at.w1), "v"(at.a), "v"(at.a1), "v"(at.ws), "v"(at.as)
                 : "memory");
}
__device__ __forceinline__ void read_block(u32x4v (&fw)[4][2], u32x4v (&fa)[2][2], float (&ws)[1][4], f32x2v& as, const Addresses& at)
{
    asm volatile("ds_read_b32 %12, %18\n\tds_read_b64 %13, %19\n\tds_read_b128 %8, %16\n\tds_read_b128 %9, %17\n\t"
                 "ds_read_b128 %10, %16 offset:2048\n\tds_read_b128 %11, %17 offset:2048\n\t" L355_READ_W("%14", "%15")
                 "s_waitcnt lgkmcnt(0)"
                 : L355_W_OUT, "=&v"(fa[0][0]), "=&v"(fa[0][1]), "=&v"(fa[1][0]), "=&v"(fa[1][1]), "=&v"(ws[0][0]), "=&v"(as)
                 : "v"(at.w), "v"(at.w1), "v"(at.a), "v"(at.a1), "v"(at.ws), "v"(at.as)
                 : "memory");
}
// with a scale for each of the lane's sixteen n
__device__ __forceinline__ void read_block(u32x4v (&fw)[4][2], u32x4v (&fa)[4][2], f32x4v (&ws)[4], f32x4v& as, const Addresses& at)
{
    asm volatile("ds_read_b128 %16, %25\n\tds_read_b128 %17, %25 offset:16\n\tds_read_b128 %18, %25 offset:32\n\tds_read_b128 %19, %25 offset:48\n\t"
                 "ds_read_b128 %20, %26\n\tds_read_b128 %8, %23\n\tds_read_b128 %9, %24\n\t"
                 "ds_read_b128 %10, %23 offset:2048\n\tds_read_b128 %11, %24 offset:2048\n\t"
                 "ds_read_b128 %12, %23 offset:4096\n\tds_read_b128 %13, %24 offset:4096\n\t"
                 "ds_read_b128 %14, %23 offset:6144\n\tds_read_b128 %15, %24 offset:6144\n\t" L355_READ_W("%21", "%22")
                 "s_waitcnt lgkmcnt(0)"
                 : L355_W_OUT, "=&v"(fa[0][0]), "=&v"(fa[0][1]), "=&v"(fa[1][0]), "=&v"(fa[1][1]), "=&v"(fa[2][0]), "=&v"(fa[2][1]), "=&v"(fa[3][0]), "=&v"(fa[3][1]),
                   "=&v"(ws[0]), "=&v"(ws[1]), "=&v"(ws[2]), "=&v"(ws[3]), "=&v"(as)
                 : "v"(at.w), "v"(at.w1), "v"(at.a), "v"(at.a1), "v"(at.ws), "v"(at.as)
                 : "memory");
}
__device__ __forceinline__ void read_block(u32x4v (&fw)[4][2], u32x4v (&fa)[2][2], f32x4v (&ws)[4], f32x2v& as, const Addresses& at)
{
    asm volatile("ds_read_b128 %12, %21\n\tds_read_b128 %13, %21 offset:16\n\tds_read_b128 %14, %21 offset:32\n\tds_read_b128 %15, %21 offset:48\n\t"
                 "ds_read_b64 %16, %22\n\tds_read_b128 %8, %19\n\tds_read_b128 %9, %20\n\t"
                 "ds_read_b128 %10, %19 offset:2048\n\tds_read_b128 %11, %20 offset:2048\n\t" L355_READ_W("%17", "%18")
                 "s_waitcnt lgkmcnt(0)"
                 : L355_W_OUT, "=&v"(fa[0][0]), "=&v"(fa[0][1]), "=&v"(fa[1][0]), "=&v"(fa[1][1]), "=&v"(ws[0]), "=&v"(ws[1]), "=&v"(ws[2]), "=&v"(ws[3]), "=&v"(as)
                 : "v"(at.w), "v"(at.w1), "v"(at.a), "v"(at.a1), "v"(at.ws), "v"(at.as)
                 : "memory");
}
#undef L355_READ_W
#undef L355_W_OUT

template <int TM, bool ROW_SCALES>
__global__ __launch_bounds__(256, 2) void matmul_fp8_tile_kernel(MatmulFp8Args a, int tiles_n, int tiles_m)
{
    constexpr int WN = 2, WM = 2, BN = 64 * WN, BM = 16 * TM * WM, TILE = (BN + BM) * 128, STAGE = TILE + 256 * (WN + WM), WAVES = WN * WM;
    constexpr int LW = BN / 8 / WAVES, LA = BM / 8 / WAVES;      // a wave's copies of eight rows of W and of A
    constexpr int COPIES = LW + LA + 1;                          // and one of scales
    static_assert(LW >= 1 && LA >= 1 && WAVES == WN + WM && (TM == 2 || TM == 4) && COPIES <= kTN * TM, "");
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    int n0, m0;
    {
        // eight neighbouring workgroups lie on different XCDs: each XCD gets a run of tiles, in groups of eight tiles of W
        const int tiles = tiles_n * tiles_m, per = tiles / 8, rest = tiles % 8, x = blockIdx.x % 8, y = blockIdx.x / 8;
        const int t = x * per + min(x, rest) + y;
        const int group = t / (8 * tiles_m), first = group * 8, width = min(8, tiles_n - first), in = t - first * tiles_m;
        n0 = (first + in % width) * BN;
        m0 = in / width * BM;
    }
    const int blocks = (a.K + kScaleCols - 1) / kScaleCols;
    // Through descriptors of the tile's rows: what lies behind the matrix reads as zero, and what a block reads behind column K
    // is the next row's or zero, and is masked.
    const int l8 = lane >> 3, c8 = lane & 7;
    const unsigned w_ld = (unsigned)a.w_ld, a_ld = (unsigned)a.a_ld, held = ((unsigned)a.K + 15u) & ~15u;
    const auto w_rows = __builtin_amdgcn_make_buffer_rsrc((void*)(a.W + n0 * a.w_ld), 0, (unsigned)(min(BN, a.N - n0) - 1) * w_ld + held, kBufferWord3);
    const auto a_rows = __builtin_amdgcn_make_buffer_rsrc((void*)(a.A + m0 * a.a_ld), 0, (unsigned)(min(BM, a.M - m0) - 1) * a_ld + held, kBufferWord3);
    const int wn = wave / WM * 64, wm = wave % WM * 16 * TM;     // the wave's part of the tile
    // scales: the first WN waves copy those of 64 rows of W each, the others those of 16 TM rows of A, in the order in which
    // lane r takes rows r, 16 + r, ..
    const bool of_w = wave < WN;
    const int first_row = of_w ? n0 / a.w_block_rows : m0, end_row = of_w ? (min(n0 + BN, a.N) - 1) / a.w_block_rows : min(m0 + BM, a.M) - 1;
    const int scale_ld = (int)(of_w ? a.w_scale_ld : a.a_scale_ld);
    const int scale_row = of_w ? (n0 + wave * 64 + lane) / a.w_block_rows : m0 + (wave - WN) * 16 * TM + 16 * (lane % TM) + (lane / TM & 15);
    const auto scales = __builtin_amdgcn_make_buffer_rsrc((void*)((of_w ? a.w_scale : a.a_scale) + (int64_t)first_row * scale_ld), 0,
                                                          4u * (unsigned)((end_row - first_row) * scale_ld + blocks), kBufferWord3);
    const unsigned scale_at = 4u * (unsigned)((scale_row - first_row) * scale_ld);
    const unsigned lds0 = (unsigned)(uintptr_t)(InLds)smem;
    // piece i of the copies of a block
    auto copy = [&](int kb, int stage, int i) {
        uint8_t* const to = smem + stage;
        const unsigned k = (unsigned)(kb * kScaleCols);
        if (i < LW) {
            const int x = wave * LW + i, row = 8 * x + l8, c = c8 ^ ((l8 >> 1) & 1) ^ (((x >> 1) & 3) << 1);
            const unsigned at = (unsigned)row * w_ld + (unsigned)(16 * c) + k;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rows, (InLds)(to + x * 1024), 16, at, 0, 0, 0);
        } else if (i < LW + LA) {
            const int x = wave * LA + i - LW, row = 8 * x + l8, c = c8 ^ (l8 >> 1) ^ ((x & 1) << 2);
            const unsigned at = (unsigned)row * a_ld + (unsigned)(16 * c) + k;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(a_rows, (InLds)(to + BN * 128 + x * 1024), 16, at, 0, 0, 0);
        } else {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(scales, (InLds)(to + TILE + wave * 256), 4, scale_at + 4u * (unsigned)kb, 0, 0, 0);
        }
    };

    // where this lane finds row r of its first fragments; the others follow at whole multiples of what the keys go by
    const int w_row = wn + 16 * (r >> 2) + (r & 3), a_row = wm + r;
    Addresses first;
    first.w = lds0 + w_row * 128 + (g ^ key_w(w_row)) * 16;
    first.w1 = first.w ^ 64u;
    first.a = lds0 + (BN + a_row) * 128 + (g ^ key_a(a_row)) * 16;
    first.a1 = first.a ^ 64u;
    first.ws = lds0 + TILE + wave / WM * 256 + (ROW_SCALES ? 64 * g : 0);
    first.as = lds0 + TILE + WN * 256 + wave % WM * 256 + 4 * TM * r;
    // n of register 0 of fragment j: sixteen neighbouring ones in a lane
    auto n_of = [&](int j) { return n0 + wn + 16 * g + 4 * j; };

    f32x4v acc[kTN][TM];
#pragma unroll
    for (int j = 0; j < kTN; ++j)
#pragma unroll
        for (int t = 0; t < TM; ++t) acc[j][t] = (f32x4v){0.f, 0.f, 0.f, 0.f};

    u32x4v fw[kTN][2], fa[TM][2];
    std::conditional_t<ROW_SCALES, f32x4v[4], float[1][4]> ws;
    std::conditional_t<TM == 4, f32x4v, f32x2v> s;
    float power[TM];
    auto read = [&](int kb, unsigned now) {
        read_block(fw, fa, ws, s, Addresses{first.w + now, first.w1 + now, first.a + now, first.a1 + now, first.ws + now, first.as + now});
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            const RowScale as = split_scale(s[t]);
            power[t] = as.power;
            // one scale of W: the product of the two is beyond fp32 only where the result is, or where the sum is zero
            s[t] = ROW_SCALES ? as.rest : within(as.rest, ws[0][0]);
        }
        if ((kb + 1) * kScaleCols > a.K) {  // zeros behind column K, in both operands: there may be NaN codes
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int left = a.K - kb * kScaleCols - 16 * g - 64 * h - 4 * i;
                    const uint32_t mask = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
                    for (int t = 0; t < TM; ++t) fa[t][h][i] &= mask;
#pragma unroll
                    for (int j = 0; j < kTN; ++j) fw[j][h][i] &= mask;
                }
        }
    };
    auto multiply = [&](int kb, int stage) {        // and copies block kb in between, if there is one
        // a product's sums are used behind the next product, so that the matrix unit does not wait for them
        constexpr int kAhead = 1, kAll = kTN * TM;
        f32x4v d[kAhead + 1];
        bf16x8 xa[TM][4], xw[4];
#pragma unroll
        for (int t = 0; t < TM; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) xa[t][q] = widen(fa[t][q >> 1][2 * (q & 1)], fa[t][q >> 1][2 * (q & 1) + 1], power[t]);
#pragma unroll
        for (int p = 0; p < kAll + kAhead; ++p) {
            if (p < kAll) {
                const int j = p / TM, t = p % TM;
                f32x4v& to = d[p % (kAhead + 1)];
                to = (f32x4v){0.f, 0.f, 0.f, 0.f};
                if (t == 0)
#pragma unroll
                    for (int q = 0; q < 4; ++q) xw[q] = widen(fw[j][q >> 1][2 * (q & 1)], fw[j][q >> 1][2 * (q & 1) + 1]);
#pragma unroll
                for (int q = 0; q < 4; ++q) to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xw[q], xa[t][q], to, 0, 0, 0);
            }
            if (p >= kAhead) {
                const int j = (p - kAhead) / TM, t = (p - kAhead) % TM;
                const f32x4v v = d[(p - kAhead) % (kAhead + 1)];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][t][i] = fmaf(ROW_SCALES ? v[i] * ws[ROW_SCALES ? j : 0][i] : v[i], s[t], acc[j][t][i]);
            }
            if (p < COPIES && kb < blocks) copy(kb, stage, p);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto barrier = []() {                   // bare: with the fence of __syncthreads() it would wait for the copies under way
        asm volatile("" : : : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
    };

    if (blocks > 0)
#pragma unroll
        for (int i = 0; i < COPIES; ++i) copy(0, 0, i);
    for (int kb = 0; kb < blocks; ++kb) {
        const int now = (kb & 1) * STAGE, next = STAGE - now;
        __builtin_amdgcn_s_waitcnt(0x0F70);         // vmcnt(0): this wave's copies of the block have arrived
        barrier();                          // everybody's have, and nobody reads the block before any more
        read(kb, now);
        multiply(kb + 1, next);
    }

    // a lane has sixteen neighbouring n: 32 or 64 bytes of a row of C
    const int n = n_of(0);
    float bias[4 * kTN];
#pragma unroll
    for (int i = 0; i < 4 * kTN; ++i) bias[i] = 0.f;
    if (a.bias)
#pragma unroll
        for (int i = 0; i < 4 * kTN; ++i) bias[i] = a.bias[min(n + i, a.N - 1)];
    // In one piece wherever it stands (elem.h): with odd rows of C (2102 x 2182 x 1254 to bf16) written element by element the
    // product took 12 us more.
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const int m = m0 + wm + 16 * t + r;
        if (m >= a.M) continue;
        float v[4 * kTN];
#pragma unroll
        for (int i = 0; i < 4 * kTN; ++i) v[i] = acc[i / 4][t][i % 4] + bias[i];
        if (a.out_bf16) store_row<Bf16, 4 * kTN>(a, m, n, v);
        else store_row<F32, 4 * kTN>(a, m, n, v);
    }
}

template <int TM, bool ROW_SCALES>
hipError_t tiles(const MatmulFp8Args& a, hipStream_t s)
{
    constexpr int BN = 128, BM = 32 * TM;
    constexpr size_t lds = 2 * (size_t)((BN + BM) * 128 + 4 * 256);     // two blocks, with their scales
    const int tn = (a.N + BN - 1) / BN, tm = (a.M + BM - 1) / BM;
    const hipError_t e = allow_dynamic_lds((const void*)matmul_fp8_tile_kernel<TM, ROW_SCALES>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((matmul_fp8_tile_kernel<TM, ROW_SCALES>), dim3(tn * tm), dim3(256), lds, s, a, tn, tm);
    return hipGetLastError();
}
int64_t tiles_in(const MatmulFp8Args& a, int rows) { return (int64_t)((a.N + 127) / 128) * ((a.M + rows - 1) / rows); }

// Tiles of 128 by 128 from so many of them on (two to a compute unit), else of 128 by 64.  4800 x 4096 x 800 (1216 tiles): 44
// against 47 us; 700 x 6000 x 1500 (282): 28 against 24.
constexpr int kLargeTiles = 512;
// Tiles of 128 by 64 up to which the kernel for few rows is faster, which spreads W over eight times as many workgroups: what a
// compute unit can have under way bounds the tiles then.  us of it and of tiles, to bf16: 128 x 2000 x 4000 (32 tiles) 18.8 and 32.6,
// 128 x 6000 x 1500 (94) 13.0 and 14.3, 400 x 2000 x 4000 (112) 39.7 and 32.6, 1000 x 1000 x 1000 (128) 12.7 and 11.0.
constexpr int kFewTiles = 96;

template <int TM>
hipError_t tiles_of(const MatmulFp8Args& a, hipStream_t s)
{
    return a.w_block_rows == 1 ? tiles<TM, true>(a, s) : tiles<TM, false>(a, s);
}

}  // namespace

hipError_t launch_matmul_fp8(const MatmulFp8Args& a, hipStream_t s)
{
    // the tiles add 32-bit offsets of their rows, and of their rows of scales, to a base
    if (a.M > 64 && tiles_in(a, 64) > kFewTiles && a.a_ld < (1 << 23) && a.w_ld < (1 << 23) && a.a_scale_ld < (1 << 21) && a.w_scale_ld < (1 << 21)) {
        return tiles_in(a, 128) >= kLargeTiles ? tiles_of<4>(a, s) : tiles_of<2>(a, s);
    }
    const dim3 block(64 * kRowsWaves);
    const unsigned n = (a.N + 15) / 16;
    if (a.M <= 16) hipLaunchKernelGGL(matmul_fp8_rows_kernel<1>, dim3(n), block, 0, s, a);
    else hipLaunchKernelGGL(matmul_fp8_rows_kernel<4>, dim3(n * ((a.M + 63) / 64)), block, 0, s, a);
    return hipGetLastError();
}

}  // namespace l355
