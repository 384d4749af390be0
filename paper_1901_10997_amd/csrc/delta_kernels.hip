// Gated delta rule: a recurrence whose state is a matrix S [Dk, Dv] for each head, which a key reads and corrects:
//
//     S_t = a_t (I - b_t k_t k_t') S_{t-1} + b_t k_t v_t'     a_t = exp(g_t)     o_t = scale S_t' q_t
//
// In blocks of 64 steps, with G the running sum of g in the block, S the state in front of it, y = exp(G), e = exp(G_last - G),
// D_ij = exp(G_i - G_j):
//
//     R = b (v - y K S)     (I + L) U = R,  L_ij = b_i D_ij k_i.k_j (j < i)     X = (I + L)^-1
//     O = scale y Q S + P U,  P_ij = scale D_ij q_i.k_j (j <= i)                 S' = exp(G_last) S + (e K)' U
//
// X, P, y and e do not depend on the state: they are made for all blocks at once (prepare).  What is left is a walk over the
// blocks, in which the columns of S do not meet: a workgroup takes 16 of them and holds them in its accumulators (walk).
// The gradient walks back, with dS' what reaches S' and dO what reaches O,
//
//     dU = P' dO + e K dS'     dR = X' dU     dv = b dR     dS = exp(G_last) dS' + scale Q' (y dO) - K' (y b dR)
//
// and leaves dS' and dR; the rest of the gradient again is made for all blocks at once (gradient).  A wave of 64 lanes holds
// one value for each step of a block.  Running sums of g, and what is taken from each other of them, are in 64 bits: with
// strong decay a sum over 64 steps has lost what the difference of two neighbours needs.
#include "common.h"
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>

namespace l355 {

namespace {

constexpr int C = kDeltaSteps;              // steps of a block, one for each lane
constexpr int kWaves = 4;                   // of a workgroup; each takes 16 steps of a block
constexpr int kTile = 16;                   // columns of S of a workgroup
constexpr int kCols = 20;                   // its row in LDS where columns lie side by side
constexpr int kRow = C + 4;                 // row in LDS with a value for each step
constexpr int kPrepared = 2 * C * C + 2 * C;   // X, P, y, e of a block
static_assert(C == 64 && kWaves * 16 == C, "");

// The matrix instruction of fp32: lane (r, g) = (lane & 15, lane >> 4) gives rows r of A and columns r of B at k = g; four of
// them take k = 4 g .. 4 g + 3 from a lane, in whatever order, so both operands are read four neighbouring k at a time.  Lane (r, g)
// ends with rows 4 g .. 4 g + 3 of column r: what the next product takes as its B.
__device__ __forceinline__ f32x4v mfma16(f32x4v a, f32x4v b, f32x4v c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x4v at4(const float* p) { return *(const f32x4v*)p; }
// four values a row apart
__device__ __forceinline__ f32x4v down4(const float* p, int ld) { return (f32x4v){p[0], p[ld], p[2 * ld], p[3 * ld]}; }
__device__ __forceinline__ f32x4v scaled4(f32x4v v, float s) { return (f32x4v){v[0] * s, v[1] * s, v[2] * s, v[3] * s}; }
__device__ __forceinline__ f32x4v times4(f32x4v a, f32x4v b) { return (f32x4v){a[0] * b[0], a[1] * b[1], a[2] * b[2], a[3] * b[3]}; }
constexpr f32x4v kZero4 = {0.f, 0.f, 0.f, 0.f};

// columns col .. col + 3 of a row that has `width` of them; 0 behind it
template <class E>
__device__ __forceinline__ f32x4v load4(const typename E::T* row, int col, int width)
{
    float v[4];
    if (col + 4 <= width) {
        load_n<E, 4, true>(row + col, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = col + i < width ? E::load(row + col + i) : 0.f;
    }
    return (f32x4v){v[0], v[1], v[2], v[3]};
}

// Where a workgroup is: block c of sequence b and head h, `n` steps of it inside the sequence
struct Block {
    int c, b, h, n;
    int64_t t0;
    int64_t index;      // among all of [blocks, B, heads]
};
__device__ __forceinline__ int length_of(const DeltaArgs& a, int b) { return a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T; }
__device__ __forceinline__ Block block_of(const DeltaArgs& a, int c, int b, int h)
{
    Block k;
    k.c = c;
    k.b = b;
    k.h = h;
    k.t0 = (int64_t)c * C;
    k.n = (int)min((int64_t)length_of(a, b) - k.t0, (int64_t)C);
    k.index = ((int64_t)c * a.B + b) * a.heads + h;
    return k;
}
template <class E>
__device__ __forceinline__ const typename E::T* row_of(const void* p, int64_t t_stride, int64_t b_stride, int64_t t, int b, int64_t first)
{
    return (const typename E::T*)p + t * t_stride + b * b_stride + first;
}
__device__ __forceinline__ int blocks_of(int T) { return (T + C - 1) / C; }
__device__ __forceinline__ float* prepared_of(const DeltaArgs& a, int64_t block) { return a.ws + block * kPrepared; }
__device__ __forceinline__ float* dstate_of(const DeltaArgs& a, int64_t block)
{
    return a.ws + (int64_t)blocks_of(a.T) * a.B * a.heads * kPrepared + block * a.Dk * a.Dv;
}
// dR of a block, and behind it e K dS'
__device__ __forceinline__ float* dupdate_of(const DeltaArgs& a, int64_t block)
{
    return a.ws + (int64_t)blocks_of(a.T) * a.B * a.heads * (kPrepared + (int64_t)a.Dk * a.Dv) + block * 2 * C * a.Dv;
}
// dq and dk of a block and key head, while not all of its heads have been added
__device__ __forceinline__ float* shared_of(const DeltaArgs& a, int64_t key_block)
{
    return a.ws + (int64_t)blocks_of(a.T) * a.B * a.heads * (kPrepared + (int64_t)(a.Dk + 2 * C) * a.Dv) + key_block * 2 * C * a.Dk;
}

// Workgroups that read the same keys and queries follow each other on one XCD: hardware deals consecutive ones over eight.
__device__ __forceinline__ unsigned by_xcd(unsigned blk, unsigned total)
{
    const unsigned each = total / 8, more = total % 8, x = blk % 8, i = blk / 8;
    return x * each + min(x, more) + i;
}

// Rows t0 .. t0 + 63 of keys or queries in LDS, 0 behind the sequence's end and behind the row
template <class E, int DKP>
__device__ __forceinline__ void stage(const typename E::T* first, int64_t t_stride, int n, int width, float* to)
{
    constexpr int kPieces = DKP / 4;
#pragma unroll 4
    for (int p = threadIdx.x; p < C * kPieces; p += 64 * kWaves) {
        const int row = p / kPieces, col = p % kPieces * 4;
        *(f32x4v*)(to + row * (DKP + 4) + col) = row < n ? load4<E>(first + row * t_stride, col, width) : kZero4;
    }
}

// A decay below exp(-10000) is 0 in fp32, and so is every product that has it; NaN stays NaN.
constexpr float kForgets = -1e4f;
// running sum of g over the lanes; behind the end it stays
__device__ __forceinline__ double running(const DeltaArgs& a, const Block& k, int lane)
{
    float g = 0.f;
    if (a.g && lane < k.n) {
        g = *row_of<F32>(a.g, a.g_t, a.g_b, k.t0 + lane, k.b, k.h);
        g = g < kForgets ? kForgets : g;
    }
    double G = g;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double before = __shfl_up(G, off);
        if (lane >= off) G += before;
    }
    return G;
}
__device__ __forceinline__ float beta_at(const DeltaArgs& a, const Block& k, int step)
{
    return step < k.n ? *row_of<F32>(a.beta, a.beta_t, a.beta_b, k.t0 + step, k.b, k.h) : 0.f;
}

// X, P, y and e of every block.  X is built of blocks of 16: those on the diagonal by substitution, a column to a lane; then
// X_ij = -X_ii sum_k L_ik X_kj, those one off the diagonal first.
template <class E, int DKP>
__global__ __launch_bounds__(64 * kWaves) void delta_prepare_kernel(DeltaArgs a)
{
    extern __shared__ float lds[];
    __shared__ double Gs[C];
    __shared__ float betas[C];
    constexpr int LD = DKP + 4;
    float *const Ks = lds, *const Qs = lds + C * LD;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const Block k = block_of(a, (int)(id / a.heads / a.B), (int)(id / a.heads % a.B), (int)(id % a.heads));
    if (k.n <= 0) return;
    const int hk = k.h / (a.heads / a.key_heads);
    stage<E, DKP>(row_of<E>(a.k, a.k_t, a.k_b, k.t0, k.b, (int64_t)hk * a.Dk), a.k_t, k.n, a.Dk, Ks);
    stage<E, DKP>(row_of<E>(a.q, a.q_t, a.q_b, k.t0, k.b, (int64_t)hk * a.Dk), a.q_t, k.n, a.Dk, Qs);
    float* const out = prepared_of(a, k.index);
    if (w == 0) {
        const double G = running(a, k, lane);
        Gs[lane] = G;
        betas[lane] = beta_at(a, k, lane);
        out[2 * C * C + lane] = expf((float)G);
        out[2 * C * C + C + lane] = expf((float)(__shfl(G, 63) - G));
    }
    __syncthreads();
    f32x4v kk[4], qk[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) kk[j] = qk[j] = kZero4;
#pragma unroll 2
    for (int d = 0; d < DKP; d += 16) {
        const f32x4v ka = at4(Ks + (16 * w + r) * LD + d + 4 * g), qa = at4(Qs + (16 * w + r) * LD + d + 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j > w) continue;
            const f32x4v kb = at4(Ks + (16 * j + r) * LD + d + 4 * g);
            kk[j] = mfma16(ka, kb, kk[j]);
            qk[j] = mfma16(qa, kb, qk[j]);
        }
    }
    __syncthreads();
    float *const Ls = Ks, *const Xs = Qs;       // which are not needed any more
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * w + 4 * g + i, col = 16 * j + r;
            float l = 0.f, p = 0.f;
            if (col <= row && row < k.n) {
                const float decay = expf((float)(Gs[row] - Gs[col]));
                p = a.scale * decay * qk[j][i];
                if (col < row) l = betas[row] * decay * kk[j][i];
            }
            Ls[row * kRow + col] = l;
            Xs[row * kRow + col] = 0.f;
            out[C * C + row * C + col] = p;
        }
    __syncthreads();
    if (lane < 16) {
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float v = i == lane ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < i; ++j) v = fmaf(-Ls[(16 * w + i) * kRow + 16 * w + j], x[j], v);
            x[i] = v;
            Xs[(16 * w + i) * kRow + 16 * w + lane] = v;
        }
    }
#pragma unroll
    for (int off = 1; off < 4; ++off) {
        __syncthreads();
        if (w < off) continue;
        const int i = w, j = w - off;
        f32x4v sum = kZero4;
        for (int m = j; m < i; ++m)
            sum = mfma16(at4(Ls + (16 * i + r) * kRow + 16 * m + 4 * g), down4(Xs + (16 * m + 4 * g) * kRow + 16 * j + r, kRow), sum);
        sum = mfma16(at4(Xs + (16 * i + r) * kRow + 16 * i + 4 * g), sum, kZero4);
#pragma unroll
        for (int q = 0; q < 4; ++q) Xs[(16 * i + 4 * g + q) * kRow + 16 * j + r] = -sum[q];
    }
    __syncthreads();
    for (int p = threadIdx.x; p < C * C / 4; p += 64 * kWaves)
        *(f32x4v*)(out + p * 4) = at4(Xs + p / 16 * kRow + p % 16 * 4);
}

// Forward: the walk over the blocks of one sequence and head, 16 columns of S.
template <class E, int DKP>
__global__ __launch_bounds__(64 * kWaves) void delta_walk_kernel(DeltaArgs a, int tiles)
{
    using T = typename E::T;
    extern __shared__ float lds[];
    constexpr int LD = DKP + 4, kParts = DKP / 64;      // tiles of 16 rows of S that a wave holds
    float *const Ks = lds, *const Ss = Ks + C * LD, *const Rs = Ss + kTile * LD, *const Us = Rs + kTile * kRow, *const Es = Us + kTile * kRow;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const int tile = (int)(id % tiles), h = (int)(id / tiles % a.heads), b = (int)(id / tiles / a.heads);
    const int hk = h / (a.heads / a.key_heads), col = tile * kTile + r;
    const bool live = col < a.Dv;
    const int len = length_of(a, b);
    const int64_t state = ((int64_t)b * a.heads + h) * a.Dk * a.Dv;
    f32x4v S[kParts];
#pragma unroll
    for (int m = 0; m < kParts; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = 16 * (w * kParts + m) + 4 * g + i;
            S[m][i] = a.S0 && live && d < a.Dk ? a.S0[state + (int64_t)d * a.Dv + col] : 0.f;
        }
    const int blocks = (len + C - 1) / C;
    for (int c = 0; c < blocks; ++c) {
        const Block k = block_of(a, c, b, h);
        const float* const ready = prepared_of(a, k.index);
        stage<E, DKP>(row_of<E>(a.k, a.k_t, a.k_b, k.t0, b, (int64_t)hk * a.Dk), a.k_t, k.n, a.Dk, Ks);
#pragma unroll
        for (int m = 0; m < kParts; ++m) *(f32x4v*)(Ss + r * LD + 16 * (w * kParts + m) + 4 * g) = S[m];
        if (a.states) {
            float* const to = a.states + ((int64_t)c * a.B * a.heads * a.Dk * a.Dv) + state;
#pragma unroll
            for (int m = 0; m < kParts; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = 16 * (w * kParts + m) + 4 * g + i;
                    if (live && d < a.Dk) to[(int64_t)d * a.Dv + col] = S[m][i];
                }
        }
        const int row = 16 * w + 4 * g;                 // the lane's four steps
        const f32x4v y = at4(ready + 2 * C * C + row), e = at4(ready + 2 * C * C + C + row);
        const float last = ready[2 * C * C + C - 1];
        float beta[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            beta[i] = beta_at(a, k, row + i);
            v[i] = live && row + i < k.n ? E::load(row_of<E>(a.v, a.v_t, a.v_b, k.t0 + row + i, b, (int64_t)h * a.Dv + col)) : 0.f;
        }
        __syncthreads();
        f32x4v ks = kZero4, qs = kZero4;
        const T* const q_row = row_of<E>(a.q, a.q_t, a.q_b, k.t0 + 16 * w + r, b, (int64_t)hk * a.Dk);
        const bool inside = 16 * w + r < k.n;
#pragma unroll 4
        for (int d = 0; d < DKP; d += 16) {
            const f32x4v s = at4(Ss + r * LD + d + 4 * g);
            ks = mfma16(at4(Ks + (16 * w + r) * LD + d + 4 * g), s, ks);
            qs = mfma16(inside ? load4<E>(q_row, d + 4 * g, a.Dk) : kZero4, s, qs);
        }
        f32x4v R;
#pragma unroll
        for (int i = 0; i < 4; ++i) R[i] = beta[i] * (v[i] - y[i] * ks[i]);
        *(f32x4v*)(Rs + r * kRow + row) = R;
        __syncthreads();
        f32x4v U = kZero4;
        for (int j = 0; j <= w; ++j) U = mfma16(at4(ready + (16 * w + r) * C + 16 * j + 4 * g), at4(Rs + r * kRow + 16 * j + 4 * g), U);
        *(f32x4v*)(Us + r * kRow + row) = U;
        *(f32x4v*)(Es + r * kRow + row) = times4(U, e);
        __syncthreads();
        f32x4v O;
#pragma unroll
        for (int i = 0; i < 4; ++i) O[i] = a.scale * y[i] * qs[i];
        for (int j = 0; j <= w; ++j) O = mfma16(at4(ready + C * C + (16 * w + r) * C + 16 * j + 4 * g), at4(Us + r * kRow + 16 * j + 4 * g), O);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (live && row + i < k.n)
                E::store((T*)row_of<E>(a.o, a.o_t, a.o_b, k.t0 + row + i, b, (int64_t)h * a.Dv + col), O[i]);
#pragma unroll
        for (int m = 0; m < kParts; ++m) {
            S[m] = scaled4(S[m], last);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                S[m] = mfma16(down4(Ks + (16 * j + 4 * g) * LD + 16 * (w * kParts + m) + r, LD), at4(Es + r * kRow + 16 * j + 4 * g), S[m]);
        }
        __syncthreads();
    }
    if (a.ST)
#pragma unroll
        for (int m = 0; m < kParts; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 16 * (w * kParts + m) + 4 * g + i;
                if (live && d < a.Dk) a.ST[state + (int64_t)d * a.Dv + col] = S[m][i];
            }
    for (int64_t t = len + (threadIdx.x >> 4); t < a.T; t += 4 * kWaves)
        if (live) E::store((T*)row_of<E>(a.o, a.o_t, a.o_b, t, b, (int64_t)h * a.Dv + col), 0.f);
}

// Few steps: a thread holds four columns of every 32nd row of S, eight threads 32 columns of a row; the sums over the rows of
// what key and query find meet in LDS once a step, and
//     u = b (v - a S'k)     o = scale (a S'q + (q.k) u)     S <- a S + k u'
template <class E, int RP>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaArgs a, int tiles)
{
    using T = typename E::T;
    __shared__ float sums[2][4][8][9];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, cg = threadIdx.x & 7, rt = threadIdx.x >> 3;
    const int tile = (int)(blockIdx.x % tiles), h = (int)(blockIdx.x / tiles % a.heads), b = (int)(blockIdx.x / tiles / a.heads);
    const int hk = h / (a.heads / a.key_heads), col = tile * 32 + cg * 4;
    const int len = length_of(a, b);
    const int64_t state = ((int64_t)b * a.heads + h) * a.Dk * a.Dv;
    f32x4v S[RP];
#pragma unroll
    for (int p = 0; p < RP; ++p) {
        const int d = rt + 32 * p;
        S[p] = a.S0 && d < a.Dk ? load4<F32>(a.S0 + state + (int64_t)d * a.Dv, col, a.Dv) : kZero4;
    }
    const auto store_state = [&](float* to) {
#pragma unroll
        for (int p = 0; p < RP; ++p) {
            const int d = rt + 32 * p;
            if (d >= a.Dk) continue;
            float* const row = to + state + (int64_t)d * a.Dv;
            if (col + 4 <= a.Dv) {
                *(f32x4v_any*)(row + col) = S[p];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (col + i < a.Dv) row[col + i] = S[p][i];
            }
        }
    };
    for (int t = 0; t < len; ++t) {
        if (a.states && t % C == 0) store_state(a.states + (int64_t)(t / C) * a.B * a.heads * a.Dk * a.Dv);
        const T* const k_row = row_of<E>(a.k, a.k_t, a.k_b, t, b, (int64_t)hk * a.Dk);
        const T* const q_row = row_of<E>(a.q, a.q_t, a.q_b, t, b, (int64_t)hk * a.Dk);
        const f32x4v v = load4<E>(row_of<E>(a.v, a.v_t, a.v_b, t, b, (int64_t)h * a.Dv), col, a.Dv);
        const float beta = *row_of<F32>(a.beta, a.beta_t, a.beta_b, t, b, h);
        const float decay = a.g ? expf(*row_of<F32>(a.g, a.g_t, a.g_b, t, b, h)) : 1.f;
        float k[RP], part[9] = {};
#pragma unroll
        for (int p = 0; p < RP; ++p) {
            const int d = rt + 32 * p;
            k[p] = d < a.Dk ? E::load(k_row + d) : 0.f;
            const float q = d < a.Dk ? E::load(q_row + d) : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                part[i] = fmaf(k[p], S[p][i], part[i]);
                part[4 + i] = fmaf(q, S[p][i], part[4 + i]);
            }
            part[8] = fmaf(q, k[p], part[8]);
        }
#pragma unroll
        for (int i = 0; i < 9; ++i) {
            part[i] += __shfl_xor(part[i], 8);
            part[i] += __shfl_xor(part[i], 16);
            part[i] += __shfl_xor(part[i], 32);
        }
        if (lane < 8)
#pragma unroll
            for (int i = 0; i < 9; ++i) sums[t & 1][w][cg][i] = part[i];
        __syncthreads();        // one is enough: the other buffer is written next
#pragma unroll
        for (int i = 0; i < 9; ++i) part[i] = sums[t & 1][0][cg][i] + sums[t & 1][1][cg][i] + sums[t & 1][2][cg][i] + sums[t & 1][3][cg][i];
        float u[4], o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[i] = beta * (v[i] - decay * part[i]);
            o[i] = a.scale * fmaf(part[8], u[i], decay * part[4 + i]);
#pragma unroll
            for (int p = 0; p < RP; ++p) S[p][i] = fmaf(k[p], u[i], decay * S[p][i]);
        }
        if (rt == 0) {
            T* const to = (T*)row_of<E>(a.o, a.o_t, a.o_b, t, b, (int64_t)h * a.Dv);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < a.Dv) E::store(to + col + i, o[i]);
        }
    }
    if (a.ST) store_state(a.ST);
    for (int64_t t = len + rt; t < a.T; t += 32)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < a.Dv) E::store((T*)row_of<E>(a.o, a.o_t, a.o_b, t, b, (int64_t)h * a.Dv) + col + i, 0.f);
}

// Gradient: the walk back over the blocks, 16 columns of dS.
template <class E, int DKP>
__global__ __launch_bounds__(64 * kWaves) void delta_walk_back_kernel(DeltaArgs a, int tiles)
{
    using T = typename E::T;
    extern __shared__ float lds[];
    constexpr int LD = DKP + 4, kParts = DKP / 64;
    float *const Ks = lds, *const Qs = Ks + C * LD, *const Ds = Qs + C * LD, *const Os = Ds + kTile * LD, *const Us = Os + kTile * kRow,
                 *const Zs = Us + kTile * kRow;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const int tile = (int)(id % tiles), h = (int)(id / tiles % a.heads), b = (int)(id / tiles / a.heads);
    const int hk = h / (a.heads / a.key_heads), col = tile * kTile + r;
    const bool live = col < a.Dv;
    const int len = length_of(a, b);
    const int64_t state = ((int64_t)b * a.heads + h) * a.Dk * a.Dv;
    f32x4v dS[kParts];
#pragma unroll
    for (int m = 0; m < kParts; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = 16 * (w * kParts + m) + 4 * g + i;
            dS[m][i] = a.dST && live && d < a.Dk ? a.dST[state + (int64_t)d * a.Dv + col] : 0.f;
        }
    for (int c = (len + C - 1) / C - 1; c >= 0; --c) {
        const Block k = block_of(a, c, b, h);
        const float* const ready = prepared_of(a, k.index);
        stage<E, DKP>(row_of<E>(a.k, a.k_t, a.k_b, k.t0, b, (int64_t)hk * a.Dk), a.k_t, k.n, a.Dk, Ks);
        stage<E, DKP>(row_of<E>(a.q, a.q_t, a.q_b, k.t0, b, (int64_t)hk * a.Dk), a.q_t, k.n, a.Dk, Qs);
        float *const behind = dstate_of(a, k.index), *const left = dupdate_of(a, k.index);
#pragma unroll
        for (int m = 0; m < kParts; ++m) {
            *(f32x4v*)(Ds + r * LD + 16 * (w * kParts + m) + 4 * g) = dS[m];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 16 * (w * kParts + m) + 4 * g + i;
                if (live && d < a.Dk) behind[(int64_t)d * a.Dv + col] = dS[m][i];
            }
        }
        const int row = 16 * w + 4 * g;
        const f32x4v y = at4(ready + 2 * C * C + row), e = at4(ready + 2 * C * C + C + row);
        const float last = ready[2 * C * C + C - 1];
        float beta[4];
        f32x4v dO;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            beta[i] = beta_at(a, k, row + i);
            dO[i] = live && row + i < k.n ? E::load(row_of<E>(a.dO, a.do_t, a.do_b, k.t0 + row + i, b, (int64_t)h * a.Dv + col)) : 0.f;
        }
        *(f32x4v*)(Os + r * kRow + row) = dO;
        __syncthreads();
        f32x4v dU = kZero4;
#pragma unroll 4
        for (int d = 0; d < DKP; d += 16) dU = mfma16(at4(Ks + (16 * w + r) * LD + d + 4 * g), at4(Ds + r * LD + d + 4 * g), dU);
        dU = times4(dU, e);
        if (live)
#pragma unroll
            for (int i = 0; i < 4; ++i) left[(int64_t)(C + row + i) * a.Dv + col] = dU[i];
        for (int j = w; j < 4; ++j)
            dU = mfma16(down4(ready + C * C + (16 * j + 4 * g) * C + 16 * w + r, C), at4(Os + r * kRow + 16 * j + 4 * g), dU);
        *(f32x4v*)(Us + r * kRow + row) = dU;
        __syncthreads();
        f32x4v dR = kZero4;
        for (int j = w; j < 4; ++j) dR = mfma16(down4(ready + (16 * j + 4 * g) * C + 16 * w + r, C), at4(Us + r * kRow + 16 * j + 4 * g), dR);
        f32x4v Z;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float dv = beta[i] * dR[i];
            Z[i] = -y[i] * dv;
            if (live) {
                left[(int64_t)(row + i) * a.Dv + col] = dR[i];
                if (row + i < k.n) E::store((T*)row_of<E>(a.dv, a.dv_t, a.dv_b, k.t0 + row + i, b, (int64_t)h * a.Dv + col), dv);
            }
        }
        *(f32x4v*)(Zs + r * kRow + row) = Z;
        __syncthreads();
        f32x4v from_o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            from_o[j] = times4(at4(Os + r * kRow + 16 * j + 4 * g), scaled4(at4(ready + 2 * C * C + 16 * j + 4 * g), a.scale));
#pragma unroll
        for (int m = 0; m < kParts; ++m) {
            dS[m] = scaled4(dS[m], last);
            const int d = 16 * (w * kParts + m) + r;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                dS[m] = mfma16(down4(Qs + (16 * j + 4 * g) * LD + d, LD), from_o[j], dS[m]);
                dS[m] = mfma16(down4(Ks + (16 * j + 4 * g) * LD + d, LD), at4(Zs + r * kRow + 16 * j + 4 * g), dS[m]);
            }
        }
        __syncthreads();
    }
    if (a.dS0)
#pragma unroll
        for (int m = 0; m < kParts; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 16 * (w * kParts + m) + 4 * g + i;
                if (live && d < a.Dk) a.dS0[state + (int64_t)d * a.Dv + col] = dS[m][i];
            }
    for (int64_t t = len + (threadIdx.x >> 4); t < a.T; t += 4 * kWaves)
        if (live) E::store((T*)row_of<E>(a.dv, a.dv_t, a.dv_b, t, b, (int64_t)h * a.Dv + col), 0.f);
}

// sum over the 16 lanes that hold the columns of a row
__device__ __forceinline__ float row16_sum(float v)
{
    v += dpp_move<0xB1>(v);
    v += dpp_move<0x4E>(v);
    v += dpp_move<0x141>(v);
    return v + dpp_move<0x140>(v);
}
// the value N lanes in front in the row of 16; 0 where there is none
template <int N>
__device__ __forceinline__ float row16_shifted(float v) { return dpp_move<0x110 + N>(v); }

// What is left of a block's gradient, from the state S in front of it, dS' behind it and dR: with U made again,
//
//     dP = D (scale dO U')     dA = -b D (dR U') below the diagonal      dq = scale y dO S' + dP K
//     dk = e U dS'' - y b dR S' + dP' Q + (dA + dA') K                   db = dR.(v - y K S) - sum_j dR.U_j D k.k_j
//     dg_t = sum_{i >= t > j} (dA_ij k_i.k_j + dP_ij q_i.k_j) + sum_{i >= t} (q.(scale y dO S') - y b dR.(K S))_i
//            + sum_{j < t} U.(e K dS')_j + exp(G_last) S.dS'
//
// (each decay's own terms; as differences of what reaches two neighbouring G, what a strong decay leaves of dg would be lost).
// A workgroup takes a block of one sequence and key head and goes through the heads that share it, 16 columns of S at a time.
template <class E, int DKP>
__global__ __launch_bounds__(64 * kWaves) void delta_gradient_kernel(DeltaArgs a)
{
    using T = typename E::T;
    extern __shared__ float lds[];
    constexpr int LD = DKP + 4, kParts = DKP / 16;
    // keys (for a while queries) | S and dS', U, R of a tile of columns; in their place later dP and dA
    float *const Ks = lds, *const Ss = Ks + C * LD, *const Ds = Ss + DKP * kCols, *const Us = Ds + DKP * kCols, *const Rs = Us + C * kCols;
    float *const Ps = Ss, *const As = Ss + C * kRow;
    __shared__ double Gs[C];
    __shared__ float ys[C], es[C], betas[C], overs[kWaves][C], fronts[C], backs[C], dbs[C], dots[kWaves];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const int c = (int)(id / a.key_heads / a.B), b = (int)(id / a.key_heads % a.B), hk = (int)(id % a.key_heads), group = a.heads / a.key_heads;
    const int64_t t0 = (int64_t)c * C;
    const int n = (int)min((int64_t)length_of(a, b) - t0, (int64_t)C), rows = (int)min((int64_t)a.T - t0, (int64_t)C);
    const int row = 16 * w + 4 * g, mine = 16 * w + r;          // the lane's steps as results, and its step as first operand
    float* const shared = shared_of(a, ((int64_t)c * a.B + b) * a.key_heads + hk);
    const T* const k_first = row_of<E>(a.k, a.k_t, a.k_b, t0, b, (int64_t)hk * a.Dk);
    const T* const q_first = row_of<E>(a.q, a.q_t, a.q_b, t0, b, (int64_t)hk * a.Dk);
    for (int hh = 0; hh < group; ++hh) {
        const Block k = block_of(a, c, b, hk * group + hh);
        if (n <= 0) {
            if (w == 0 && lane < rows) {
                if (a.dg) *(float*)row_of<F32>(a.dg, a.dg_t, a.dg_b, t0 + lane, b, k.h) = 0.f;
                *(float*)row_of<F32>(a.dbeta, a.dbeta_t, a.dbeta_b, t0 + lane, b, k.h) = 0.f;
            }
            continue;
        }
        const float *const ready = prepared_of(a, k.index), *const behind = dstate_of(a, k.index), *const left = dupdate_of(a, k.index);
        const float* const front = a.states + k.index * a.Dk * a.Dv;
        stage<E, DKP>(k_first, a.k_t, n, a.Dk, Ks);
        if (w == 0) {
            Gs[lane] = running(a, k, lane);
            ys[lane] = ready[2 * C * C + lane];
            es[lane] = ready[2 * C * C + C + lane];
            betas[lane] = beta_at(a, k, lane);
        }
        __syncthreads();
        f32x4v dP[4], dL[4], y, beta;
        f32x4v dq[kParts], dk[kParts];
#pragma unroll
        for (int m = 0; m < kParts; ++m) dq[m] = dk[m] = kZero4;
        float db[4], from_front[4], to_back[4], dot = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) dP[j] = dL[j] = kZero4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = ys[row + i];
            beta[i] = betas[row + i];
            db[i] = from_front[i] = to_back[i] = 0.f;
        }
        const float y_mine = ys[mine], e_mine = es[mine], yb_mine = -y_mine * betas[mine];
        for (int c0 = 0; c0 < a.Dv; c0 += kTile) {
            __syncthreads();
#pragma unroll
            for (int p = threadIdx.x; p < DKP * 4; p += 64 * kWaves) {
                const int d = p / 4, at = c0 + p % 4 * 4;
                const f32x4v s = d < a.Dk ? load4<F32>(front + (int64_t)d * a.Dv, at, a.Dv) : kZero4;
                const f32x4v ds = d < a.Dk ? load4<F32>(behind + (int64_t)d * a.Dv, at, a.Dv) : kZero4;
                *(f32x4v*)(Ss + d * kCols + p % 4 * 4) = s;
                *(f32x4v*)(Ds + d * kCols + p % 4 * 4) = ds;
#pragma unroll
                for (int i = 0; i < 4; ++i) dot = fmaf(s[i], ds[i], dot);
            }
            const int col = c0 + r;
            float v[4], dR[4], found[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool there = col < a.Dv && row + i < n;
                v[i] = there ? E::load(row_of<E>(a.v, a.v_t, a.v_b, t0 + row + i, b, (int64_t)k.h * a.Dv + col)) : 0.f;
                dR[i] = there ? left[(int64_t)(row + i) * a.Dv + col] : 0.f;
                found[i] = there ? left[(int64_t)(C + row + i) * a.Dv + col] : 0.f;
            }
            const bool has = mine < n;
            const f32x4v dO_mine = has ? scaled4(load4<E>(row_of<E>(a.dO, a.do_t, a.do_b, t0 + mine, b, (int64_t)k.h * a.Dv), c0 + 4 * g, a.Dv), a.scale) : kZero4;
            const f32x4v dR_mine = has ? load4<F32>(left + (int64_t)mine * a.Dv, c0 + 4 * g, a.Dv) : kZero4;
            __syncthreads();
            f32x4v ks = kZero4;
#pragma unroll 4
            for (int d = 0; d < DKP; d += 16) ks = mfma16(at4(Ks + mine * LD + d + 4 * g), down4(Ss + (d + 4 * g) * kCols + r, kCols), ks);
            f32x4v R;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float miss = v[i] - y[i] * ks[i];
                R[i] = beta[i] * miss;
                db[i] = fmaf(dR[i], miss, db[i]);
                from_front[i] = fmaf(-y[i] * beta[i] * dR[i], ks[i], from_front[i]);
            }
            *(f32x4v*)(Rs + r * kRow + row) = R;
            __syncthreads();
            f32x4v U = kZero4;
            for (int j = 0; j <= w; ++j) U = mfma16(at4(ready + mine * C + 16 * j + 4 * g), at4(Rs + r * kRow + 16 * j + 4 * g), U);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                Us[(row + i) * kCols + r] = U[i];
                to_back[i] = fmaf(U[i], found[i], to_back[i]);
            }
            __syncthreads();
            const f32x4v yO = scaled4(dO_mine, y_mine), eU = scaled4(at4(Us + mine * kCols + 4 * g), e_mine), Z = scaled4(dR_mine, yb_mine);
#pragma unroll
            for (int m = 0; m < kParts; ++m) {
                const f32x4v s = at4(Ss + (16 * m + r) * kCols + 4 * g);
                dq[m] = mfma16(yO, s, dq[m]);
                dk[m] = mfma16(Z, s, dk[m]);
                dk[m] = mfma16(eU, at4(Ds + (16 * m + r) * kCols + 4 * g), dk[m]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j > w) continue;
                const f32x4v u = at4(Us + (16 * j + r) * kCols + 4 * g);
                dP[j] = mfma16(dO_mine, u, dP[j]);
                dL[j] = mfma16(dR_mine, u, dL[j]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int m = 0; m < kParts; ++m) {
                const int d = 16 * m + r;
                const float q = row + i < n && d < a.Dk ? E::load(q_first + (row + i) * a.q_t + d) : 0.f;
                from_front[i] = fmaf(q, dq[m][i], from_front[i]);
            }
        f32x4v kk[4], qk[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kk[j] = qk[j] = kZero4;
#pragma unroll 2
        for (int d = 0; d < DKP; d += 16) {
            const f32x4v ka = at4(Ks + mine * LD + d + 4 * g), qa = mine < n ? load4<E>(q_first + mine * a.q_t, d + 4 * g, a.Dk) : kZero4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j > w) continue;
                const f32x4v kb = at4(Ks + (16 * j + r) * LD + d + 4 * g);
                kk[j] = mfma16(ka, kb, kk[j]);
                qk[j] = mfma16(qa, kb, qk[j]);
            }
        }
        float in_front[4] = {};     // pairs of the lane's steps with all steps of the tiles in front of this one
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float over = 0.f;       // pairs that the decay at step 16 j + r lies between, of the lane's steps
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = row + i, other = 16 * j + r;
                float p = 0.f, l = 0.f, pair = 0.f;
                if (j <= w && other <= at && at < n) {
                    const float decay = expf((float)(Gs[at] - Gs[other]));
                    p = decay * dP[j][i];
                    if (other < at) {
                        l = decay * dL[j][i];
                        db[i] = fmaf(-l, kk[j][i], db[i]);
                        l *= -beta[i];
                        pair = fmaf(l, kk[j][i], p * qk[j][i]);
                    }
                }
                if (j <= w) {
                    Ps[at * kRow + other] = p;
                    As[at * kRow + other] = l;
                }
                // over the steps in front of 16 j + r: the 16 of the tile by shifts along the row of lanes
                float sum = row16_shifted<1>(pair);
                sum += row16_shifted<1>(sum);
                sum += row16_shifted<2>(sum);
                sum += row16_shifted<4>(sum);
                sum += row16_shifted<8>(sum);
                if (other <= at) over += in_front[i] + sum;
                in_front[i] += row16_sum(pair);
            }
            over += __shfl_xor(over, 16);
            over += __shfl_xor(over, 32);
            if (g == 0) overs[w][16 * j + r] = over;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = row16_sum(from_front[i]), l = row16_sum(to_back[i]), d = row16_sum(db[i]);
            if (r == 0) {
                fronts[row + i] = f;
                backs[row + i] = l;
                dbs[row + i] = d;
            }
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) dot += __shfl_xor(dot, off);
        if (lane == 0) dots[w] = dot;
        __syncthreads();
        if (w == 0) {
            double from = fronts[lane], to = backs[lane], dg = (double)overs[0][lane] + overs[1][lane] + overs[2][lane] + overs[3][lane];
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const double after = __shfl_down(from, off), before = __shfl_up(to, off);
                if (lane + off < 64) from += after;
                if (lane >= off) to += before;
            }
            to = __shfl_up(to, 1);
            dg += from + (lane > 0 ? to : 0.0) + (double)ys[C - 1] * ((double)dots[0] + dots[1] + dots[2] + dots[3]);
            if (lane < rows) {
                if (a.dg) *(float*)row_of<F32>(a.dg, a.dg_t, a.dg_b, t0 + lane, b, k.h) = lane < n ? (float)dg : 0.f;
                *(float*)row_of<F32>(a.dbeta, a.dbeta_t, a.dbeta_b, t0 + lane, b, k.h) = lane < n ? dbs[lane] : 0.f;
            }
        }
        f32x4v both[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            both[j] = kZero4;
            if (j <= w) both[j] += at4(As + mine * kRow + 16 * j + 4 * g);
            if (j >= w) both[j] += down4(As + (16 * j + 4 * g) * kRow + mine, kRow);
        }
#pragma unroll 2
        for (int m = 0; m < kParts; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4v kb = down4(Ks + (16 * j + 4 * g) * LD + 16 * m + r, LD);
                if (j <= w) dq[m] = mfma16(at4(Ps + mine * kRow + 16 * j + 4 * g), kb, dq[m]);
                dk[m] = mfma16(both[j], kb, dk[m]);
            }
        __syncthreads();
        stage<E, DKP>(q_first, a.q_t, n, a.Dk, Ks);
        __syncthreads();
#pragma unroll 2
        for (int m = 0; m < kParts; ++m)
            for (int j = w; j < 4; ++j)
                dk[m] = mfma16(down4(Ps + (16 * j + 4 * g) * kRow + mine, kRow), down4(Ks + (16 * j + 4 * g) * LD + 16 * m + r, LD), dk[m]);
        __syncthreads();
#pragma unroll
        for (int m = 0; m < kParts; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 16 * m + r;
                if (d >= a.Dk || row + i >= rows) continue;
                float* const part = shared + (row + i) * a.Dk + d;
                float vq = row + i < n ? dq[m][i] : 0.f, vk = row + i < n ? dk[m][i] : 0.f;
                if (hh > 0) {
                    vq += part[0];
                    vk += part[C * a.Dk];
                }
                if (hh + 1 < group) {
                    part[0] = vq;
                    part[C * a.Dk] = vk;
                } else {
                    E::store((T*)row_of<E>(a.dq, a.dq_t, a.dq_b, t0 + row + i, b, (int64_t)hk * a.Dk + d), vq);
                    E::store((T*)row_of<E>(a.dk, a.dk_t, a.dk_b, t0 + row + i, b, (int64_t)hk * a.Dk + d), vk);
                }
            }
    }
    if (n > 0) return;
    for (int p = threadIdx.x; p < rows * a.Dk; p += 64 * kWaves) {
        E::store((T*)row_of<E>(a.dq, a.dq_t, a.dq_b, t0 + p / a.Dk, b, (int64_t)hk * a.Dk + p % a.Dk), 0.f);
        E::store((T*)row_of<E>(a.dk, a.dk_t, a.dk_b, t0 + p / a.Dk, b, (int64_t)hk * a.Dk + p % a.Dk), 0.f);
    }
}

// ---- host

constexpr int kFewSteps = 8;

int64_t blocks(int T) { return (T + C - 1) / C; }

template <class Kernel>
hipError_t launch(Kernel kernel, int64_t grid, size_t lds_floats, const DeltaArgs& a, int tiles, hipStream_t s)
{
    const size_t lds = lds_floats * sizeof(float);
    const hipError_t e = allow_dynamic_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kWaves), lds, s, a, tiles);
    return hipGetLastError();
}
template <class Kernel>
hipError_t launch(Kernel kernel, int64_t grid, size_t lds_floats, const DeltaArgs& a, hipStream_t s)
{
    const size_t lds = lds_floats * sizeof(float);
    const hipError_t e = allow_dynamic_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kWaves), lds, s, a);
    return hipGetLastError();
}

template <class E, int DKP>
hipError_t prepare(const DeltaArgs& a, hipStream_t s)
{
    return launch(delta_prepare_kernel<E, DKP>, blocks(a.T) * a.B * a.heads, 2 * C * (DKP + 4), a, s);
}

template <class E, int DKP>
hipError_t forward(const DeltaArgs& a, hipStream_t s)
{
    if (a.T <= kFewSteps) {
        const int tiles = (a.Dv + 31) / 32;
        hipLaunchKernelGGL((delta_step_kernel<E, DKP / 32>), dim3((unsigned)((int64_t)a.B * a.heads * tiles)), dim3(256), 0, s, a, tiles);
        return hipGetLastError();
    }
    const hipError_t e = prepare<E, DKP>(a, s);
    if (e != hipSuccess) return e;
    const int tiles = (a.Dv + kTile - 1) / kTile;
    return launch(delta_walk_kernel<E, DKP>, (int64_t)a.B * a.heads * tiles, (C + kTile) * (DKP + 4) + 3 * kTile * kRow, a, tiles, s);
}

template <class E, int DKP>
hipError_t backward(const DeltaArgs& a, hipStream_t s)
{
    hipError_t e = a.T > 0 ? prepare<E, DKP>(a, s) : hipSuccess;
    if (e != hipSuccess) return e;
    const int tiles = (a.Dv + kTile - 1) / kTile;
    e = launch(delta_walk_back_kernel<E, DKP>, (int64_t)a.B * a.heads * tiles, (2 * C + kTile) * (DKP + 4) + 3 * kTile * kRow, a, tiles, s);
    if (e != hipSuccess || a.T == 0) return e;
    const size_t tile = 2 * DKP * kCols + C * kCols + kTile * kRow;
    return launch(delta_gradient_kernel<E, DKP>, blocks(a.T) * a.B * a.key_heads, C * (DKP + 4) + std::max<size_t>(tile, 2 * C * kRow), a, s);
}

}  // namespace

size_t delta_workspace_bytes(int T, int B, int heads, int key_heads, int Dk, int Dv, bool back)
{
    const size_t each = back ? kPrepared + (size_t)(Dk + 2 * C) * Dv : T <= kFewSteps ? 0 : kPrepared;
    const size_t shared = back && heads > key_heads ? (size_t)key_heads * 2 * C * Dk : 0;
    return std::max<size_t>(256, (size_t)blocks(T) * B * (heads * each + shared) * sizeof(float));
}

// a grid's threads have to stay under 2^32, and what the workspace needs under 2^60
bool delta_fits(int T, int B, int heads, int Dk, int Dv)
{
    const int64_t of_state = (int64_t)B * heads * ((Dv + kTile - 1) / kTile);
    return (int64_t)B * heads < (1 << 24) && of_state < (1 << 24) && blocks(T) * B * heads < (1 << 24);
}

template <class E>
static hipError_t by_width(const DeltaArgs& a, bool back, hipStream_t s)
{
    if (a.Dk <= 64) return back ? backward<E, 64>(a, s) : forward<E, 64>(a, s);
    if (a.Dk <= 128) return back ? backward<E, 128>(a, s) : forward<E, 128>(a, s);
    return back ? backward<E, 256>(a, s) : forward<E, 256>(a, s);
}
hipError_t launch_delta_forward(const DeltaArgs& a, hipStream_t s) { return a.bf16 ? by_width<Bf16>(a, false, s) : by_width<F32>(a, false, s); }
hipError_t launch_delta_backward(const DeltaArgs& a, hipStream_t s) { return a.bf16 ? by_width<Bf16>(a, true, s) : by_width<F32>(a, true, s); }

}  // namespace l355
