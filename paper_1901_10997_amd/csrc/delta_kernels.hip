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
// and leaves dS' and dR; the rest of the gradient again is made for all blocks at once (update, gradient).  A wave of 64 lanes
// holds one value for each step of a block.  Running sums of g, and what is taken from each other of them, are in 64 bits: with
// strong decay a sum over 64 steps has lost what the difference of two neighbours needs.
//
// Products.  The matrix instruction of bf16 is sixteen times as fast as that of fp32, so fp32 values are split into planes, each the
// nearest bf16 to what those in front of it leave: three hold all 24 bits.  The product of planes i and j counts where i + j is below the
// larger number of planes; what is left out is below 2^-24 of the product.  Keys, queries and dO in bf16 are one plane, everything else is three, also where
// the result is rounded to bf16: a sum may be far smaller than its terms.  (Two there were off by 2^-17 of a term; 8192 steps of 16 heads of 128 x 128 bf16
// took 307 us so and take 330, a training step of 8 x 1024 805 and 811.)
#include "common.h"
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>

namespace l355 {

namespace {

constexpr int C = kDeltaSteps;              // steps of a block, one for each lane
constexpr int kWaves = 4;                   // of a workgroup; each takes 16 steps of a block
constexpr int kThreads = 64 * kWaves;
constexpr int kTile = 16;                   // columns of S of a workgroup
constexpr int kRow = C + 4;                 // row of fp32 in LDS with a value for each step
constexpr int kSteps = C + 8;               // row of a plane in LDS with a value for each step
static_assert(C == 64 && kWaves * 16 == C, "");

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16;

// planes of keys, queries and other operands of type E; whether a walk has registers to keep what it could also work out or read again
template <class E>
constexpr int kPlanes = E::kBytes == 2 ? 1 : 3;
template <class E, int DKP, int NT>
constexpr bool kRoom = NT == 1 && DKP / 64 * kPlanes<E> <= 6;

constexpr f32x4v kZero4 = {0.f, 0.f, 0.f, 0.f};
__device__ __forceinline__ f32x4v at4(const float* p) { return *(const f32x4v*)p; }
__device__ __forceinline__ f32x4v scaled4(f32x4v v, float s) { return (f32x4v){v[0] * s, v[1] * s, v[2] * s, v[3] * s}; }
__device__ __forceinline__ f32x4v times4(f32x4v a, f32x4v b) { return (f32x4v){a[0] * b[0], a[1] * b[1], a[2] * b[2], a[3] * b[3]}; }

// The matrix instruction: lane (r, g) = (lane & 15, lane >> 4) gives row r of A and column r of B at k = 8 g .. 8 g + 7 and ends with rows
// 4 g .. 4 g + 3 of column r.  Where one product follows another, each order of planes has a sum of its own, so that they do not wait
// for each other; where there are tiles enough, one holds all.
template <int N>
struct SumsOf {
    f32x4v of[N];
    __device__ __forceinline__ SumsOf()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) of[i] = kZero4;
    }
    __device__ __forceinline__ f32x4v total() const
    {
        if constexpr (N == 1) return of[0];
        else return of[0] + (of[1] + of[2]);
    }
};
typedef SumsOf<3> Sums;
typedef SumsOf<1> Sum;
template <int N, int PA, int PB>
__device__ __forceinline__ void multiply(SumsOf<N>& s, const bf16x8 (&a)[PA], const bf16x8 (&b)[PB])
{
    constexpr int kOrders = PA > PB ? PA : PB;
#pragma unroll
    for (int o = kOrders - 1; o >= 0; --o)
#pragma unroll
        for (int i = 0; i < PA; ++i)
#pragma unroll
            for (int j = 0; j < PB; ++j)
                if (i + j == o) s.of[N == 1 ? 0 : o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], s.of[N == 1 ? 0 : o], 0, 0, 0);
}
// Planes in memory stand as the instruction takes them: tile after tile of 16 rows, of it step after step of 32 k, of it the eight values of
// lane after lane.  (In rows, sixteen lanes that are served together met sixteen lines: the walk took 456 us for 128 blocks, 16 bytes
// a clock.)
constexpr int kFragment = 512;
__device__ __forceinline__ int fragment_at(int tile, int steps, int step) { return (tile * steps + step) * kFragment; }
// the lane's eight values of a fragment (or eight neighbouring k of a row in LDS), in planes `plane` elements apart
template <int N>
__device__ __forceinline__ void fragment(bf16x8 (&f)[N], const u16* p, int64_t plane)
{
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = *(const bf16x8*)(p + i * plane);
}
// four values as planes
template <int N>
__device__ __forceinline__ void split4(f32x4v v, u32x2v (&out)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        out[i] = (u32x2v){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        if (i + 1 < N) {
            v[0] -= bf16_lo(out[i][0]);
            v[1] -= bf16_hi(out[i][0]);
            v[2] -= bf16_lo(out[i][1]);
            v[3] -= bf16_hi(out[i][1]);
        }
    }
}
template <int N>
__device__ __forceinline__ void split8(f32x4v lo, f32x4v hi, bf16x8 (&out)[N])
{
    u32x2v l[N], h[N];
    split4<N>(lo, l);
    split4<N>(hi, h);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = __builtin_bit_cast(bf16x8, (u32x4v){l[i][0], l[i][1], h[i][0], h[i][1]});
}
template <int N>
__device__ __forceinline__ void store_split(f32x4v v, u16* p, int plane)
{
    u32x2v s[N];
    split4<N>(v, s);
#pragma unroll
    for (int i = 0; i < N; ++i) *(u32x2v*)(p + i * plane) = s[i];
}
template <int N>
__device__ __forceinline__ void store_split8(f32x4v lo, f32x4v hi, u16* p, int64_t plane)
{
    bf16x8 s[N];
    split8<N>(lo, hi, s);
#pragma unroll
    for (int i = 0; i < N; ++i) *(bf16x8*)(p + i * plane) = s[i];
}
// A barrier that waits for LDS alone: what is under way from memory stays under way.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// 0 that the compiler does not know: what is worked out from it stays where it stands (addresses of a loop's end, worked out in front of
// the loop, would hold a hundred registers through it).
__device__ __forceinline__ int zero_here()
{
    int z = 0;
    asm volatile("" : "+s"(z));
    return z;
}
// Keeps the loads of a later turn of an unrolled loop out of the turns in front of it, where their registers would not be there.
__device__ __forceinline__ void one_by_one() { asm volatile("" : : : "memory"); }

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

// The same in two steps, without a branch and with nothing that waits in the first, so that loads that follow each other, and what is
// worked on meanwhile, do not wait for them.  WHOLE: width is a multiple of 4, and four columns move at once; else one by one, those
// behind the row standing for its last.
template <class E, bool WHOLE>
struct Four {
    using T = typename E::T;
    T raw[4];
    __device__ __forceinline__ void load(const T* row, int col, int width)
    {
        if constexpr (WHOLE) {
            if constexpr (E::kBytes == 4) __builtin_memcpy(raw, (const f32x4v_any*)(row + min(col, width - 4)), 16);
            else __builtin_memcpy(raw, (const u32x2v_any*)(row + min(col, width - 4)), 8);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = row[min(col + i, width - 1)];
        }
    }
    __device__ __forceinline__ f32x4v take(int col, int width) const
    {
        f32x4v v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (WHOLE ? col : col + i) < width ? E::load(raw + i) : 0.f;
        return v;
    }
};
__device__ __forceinline__ f32x4v if4(bool c, f32x4v v) { return (f32x4v){c ? v[0] : 0.f, c ? v[1] : 0.f, c ? v[2] : 0.f, c ? v[3] : 0.f}; }
// of a row of the workspace, which is padded: columns behind `width` are 0 whatever stands there
__device__ __forceinline__ f32x4v within4(f32x4v v, int col, int width)
{
    return (f32x4v){col < width ? v[0] : 0.f, col + 1 < width ? v[1] : 0.f, col + 2 < width ? v[2] : 0.f, col + 3 < width ? v[3] : 0.f};
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

// What prepare leaves in the workspace, in planes of fragments: for a block and key head K and Q, rows of steps, and K', Q', rows of key columns
// (Q' for the gradient only); for a block and head X and P (or X, X' and P' for the gradient), then y and e.  Rows behind the end
// and columns behind the key's are 0, so that the walks meet neither.  Then, for the gradient, fp32: dS', dR, e K dS', U, what
// tiles of columns add to sums over a step's columns, and dq and dk of heads that share a key.
template <class E, int DKP, bool BACK>
struct Place {
    static constexpr int kP = kPlanes<E>;
    static constexpr int64_t kMatrix = (int64_t)kP * C * DKP, kKeys = (BACK ? 4 : 3) * kMatrix;
    static constexpr int64_t kHead = (BACK ? 9 : 6) * C * C + 4 * C;
    static constexpr int kParts = 256;      // sums of a tile of columns: 64 each of three, and one
    const DeltaArgs& a;
    const int64_t key_blocks, head_blocks;
    __host__ __device__ explicit Place(const DeltaArgs& args)
        : a(args), key_blocks((int64_t)((args.T + C - 1) / C) * args.B * args.key_heads), head_blocks((int64_t)((args.T + C - 1) / C) * args.B * args.heads)
    {
    }
    __host__ __device__ int tiles() const { return (a.Dv + kTile - 1) / kTile; }
    __device__ u16* keys(const Block& k) const
    {
        return (u16*)a.ws + (((int64_t)k.c * a.B + k.b) * a.key_heads + k.h / (a.heads / a.key_heads)) * kKeys;
    }
    __device__ u16* K(const Block& k) const { return keys(k); }
    __device__ u16* KT(const Block& k) const { return keys(k) + kMatrix; }
    __device__ u16* Q(const Block& k) const { return keys(k) + 2 * kMatrix; }
    __device__ u16* QT(const Block& k) const { return keys(k) + 3 * kMatrix; }
    __device__ u16* X(const Block& k) const { return (u16*)a.ws + key_blocks * kKeys + k.index * kHead; }
    __device__ u16* P(const Block& k) const { return X(k) + 3 * C * C; }
    __device__ u16* XT(const Block& k) const { return X(k) + 3 * C * C; }
    __device__ u16* PT(const Block& k) const { return X(k) + 6 * C * C; }
    __device__ float* y(const Block& k) const { return (float*)(X(k) + kHead - 4 * C); }
    __device__ float* e(const Block& k) const { return y(k) + C; }
    __host__ __device__ int64_t first_floats() const { return (key_blocks * kKeys + head_blocks * kHead) / 2; }
    __device__ float* floats() const { return a.ws + first_floats(); }
    __host__ __device__ int row() const { return (a.Dv + 31) / 32 * 32; }       // of the fp32 matrices
    __device__ float* dS(const Block& k) const { return floats() + k.index * a.Dk * row(); }
    __host__ __device__ int64_t of_dS() const { return head_blocks * a.Dk * row(); }
    __device__ float* dR(const Block& k) const { return floats() + of_dS() + k.index * 3 * C * row(); }
    __device__ float* found(const Block& k) const { return dR(k) + C * row(); }
    __device__ float* U(const Block& k) const { return found(k) + C * row(); }
    __host__ __device__ int64_t to_parts() const { return of_dS() + head_blocks * 3 * C * row(); }
    __device__ float* parts(const Block& k, int tile) const { return floats() + to_parts() + (k.index * tiles() + tile) * kParts; }
    __host__ __device__ int64_t to_shared() const { return to_parts() + head_blocks * tiles() * kParts; }
    __device__ float* shared(const Block& k) const
    {
        return floats() + to_shared() + (((int64_t)k.c * a.B + k.b) * a.key_heads + k.h / (a.heads / a.key_heads)) * 2 * C * DKP;
    }
    __host__ __device__ int64_t to_sink() const { return BACK ? to_shared() + (a.heads > a.key_heads ? key_blocks * 2 * C * DKP : 0) : 0; }
    // where lanes write that have nothing to write: a store without a branch leaves the count of what is under way known, so that
    // nobody waits for more than it needs
    __device__ float* sink() const { return floats() + to_sink(); }
    __host__ size_t bytes() const { return (size_t)(first_floats() + to_sink() + 64) * sizeof(float); }
};

// Workgroups that read the same keys and queries follow each other on one XCD: hardware deals consecutive ones over eight.
__device__ __forceinline__ unsigned by_xcd(unsigned blk, unsigned total)
{
    const unsigned each = total / 8, more = total % 8, x = blk % 8, i = blk / 8;
    return x * each + min(x, more) + i;
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

// The matrix instruction of fp32, in the same layout of rows, columns and results at k = 4 g .. 4 g + 3: for products of 16 by 16
// blocks, whose result then is the next one's B as it stands.
__device__ __forceinline__ f32x4v mfma16(f32x4v a, f32x4v b, f32x4v c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x4v down4(const float* p, int ld) { return (f32x4v){p[0], p[ld], p[2 * ld], p[3 * ld]}; }

// Rows of keys or queries in LDS as they come: bf16 in rows of DKP + 8, fp32 in rows of DKP + 4; 0 behind the end and behind the row
template <class E, int DKP>
constexpr int kStaged = E::kBytes == 2 ? DKP + 8 : DKP + 4;
template <class E, int DKP, bool WHOLE>
__device__ __forceinline__ void stage(const typename E::T* first, int64_t t_stride, int n, int width, typename E::T* to)
{
    constexpr int kPieces = DKP / 4;
    constexpr int kEach = WHOLE && C * kPieces / kThreads > 8 ? 8 : C * kPieces / kThreads / (WHOLE ? 1 : 2);
#pragma unroll 1
    for (int p0 = threadIdx.x; p0 < C * kPieces; p0 += kEach * kThreads) {
        Four<E, WHOLE> v[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int p = p0 + i * kThreads;
            v[i].load(first + min(p / kPieces, n - 1) * t_stride, p % kPieces * 4, width);
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int p = p0 + i * kThreads, row = p / kPieces, col = p % kPieces * 4;
            const f32x4v s = if4(row < n, v[i].take(col, width));
            const float f[4] = {s[0], s[1], s[2], s[3]};
            store_n<E, 4>(to + row * kStaged<E, DKP> + col, f);
        }
    }
}
// Planes of a staged matrix and of its transpose
template <class E, int DKP>
__device__ __forceinline__ void write_planes(const typename E::T* from, u16* rows, u16* columns)
{
    constexpr int LD = kStaged<E, DKP>;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    if (rows)
#pragma unroll 2
        for (int f = w; f < C * DKP / kFragment; f += kWaves) {
            const int at = (16 * (f / (DKP / 32)) + r) * LD + 32 * (f % (DKP / 32)) + 8 * g;
            u16* const to = rows + f * kFragment + 8 * lane;
            if constexpr (E::kBytes == 2) *(u32x4v*)to = *(const u32x4v*)(from + at);
            else store_split8<3>(at4(from + at), at4(from + at + 4), to, C * DKP);
        }
    if (columns)
#pragma unroll 2
        for (int f = w; f < C * DKP / kFragment; f += kWaves) {
            const typename E::T* const at = from + (32 * (f % 2) + 8 * g) * LD + 16 * (f / 2) + r;
            u16* const to = columns + f * kFragment + 8 * lane;
            typename E::T v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = at[i * LD];
            if constexpr (E::kBytes == 2)
                *(u32x4v*)to = (u32x4v){(uint32_t)v[0] | (uint32_t)v[1] << 16, (uint32_t)v[2] | (uint32_t)v[3] << 16, (uint32_t)v[4] | (uint32_t)v[5] << 16,
                                        (uint32_t)v[6] | (uint32_t)v[7] << 16};
            else store_split8<3>((f32x4v){v[0], v[1], v[2], v[3]}, (f32x4v){v[4], v[5], v[6], v[7]}, to, C * DKP);
        }
}
// Planes of a matrix of 64 by 64 in LDS, or of its transpose
template <int N, bool TRANSPOSED>
__device__ __forceinline__ void write_square(const float* from, u16* to)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int f = w; f < C * C / kFragment; f += kWaves) {
        const int row = 16 * (f / 2) + r, col = 32 * (f % 2) + 8 * g;
        u16* const out = to + f * kFragment + 8 * lane;
        if constexpr (TRANSPOSED) store_split8<N>(down4(from + col * kRow + row, kRow), down4(from + (col + 4) * kRow + row, kRow), out, C * C);
        else store_split8<N>(at4(from + row * kRow + col), at4(from + row * kRow + col + 4), out, C * C);
    }
}

// X, P, y and e of every block, and the planes of keys and queries.  X is built of blocks of 16: those on the diagonal by substitution, a
// column to a lane; then X_ij = -X_ii sum_k L_ik X_kj, those one off the diagonal first.
//
// Measured, one key head of 128 for two of 16 heads: 8 x 1024 steps bf16 54 us without and 62 with what the gradient needs, which is 148 and 214 MB written,
// 2.7 and 3.5 TB/s; 16 x 300 steps of 8 heads of 100 fp32 46 and 49 us, where the fp32 instruction's products and the chain of the inverse, four
// barriers long, bound it.
template <class E, int DKP, bool BACK, bool WHOLE>
__global__ __launch_bounds__(kThreads) void delta_prepare_kernel(DeltaArgs a)
{
    using T = typename E::T;
    extern __shared__ float lds[];
    __shared__ double Gs[C];
    __shared__ float betas[C];
    constexpr int LD = kStaged<E, DKP>;
    T *const Ks = (T*)lds, *const Qs = Ks + C * LD;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const Block k = block_of(a, (int)(id / a.heads / a.B), (int)(id / a.heads % a.B), (int)(id % a.heads));
    if (k.n <= 0) return;
    const Place<E, DKP, BACK> at(a);
    const int group = a.heads / a.key_heads, hk = k.h / group;
    stage<E, DKP, WHOLE>(row_of<E>(a.k, a.k_t, a.k_b, k.t0, k.b, (int64_t)hk * a.Dk), a.k_t, k.n, a.Dk, Ks);
    stage<E, DKP, WHOLE>(row_of<E>(a.q, a.q_t, a.q_b, k.t0, k.b, (int64_t)hk * a.Dk), a.q_t, k.n, a.Dk, Qs);
    if (w == 0) {
        const double G = running(a, k, lane);
        Gs[lane] = G;
        betas[lane] = beta_at(a, k, lane);
        at.y(k)[lane] = expf((float)G);
        at.e(k)[lane] = expf((float)(__shfl(G, 63) - G));
    }
    __syncthreads();
    if (k.h % group == 0) {
        write_planes<E, DKP>(Ks, at.K(k), at.KT(k));
        write_planes<E, DKP>(Qs, at.Q(k), BACK ? at.QT(k) : nullptr);
    }
    f32x4v kk[4], qk[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) kk[j] = qk[j] = kZero4;
    if constexpr (E::kBytes == 2) {
#pragma unroll
        for (int d = 0; d < DKP; d += 32) {
            const bf16x8 ka = *(const bf16x8*)(Ks + (16 * w + r) * LD + d + 8 * g), qa = *(const bf16x8*)(Qs + (16 * w + r) * LD + d + 8 * g);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j > w) continue;
                const bf16x8 kb = *(const bf16x8*)(Ks + (16 * j + r) * LD + d + 8 * g);
                kk[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, kb, kk[j], 0, 0, 0);
                qk[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qa, kb, qk[j], 0, 0, 0);
            }
        }
    } else {
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
    }
    __syncthreads();
    float *const Ls = lds, *const Xs = Ls + C * kRow, *const Ps = Xs + C * kRow;       // in place of what is not needed any more
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
            Ps[row * kRow + col] = p;
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
    if constexpr (BACK) write_square<3, true>(Ps, at.PT(k));
    else write_square<3, false>(Ps, at.P(k));
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
    write_square<3, false>(Xs, at.X(k));
    if constexpr (BACK) write_square<3, true>(Xs, at.XT(k));
}

// 16 columns of a state [Dk, Dv] as the accumulators of the workgroup hold them: wave w its rows 16 w DKP / 64 .., lane (r, g) four rows of
// column r of each tile of 16
template <int DKP>
struct StateTile {
    static constexpr int kParts = DKP / 64, LD = DKP + 8;
    f32x4v v[kParts];
    // of rows of `ld`, without a branch between the loads
    __device__ __forceinline__ void load(const float* from, int ld, const DeltaArgs& a, int w, int g, int col)
    {
#pragma unroll
        for (int m = 0; m < kParts; ++m) v[m] = kZero4;
        if (!from) return;
#pragma unroll
        for (int m = 0; m < kParts; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[m][i] = from[(int64_t)min(16 * (w * kParts + m) + 4 * g + i, a.Dk - 1) * ld + min(col, a.Dv - 1)];
#pragma unroll
        for (int m = 0; m < kParts; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[m][i] = col < a.Dv && 16 * (w * kParts + m) + 4 * g + i < a.Dk ? v[m][i] : 0.f;
    }
    __device__ __forceinline__ void store(float* to, const DeltaArgs& a, int w, int g, int col) const
    {
#pragma unroll
        for (int m = 0; m < kParts; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 16 * (w * kParts + m) + 4 * g + i;
                if (col < a.Dv && d < a.Dk) to[(int64_t)d * a.Dv + col] = v[m][i];
            }
    }
    // without a branch: what the tile has more than the state goes to `sink`
    __device__ __forceinline__ void store_all(float* to, int ld, float* sink, const DeltaArgs& a, int w, int g, int col) const
    {
#pragma unroll
        for (int m = 0; m < kParts; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 16 * (w * kParts + m) + 4 * g + i;
                float* const p = col < a.Dv && d < a.Dk ? to + d * ld + col : sink;
                *p = v[m][i];
            }
    }
    // planes of it in LDS, a row for each column
    __device__ __forceinline__ void publish(u16* to, int w, int r, int g) const
    {
#pragma unroll
        for (int m = 0; m < kParts; ++m) store_split<3>(v[m], to + r * LD + 16 * (w * kParts + m) + 4 * g, kTile * LD);
    }
};

// Four steps of one column in rows of [T, B], from `row` of a block on.  Steps behind the sequence's end, `rest` of the last block, stand for the last one,
// and are 0 when taken; no load has a branch, and nothing waits for one here.  KEPT: the rows' places are worked out once, in sixteen registers (8192
// steps on one tile to a workgroup 260 us, worked out each time 269, when reads and updates had two planes); without registers to spare each time.
template <bool KEPT>
struct FourRows {
    int row, rest;
    int64_t stride, whole[4], last[4];
    __device__ __forceinline__ FourRows(int row, int64_t stride, int rest) : row(row), rest(rest), stride(stride)
    {
        if constexpr (KEPT)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                whole[i] = (row + i) * stride;
                last[i] = min(row + i, rest - 1) * stride;
            }
    }
    __device__ __forceinline__ int64_t at(int i, bool is_last) const
    {
        if constexpr (KEPT) return is_last ? last[i] : whole[i];
        else return min(row + i, (is_last ? rest : C) + zero_here() - 1) * stride;
    }
};
template <class E>
struct FourSteps {
    typename E::T raw[4];
    template <bool KEPT>
    __device__ __forceinline__ void load(const typename E::T* from, const FourRows<KEPT>& rows, bool is_last)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = from[rows.at(i, is_last)];
    }
    __device__ __forceinline__ f32x4v take(int row, int n) const
    {
        f32x4v v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = row + i < n ? E::load(raw + i) : 0.f;
        return v;
    }
};

// Forward: the walk over the blocks of one sequence and head, NT tiles of 16 columns of S.  Keys, queries, X and P come from memory as the
// matrix instruction takes them, those of the next block while this one is worked on; S, R and U pass through LDS in planes.
//
// Bound: with few workgroups the chain S -> R -> U -> S of a block, three products with a barrier behind each, by one wave on a SIMD; what is
// not on it (Q S, P U, O and all loads) stands where the chain waits: Q S behind R's barrier, P U behind the next block's first.  With many, what
// a tile takes of keys and queries from the caches, which two tiles halve.
//
// Measured: 8192 steps of 16 heads of 128 x 128, bf16, 279 us, 2.2 us a block on 128 workgroups (on the fp32 instruction, without planes, 1564 with the
// preparation, 330 now; a sum for each order of planes, so that the products do not wait for each other, changed nothing); 8 x 1024 steps 132 us with the
// states kept, on two workgroups a compute unit (with two planes where there were two 127, and on one, when what could be read again or worked out again
// was kept in 290 registers, 146); 16 x 300 steps of 8 heads of 100 x 100, fp32, 68 us, one workgroup a compute unit.  The matrix units are 17 to 23 % busy.
template <class E, int DKP, int NT, bool STATES>
__global__ __launch_bounds__(kThreads, (DKP <= 128 && DKP / 64 * kPlanes<E> * NT <= 4 ? 2 : 1)) void delta_walk_kernel(DeltaArgs a, int tiles)
{
    using T = typename E::T;
    constexpr int kP = kPlanes<E>, LD = DKP + 8, kParts = DKP / 64, kK = DKP / 32, kS = kTile * kSteps;
    extern __shared__ u16 planes[];
    u16 *const Ss = planes, *const Rs = Ss + NT * 3 * kTile * LD, *const Us = Rs + NT * 3 * kS, *const Es = Us + NT * 3 * kS;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const int tile = (int)(id % tiles), h = (int)(id / tiles % a.heads), b = (int)(id / tiles / a.heads);
    const int col = tile * NT * kTile + r, row = 16 * w + 4 * g;        // the lane's first column and the first of its four steps
    const int len = length_of(a, b), blocks = (len + C - 1) / C;
    const int64_t state = ((int64_t)b * a.heads + h) * a.Dk * a.Dv, states_step = (int64_t)a.B * a.heads * a.Dk * a.Dv;
    const Place<E, DKP, false> at(a);
    StateTile<DKP> S[NT];
#pragma unroll
    for (int q = 0; q < NT; ++q) S[q].load(a.S0 ? a.S0 + state : nullptr, a.Dv, a, w, g, col + q * kTile);
    if (blocks > 0) {
        // addresses: the same for all lanes, and a lane's own 32 bits
        const Block first = {0, b, h, 0, 0, (int64_t)b * a.heads + h};
        const int64_t keys_step = (int64_t)a.B * a.key_heads * at.kKeys, head_step = (int64_t)a.B * a.heads * at.kHead;
        const u16 *K0 = at.K(first) + fragment_at(w, kK, 0), *Q0 = at.Q(first) + fragment_at(w, kK, 0), *KT0 = at.KT(first) + fragment_at(w * kParts, 2, 0),
                  *X0 = at.X(first) + fragment_at(w, 2, 0), *P0 = at.P(first) + fragment_at(w, 2, 0);
        const float* y0 = at.y(first);
        const unsigned mine = 8 * lane;
        const float* beta0 = row_of<F32>(a.beta, a.beta_t, a.beta_b, 0, b, h);
        const T* v0 = row_of<E>(a.v, a.v_t, a.v_b, 0, b, (int64_t)h * a.Dv);
        T* const o0 = (T*)row_of<E>(a.o, a.o_t, a.o_b, 0, b, (int64_t)h * a.Dv);
        float* const sink = at.sink() + lane;
        bf16x8 K[kK][kP], Q[kK][kP], X[2][3], KT[kParts][2][kP], P[2][3];
        f32x4v y, e, O[NT];
        FourSteps<E> v[NT];
        FourSteps<F32> beta;
        float last;
        const int rest = len - (blocks - 1) * C;        // steps of the last block
        const FourRows<kRoom<E, DKP, NT>> v_rows(row, a.v_t, rest), beta_rows(row, a.beta_t, rest);
        const auto load_keys = [&](int c) {
#pragma unroll
            for (int s = 0; s < kK; ++s) fragment<kP>(K[s], K0 + fragment_at(0, kK, s) + mine, C * DKP);
#pragma unroll
            for (int q = 0; q < NT; ++q) v[q].load(v0 + min(col + q * kTile, a.Dv - 1), v_rows, c == blocks - 1);
            beta.load(beta0, beta_rows, c == blocks - 1);
        };
        const auto load_queries = [&]() {
#pragma unroll
            for (int s = 0; s < kK; ++s) fragment<kP>(Q[s], Q0 + fragment_at(0, kK, s) + mine, C * DKP);
            y = at4(y0 + row);
            e = at4(y0 + C + row);
            last = y0[C - 1];
        };
        const auto load_inverse = [&]() {
#pragma unroll
            for (int s = 0; s < 2; ++s) fragment<3>(X[s], X0 + fragment_at(0, 2, s) + mine, C * C);
        };
        const auto load_columns = [&]() {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int m = 0; m < kParts; ++m) fragment<kP>(KT[m][s], KT0 + fragment_at(m, 2, s) + mine, C * DKP);
        };
        const auto load_pairs = [&]() {
#pragma unroll
            for (int s = 0; s < 2; ++s) fragment<3>(P[s], P0 + fragment_at(0, 2, s) + mine, C * C);
        };
        // O of a block whose U is in LDS
        const auto finish = [&](int c) {
            const int n = len - c * C, late = row + (kRoom<E, DKP, NT> ? 0 : zero_here());
            T* const to = o0 + (int64_t)c * C * a.o_t;
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                Sum pu;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    bf16x8 uf[3];
                    fragment<3>(uf, Us + q * 3 * kS + r * kSteps + 32 * s + 8 * g, kS);
                    multiply(pu, P[s], uf);
                }
                O[q] += pu.total();
                const int at_col = col + q * kTile;
#pragma unroll
                for (int i = 0; i < 4; ++i) E::store(at_col < a.Dv && c >= 0 && row + i < n ? to + (late + i) * a.o_t + at_col : (T*)sink, O[q][i]);
            }
        };
        load_keys(0);
        load_queries();
        load_inverse();
        load_columns();
        load_pairs();
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            O[q] = kZero4;
            S[q].publish(Ss + q * 3 * kTile * LD, w, r, g);
        }
        // No branch in here: where one followed a matrix instruction the compiler has left out the wait in front of its result (two of the
        // eight instructions that lie between them elsewhere), and half of a result was what stood there before.
#pragma unroll 1
        for (int c = 0; c < blocks; ++c) {
            if constexpr (STATES)
#pragma unroll
                for (int q = 0; q < NT; ++q) S[q].store_all(a.states + c * states_step + state, a.Dv, sink, a, w, g, col + q * kTile);
            lds_barrier();
            const int n = len - c * C;
            const bool more = c + 1 < blocks;
            Sum qs[NT];
            const f32x4v b4 = beta.take(row, n), decay = e, y4 = y;
            const float decayed = last;
            bf16x8 f[kK][3];
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                Sum ks;
#pragma unroll
                for (int s = 0; s < kK; ++s) fragment<3>(f[s], Ss + q * 3 * kTile * LD + r * LD + 32 * s + 8 * g, kTile * LD);
#pragma unroll
                for (int s = 0; s < kK; ++s) multiply(ks, K[s], f[s]);
                const f32x4v v4 = v[q].take(row, n), found = ks.total();
                f32x4v R;
#pragma unroll
                for (int i = 0; i < 4; ++i) R[i] = b4[i] * (v4[i] - y4[i] * found[i]);
                store_split<3>(R, Rs + q * 3 * kS + r * kSteps + row, kS);
            }
            finish(c - 1);                      // in front of the first block of nothing, to nowhere
            lds_barrier();
            // of the next block what this one has done with, each as soon as that is so
            K0 += more ? keys_step : 0;
            v0 += more ? C * a.v_t : 0;
            beta0 += more ? C * a.beta_t : 0;
            load_keys(more ? c + 1 : c);
            load_pairs();                       // of this block: taken behind the next one's first barrier
            P0 += more ? head_step : 0;
            f32x4v U[NT];
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                Sum u;
                bf16x8 rf[2][3];
#pragma unroll
                for (int s = 0; s < 2; ++s) fragment<3>(rf[s], Rs + q * 3 * kS + r * kSteps + 32 * s + 8 * g, kS);
#pragma unroll
                for (int s = 0; s < kK; ++s) {
                    // without room S once more: of two tiles it would take a hundred registers from the first product to here
                    if constexpr (!kRoom<E, DKP, NT>) fragment<3>(f[s], Ss + q * 3 * kTile * LD + r * LD + 32 * s + 8 * g, kTile * LD);
                    multiply(qs[q], Q[s], f[s]);
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) multiply(u, X[s], rf[s]);
                U[q] = u.total();
                store_split<3>(times4(U[q], decay), Es + q * 3 * kS + r * kSteps + row, kS);
                O[q] = times4(qs[q].total(), scaled4(y4, a.scale));
            }
            lds_barrier();
            Q0 += more ? keys_step : 0;
            X0 += more ? head_step : 0;
            y0 += more ? head_step / 2 : 0;
            load_queries();
            load_inverse();
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                bf16x8 ef[2][3];
#pragma unroll
                for (int s = 0; s < 2; ++s) fragment<3>(ef[s], Es + q * 3 * kS + r * kSteps + 32 * s + 8 * g, kS);
                store_split<3>(U[q], Us + q * 3 * kS + r * kSteps + row, kS);
#pragma unroll
                for (int m = 0; m < kParts; ++m) {
                    Sum sum;
#pragma unroll
                    for (int s = 0; s < 2; ++s) multiply(sum, KT[m][s], ef[s]);
                    S[q].v[m] = scaled4(S[q].v[m], decayed) + sum.total();
                }
                S[q].publish(Ss + q * 3 * kTile * LD, w, r, g);
            }
            KT0 += more ? keys_step : 0;
            load_columns();
        }
        lds_barrier();
        finish(blocks - 1);
    }
#pragma unroll
    for (int q = 0; q < NT; ++q) {
        const int at_col = col + q * kTile;
        if (a.ST) S[q].store(a.ST + state, a, w, g, at_col);
        for (int64_t t = len + (threadIdx.x >> 4); t < a.T; t += 4 * kWaves)
            if (at_col < a.Dv) E::store((T*)row_of<E>(a.o, a.o_t, a.o_b, t, b, (int64_t)h * a.Dv + at_col), 0.f);
    }
}

// Few steps: a thread holds four columns of every 32nd row of S, eight threads 32 columns of a row; the sums over the rows of
// what key and query find meet in LDS once a step, and
//     u = b (v - a S'k)     o = scale (a S'q + (q.k) u)     S <- a S + k u'
//
// A single step is bound by moving the state once each way: 64 sequences of 16 heads of 128 x 128 34 us for 135 MB, 3.9 TB/s; one sequence of 12 heads of
// 125 x 125 6.1 us, a launch and three trips to memory one after the other.
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

// Gradient: the walk back over the blocks, NT tiles of 16 columns of dS.  Its chain is dS' -> dU -> dR -> dS; Q' (y dO) stands where dR is
// waited for.  Measured: 8 x 1024 steps of 16 heads of 128 x 128, bf16, 166 us, two workgroups a compute unit (197 with one, whose 355 registers held
// results until the block's end; they leave now as soon as they are there), 305 MB written (dS', dR and e K dS' in fp32, dv); 16 x 300 steps of 8 heads of 100 x 100,
// fp32, 68 us, one workgroup a compute unit.  The matrix units are 16 % busy.
template <class E, int DKP, int NT>
__global__ __launch_bounds__(kThreads, (DKP <= 128 && DKP / 64 * kPlanes<E> * NT <= 4 ? 2 : 1)) void delta_walk_back_kernel(DeltaArgs a, int tiles)
{
    using T = typename E::T;
    constexpr int kP = kPlanes<E>, LD = DKP + 8, kParts = DKP / 64, kK = DKP / 32, kS = kTile * kSteps;
    extern __shared__ u16 planes[];
    u16 *const Ds = planes, *const Os = Ds + NT * 3 * kTile * LD, *const Us = Os + NT * kP * kS, *const Ys = Us + NT * 3 * kS, *const Zs = Ys + NT * 3 * kS;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const int tile = (int)(id % tiles), h = (int)(id / tiles % a.heads), b = (int)(id / tiles / a.heads);
    const int col = tile * NT * kTile + r, row = 16 * w + 4 * g;
    const int len = length_of(a, b), blocks = (len + C - 1) / C;
    const int64_t state = ((int64_t)b * a.heads + h) * a.Dk * a.Dv;
    const Place<E, DKP, true> at(a);
    StateTile<DKP> dS[NT];
#pragma unroll
    for (int q = 0; q < NT; ++q) dS[q].load(a.dST ? a.dST + state : nullptr, a.Dv, a, w, g, col + q * kTile);
    if (blocks > 0) {
        const Block behind = {blocks - 1, b, h, 0, 0, ((int64_t)(blocks - 1) * a.B + b) * a.heads + h};
        const int64_t keys_step = (int64_t)a.B * a.key_heads * at.kKeys, head_step = (int64_t)a.B * a.heads * at.kHead;
        const u16 *K0 = at.K(behind) + fragment_at(w, kK, 0), *KT0 = at.KT(behind) + fragment_at(w * kParts, 2, 0), *QT0 = at.QT(behind) + fragment_at(w * kParts, 2, 0),
                  *XT0 = at.XT(behind) + fragment_at(w, 2, 0), *PT0 = at.PT(behind) + fragment_at(w, 2, 0);
        const float* y0 = at.y(behind);
        const unsigned mine = 8 * lane;
        const float* beta0 = row_of<F32>(a.beta, a.beta_t, a.beta_b, (int64_t)behind.c * C, b, h);
        const T* dO0 = row_of<E>(a.dO, a.do_t, a.do_b, (int64_t)behind.c * C, b, (int64_t)h * a.Dv);
        T* const dv0 = (T*)row_of<E>(a.dv, a.dv_t, a.dv_b, 0, b, (int64_t)h * a.Dv);
        float* const sink = at.sink() + lane;
        const int ld = at.row();
        bf16x8 K[kK][kP], PT[2][3], XT[2][3], KT[kParts][2][kP], QT[kParts][2][kP];
        f32x4v y, e, dO[NT], b4;
        FourSteps<E> raw[NT];
        FourSteps<F32> beta;
        float last;
        const int rest = len - behind.c * C;
        const auto load_gates = [&]() {
            y = at4(y0 + row);
            e = at4(y0 + C + row);
            last = y0[C - 1];
        };
        const auto load_keys = [&]() {
#pragma unroll
            for (int s = 0; s < kK; ++s) fragment<kP>(K[s], K0 + fragment_at(0, kK, s) + mine, C * DKP);
        };
        const FourRows<kRoom<E, DKP, NT>> dO_rows(row, a.do_t, rest), beta_rows(row, a.beta_t, rest);
        const auto load_pairs = [&](bool is_last) {
#pragma unroll
            for (int s = 0; s < 2; ++s) fragment<3>(PT[s], PT0 + fragment_at(0, 2, s) + mine, C * C);
#pragma unroll
            for (int q = 0; q < NT; ++q) raw[q].load(dO0 + min(col + q * kTile, a.Dv - 1), dO_rows, is_last);
            beta.load(beta0, beta_rows, is_last);
        };
        const auto load_inverse = [&]() {
#pragma unroll
            for (int s = 0; s < 2; ++s) fragment<3>(XT[s], XT0 + fragment_at(0, 2, s) + mine, C * C);
        };
        const auto load_columns = [&](bf16x8(&to)[kParts][2][kP], const u16* from) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int m = 0; m < kParts; ++m) fragment<kP>(to[m][s], from + fragment_at(m, 2, s) + mine, C * DKP);
        };
        const auto take_pairs = [&](int n) {    // of the block that comes next; its dO in LDS
            b4 = beta.take(row, n);
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                dO[q] = raw[q].take(row, n);
                store_split<kP>(dO[q], Os + q * kP * kS + r * kSteps + row, kS);
            }
        };
        load_pairs(true);
        load_gates();
        load_keys();
        load_inverse();
        load_columns(QT, QT0);
        load_columns(KT, KT0);
        take_pairs(rest);
#pragma unroll
        for (int q = 0; q < NT; ++q) dS[q].publish(Ds + q * 3 * kTile * LD, w, r, g);
        // no branch in here, as in the walk forward
#pragma unroll 1
        for (int c = blocks - 1; c >= 0; --c) {
            const int n = len - c * C;
            Block k = behind;
            k.index = ((int64_t)c * a.B + b) * a.heads + h;
#pragma unroll
            for (int q = 0; q < NT; ++q) dS[q].store_all(at.dS(k), ld, sink, a, w, g, col + q * kTile);
            const f32x4v beta4 = b4;
            const bool more = c > 0;
            lds_barrier();
            f32x4v yb;
            const float decayed = last;
#pragma unroll
            for (int i = 0; i < 4; ++i) yb[i] = -y[i] * beta4[i];
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                bf16x8 f[kK][3];
                Sum kd, po;
#pragma unroll
                for (int s = 0; s < kK; ++s) fragment<3>(f[s], Ds + q * 3 * kTile * LD + r * LD + 32 * s + 8 * g, kTile * LD);
#pragma unroll
                for (int s = 0; s < kK; ++s) multiply(kd, K[s], f[s]);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    bf16x8 o[kP];
                    fragment<kP>(o, Os + q * kP * kS + r * kSteps + 32 * s + 8 * g, kS);
                    multiply(po, PT[s], o);
                }
                const f32x4v found = times4(kd.total(), e);
                store_split<3>(found + po.total(), Us + q * 3 * kS + r * kSteps + row, kS);
                // the workspace's rows hold a whole number of two tiles
                float* const f0 = at.found(k) + (row + zero_here()) * ld + col + q * kTile;
#pragma unroll
                for (int i = 0; i < 4; ++i) f0[i * ld] = found[i];
                store_split<3>(times4(scaled4(y, a.scale), dO[q]), Ys + q * 3 * kS + r * kSteps + row, kS);
            }
            lds_barrier();
            K0 -= more ? keys_step : 0;
            PT0 -= more ? head_step : 0;
            XT0 -= more ? head_step : 0;
            y0 -= more ? head_step / 2 : 0;
            dO0 -= more ? C * a.do_t : 0;
            beta0 -= more ? C * a.beta_t : 0;
            load_pairs(!more && blocks == 1);   // all blocks but the last are whole
            load_gates();
            load_keys();
            Sum sums[NT][kParts];
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                if (q > 0) one_by_one();
                Sum dr;
                bf16x8 uf[2][3], yf[2][3];
#pragma unroll
                for (int s = 0; s < 2; ++s) fragment<3>(uf[s], Us + q * 3 * kS + r * kSteps + 32 * s + 8 * g, kS);
#pragma unroll
                for (int s = 0; s < 2; ++s) fragment<3>(yf[s], Ys + q * 3 * kS + r * kSteps + 32 * s + 8 * g, kS);
#pragma unroll
                for (int s = 0; s < 2; ++s) multiply(dr, XT[s], uf[s]);
#pragma unroll
                for (int m = 0; m < kParts; ++m)
#pragma unroll
                    for (int s = 0; s < 2; ++s) multiply(sums[q][m], QT[m][s], yf[s]);
                const f32x4v dR = dr.total();
                store_split<3>(times4(yb, dR), Zs + q * 3 * kS + r * kSteps + row, kS);
                const int at_col = col + q * kTile, late = row + zero_here();
                float* const left = at.dR(k) + late * ld + at_col;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    left[i * ld] = dR[i];
                    E::store(at_col < a.Dv && row + i < n ? dv0 + (int64_t)c * C * a.dv_t + (late + i) * a.dv_t + at_col : (T*)sink, beta4[i] * dR[i]);
                }
            }
            QT0 -= more ? keys_step : 0;
            load_columns(QT, QT0);
            load_inverse();
            lds_barrier();
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                bf16x8 zf[2][3];
#pragma unroll
                for (int s = 0; s < 2; ++s) fragment<3>(zf[s], Zs + q * 3 * kS + r * kSteps + 32 * s + 8 * g, kS);
#pragma unroll
                for (int m = 0; m < kParts; ++m) {
#pragma unroll
                    for (int s = 0; s < 2; ++s) multiply(sums[q][m], KT[m][s], zf[s]);
                    dS[q].v[m] = scaled4(dS[q].v[m], decayed) + sums[q][m].total();
                }
                dS[q].publish(Ds + q * 3 * kTile * LD, w, r, g);
            }
            KT0 -= more ? keys_step : 0;
            load_columns(KT, KT0);
            take_pairs(C);
        }
    }
#pragma unroll
    for (int q = 0; q < NT; ++q) {
        const int at_col = col + q * kTile;
        if (a.dS0) dS[q].store(a.dS0 + state, a, w, g, at_col);
        for (int64_t t = len + (threadIdx.x >> 4); t < a.T; t += 4 * kWaves)
            if (at_col < a.Dv) E::store((T*)row_of<E>(a.dv, a.dv_t, a.dv_b, t, b, (int64_t)h * a.Dv + at_col), 0.f);
    }
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

// U of every block again, from the state in front of it, 16 columns to a workgroup, and the columns' part of what sums over a
// step's columns: dR.(v - y K S), -y b dR.(K S), U.(e K dS'); and of S.dS'.  One tile to a workgroup, several workgroups to a compute unit: each is loads, two
// products and a sum one after the other, and the others fill its waits.  (Eight tiles one after the other, K and X kept and the next tile on its way,
// took registers for the addresses and halved the workgroups: 163 us against 164.)  Measured: 8 x 1024 steps of 16 heads of 128 x 128, bf16, 164 us for 325 MB from and
// to memory, 2.0 TB/s; 16 x 300 steps of 8 heads of 100 x 100, fp32, 42 us.
template <class E, int DKP>
__global__ __launch_bounds__(kThreads) void delta_update_kernel(DeltaArgs a, int tiles)
{
    constexpr int kP = kPlanes<E>, LD = DKP + 8, kK = DKP / 32;
    __shared__ u16 Ss[3 * kTile * LD], Rs[3 * kTile * kSteps];
    __shared__ float dots[kWaves];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const int tile = (int)(id % tiles), h = (int)(id / tiles % a.heads), b = (int)(id / tiles / a.heads % a.B), c = (int)(id / tiles / a.heads / a.B);
    const int col = tile * kTile + r, row = 16 * w + 4 * g;
    const bool live = col < a.Dv;
    const Block k = block_of(a, c, b, h);
    if (k.n <= 0) return;
    const Place<E, DKP, true> at(a);
    StateTile<DKP> S, dS;
    const int ld = at.row();
    const FourRows<false> v_rows(row, a.v_t, k.n), beta_rows(row, a.beta_t, k.n);
    FourSteps<E> raw;
    FourSteps<F32> raw_beta;
    S.load(a.states + k.index * a.Dk * a.Dv, a.Dv, a, w, g, col);
    dS.load(at.dS(k), ld, a, w, g, col);
    raw.load(row_of<E>(a.v, a.v_t, a.v_b, k.t0, b, (int64_t)h * a.Dv + min(col, a.Dv - 1)), v_rows, true);
    raw_beta.load(row_of<F32>(a.beta, a.beta_t, a.beta_b, k.t0, b, h), beta_rows, true);
    float dot = 0.f, dR[4], found[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        dR[i] = at.dR(k)[(row + i) * ld + col];
        found[i] = at.found(k)[(row + i) * ld + col];
    }
    bf16x8 K[kK][kP], X[2][3];
#pragma unroll
    for (int s = 0; s < kK; ++s) fragment<kP>(K[s], at.K(k) + fragment_at(w, kK, s) + 8 * lane, C * DKP);
#pragma unroll
    for (int s = 0; s < 2; ++s) fragment<3>(X[s], at.X(k) + fragment_at(w, 2, s) + 8 * lane, C * C);
    const f32x4v y = at4(at.y(k) + row);
    S.publish(Ss, w, r, g);
#pragma unroll
    for (int m = 0; m < DKP / 64; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) dot = fmaf(S.v[m][i], dS.v[m][i], dot);
    const f32x4v v = raw.take(row, k.n), beta = raw_beta.take(row, k.n);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        dR[i] = live ? dR[i] : 0.f;
        found[i] = live ? found[i] : 0.f;
    }
    lds_barrier();
    Sums ks;
#pragma unroll
    for (int s = 0; s < kK; ++s) {
        bf16x8 f[3];
        fragment<3>(f, Ss + r * LD + 32 * s + 8 * g, kTile * LD);
        multiply(ks, K[s], f);
    }
    const f32x4v read = ks.total();
    f32x4v R;
    float db[4], from_front[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float miss = v[i] - y[i] * read[i];
        R[i] = beta[i] * miss;
        db[i] = dR[i] * miss;
        from_front[i] = -y[i] * beta[i] * dR[i] * read[i];
    }
    store_split<3>(R, Rs + r * kSteps + row, kTile * kSteps);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) dot += __shfl_xor(dot, off);
    if (lane == 0) dots[w] = dot;
    lds_barrier();
    Sums u;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        bf16x8 f[3];
        fragment<3>(f, Rs + r * kSteps + 32 * s + 8 * g, kTile * kSteps);
        multiply(u, X[s], f);
    }
    const f32x4v U = u.total();
    float* const parts = at.parts(k, tile);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        at.U(k)[(row + i) * ld + col] = U[i];
        const float d = row16_sum(db[i]), f = row16_sum(from_front[i]), l = row16_sum(U[i] * found[i]);
        if (r == 0) {
            parts[row + i] = d;
            parts[C + row + i] = f;
            parts[2 * C + row + i] = l;
        }
    }
    if (threadIdx.x == 0) parts[3 * C] = dots[0] + dots[1] + dots[2] + dots[3];
}

// What is left of a block's gradient, from the state S in front of it, dS' behind it, dR and U:
//
//     dP = D (scale dO U')     dA = -b D (dR U') below the diagonal      dq = scale y dO S' + dP K
//     dk = e U dS'' - y b dR S' + dP' Q + (dA + dA') K                   db = dR.(v - y K S) - sum_j dR.U_j D k.k_j
//     dg_t = sum_{i >= t > j} (dA_ij k_i.k_j + dP_ij q_i.k_j) + sum_{i >= t} (q.(scale y dO S') - y b dR.(K S))_i
//            + sum_{j < t} U.(e K dS')_j + exp(G_last) S.dS'
//
// (each decay's own terms; as differences of what reaches two neighbouring G, what a strong decay leaves of dg would be lost).
// A workgroup of eight waves takes a block of one sequence and key head and goes through the heads that share it, 32 columns of S at a time,
// whose planes its threads make together while the next ones are on their way.  Waves w and w + 4 hold the results of the same 16 steps, each
// for half of a tile's key columns; of the pairs of steps the first makes dP, the second dA.
//
// One workgroup has a compute unit, its results 128 registers of each lane: what bounds it is that nobody works while it waits, at the tiles' barriers and
// in the end of a block, which is a third of it.  Measured: 8 x 1024 steps of 16 heads of 128 x 128, bf16, 262 us for 470 MB, matrix units 18 % busy; 16 x 300
// steps of 8 heads of 100 x 100, fp32, 150 us, 16 %.
constexpr int kGradientWaves = 8, kGradientThreads = 64 * kGradientWaves;
constexpr int kWide = 32, kWideRow = kWide + 8;         // columns of a tile, and its row in LDS
constexpr int kRowsAtOnce = 128;                        // of S and dS' in LDS
template <class E, int DKP, bool WHOLE>
__global__ __launch_bounds__(kGradientThreads, 2) void delta_gradient_kernel(DeltaArgs a)
{
    using T = typename E::T;
    extern __shared__ float lds[];
    constexpr int kP = kPlanes<E>, kRows = DKP < kRowsAtOnce ? DKP : kRowsAtOnce, kTurns = DKP / kRows;
    constexpr int kParts = DKP / 32, kEach = kRows / 32;        // tiles of 16 key columns of a wave, those of a turn
    constexpr int kLoads = kRows * kWide / 4 / kGradientThreads;
    // S, dS' and U of a tile of columns, three planes each; in their place later dP and dA
    u16 *const Ss = (u16*)lds, *const Ds = Ss + 3 * kRows * kWideRow, *const Us = Ds + 3 * kRows * kWideRow;
    float *const Ps = lds, *const As = Ps + C * kRow;
    __shared__ double Gs[C];
    __shared__ float ys[C], es[C], betas[C], overs[kGradientWaves][C], fronts[2][C], backs[C], dbs[2][C];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3, half = wave >> 2, r = lane & 15, g = lane >> 4;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x);
    const int c = (int)(id / a.key_heads / a.B), b = (int)(id / a.key_heads % a.B), hk = (int)(id % a.key_heads), group = a.heads / a.key_heads;
    const int64_t t0 = (int64_t)c * C;
    const int n = (int)min((int64_t)length_of(a, b) - t0, (int64_t)C), rows = (int)min((int64_t)a.T - t0, (int64_t)C);
    if (n <= 0) {       // behind the sequence's end
        for (int p = threadIdx.x; p < rows * a.Dk; p += kGradientThreads) {
            E::store((T*)row_of<E>(a.dq, a.dq_t, a.dq_b, t0 + p / a.Dk, b, (int64_t)hk * a.Dk + p % a.Dk), 0.f);
            E::store((T*)row_of<E>(a.dk, a.dk_t, a.dk_b, t0 + p / a.Dk, b, (int64_t)hk * a.Dk + p % a.Dk), 0.f);
        }
        for (int p = threadIdx.x; p < rows * group; p += kGradientThreads) {
            if (a.dg) *(float*)row_of<F32>(a.dg, a.dg_t, a.dg_b, t0 + p / group, b, hk * group + p % group) = 0.f;
            *(float*)row_of<F32>(a.dbeta, a.dbeta_t, a.dbeta_b, t0 + p / group, b, hk * group + p % group) = 0.f;
        }
        return;
    }
    const int row = 16 * w + 4 * g, mine = 16 * w + r;          // the lane's steps as results, and its step as first operand
    const Place<E, DKP, true> at(a);
    const int ld = at.row(), wides = (a.Dv + kWide - 1) / kWide;
    // tile m of the wave in turn d0 stands for the key columns from here on
    const auto key_column = [&](int turn, int m) { return turn * kRows + 16 * (half * kEach + m); };
    for (int hh = 0; hh < group; ++hh) {
        const Block k = block_of(a, c, b, hk * group + hh);
        const float *const behind = at.dS(k), *const left = at.dR(k), *const updates = at.U(k), *const front = a.states + k.index * a.Dk * a.Dv;
        const T* const o_row = row_of<E>(a.dO, a.do_t, a.do_b, t0 + min(mine, n - 1), b, (int64_t)k.h * a.Dv);
        if (wave == 0) {
            Gs[lane] = running(a, k, lane);
            ys[lane] = at.y(k)[lane];
            es[lane] = at.e(k)[lane];
            betas[lane] = beta_at(a, k, lane);
        }
        Sum dq[kParts], from_dS[kParts], from_dR[kParts], pairs[4];     // pairs: dO U' or dR U'
        Four<F32, WHOLE> s4[kLoads];
        Four<E, WHOLE> o4[2];
        f32x4v ds4[kLoads], u4, l4[2];
        const auto fetch_states = [&](int turn) {
            const int c0 = turn / kTurns * kWide, d0 = turn % kTurns * kRows;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int p = threadIdx.x + i * kGradientThreads, d = min(d0 + p / (kWide / 4), a.Dk - 1), from = c0 + p % (kWide / 4) * 4;
                s4[i].load(front + (int64_t)d * a.Dv, from, a.Dv);
                ds4[i] = at4(behind + d * ld + from);
            }
        };
        const auto fetch_rows = [&](int wide) {
            const int c8 = wide * kWide + 8 * g;
            o4[0].load(o_row, c8, a.Dv);
            o4[1].load(o_row, c8 + 4, a.Dv);
            l4[0] = at4(left + mine * ld + c8);
            l4[1] = at4(left + mine * ld + c8 + 4);
            u4 = at4(updates + threadIdx.x / (kWide / 4) * ld + wide * kWide + threadIdx.x % (kWide / 4) * 4);
        };
        static_assert(C * kWide / 4 == kGradientThreads, "");
        fetch_states(0);
        fetch_rows(0);
        for (int wide = 0; wide < wides; ++wide) {
            bf16x8 dO[kP], dR[3], U[3];
#pragma unroll
            for (int turn = 0; turn < kTurns; ++turn) {
                lds_barrier();
                if (turn == 0) {
                    const int c8 = wide * kWide + 8 * g, cu = wide * kWide + threadIdx.x % (kWide / 4) * 4;
                    split8<kP>(if4(mine < n, o4[0].take(c8, a.Dv)), if4(mine < n, o4[1].take(c8 + 4, a.Dv)), dO);
                    split8<3>(within4(l4[0], c8, a.Dv), within4(l4[1], c8 + 4, a.Dv), dR);
                    store_split<3>(within4(u4, cu, a.Dv), Us + threadIdx.x / (kWide / 4) * kWideRow + threadIdx.x % (kWide / 4) * 4, C * kWideRow);
                }
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int p = threadIdx.x + i * kGradientThreads, d = p / (kWide / 4), from = p % (kWide / 4) * 4;
                    const bool there = turn * kRows + d < a.Dk;
                    store_split<3>(if4(there, s4[i].take(wide * kWide + from, a.Dv)), Ss + d * kWideRow + from, kRows * kWideRow);
                    store_split<3>(if4(there, within4(ds4[i], wide * kWide + from, a.Dv)), Ds + d * kWideRow + from, kRows * kWideRow);
                }
                fetch_states(min(wide * kTurns + turn + 1, wides * kTurns - 1));
                if (turn == 0) fetch_rows(min(wide + 1, wides - 1));
                lds_barrier();
                if (turn == 0) {
                    fragment<3>(U, Us + mine * kWideRow + 8 * g, C * kWideRow);
                    const auto multiply_pairs = [&](const auto& first) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            bf16x8 u[3];
                            fragment<3>(u, Us + (16 * j + r) * kWideRow + 8 * g, C * kWideRow);
                            multiply(pairs[j], first, u);
                        }
                    };
                    if (half == 0) multiply_pairs(dO);
                    else multiply_pairs(dR);
                }
#pragma unroll
                for (int m = 0; m < kEach; ++m) {
                    bf16x8 s[3], ds[3];
                    const int at_row = (16 * (half * kEach + m) + r) * kWideRow + 8 * g;
                    fragment<3>(s, Ss + at_row, kRows * kWideRow);
                    fragment<3>(ds, Ds + at_row, kRows * kWideRow);
                    multiply(dq[turn * kEach + m], dO, s);
                    multiply(from_dR[turn * kEach + m], dR, s);
                    multiply(from_dS[turn * kEach + m], U, ds);
                }
            }
        }
        __syncthreads();
        f32x4v dq_sum[kParts], dk_sum[kParts], y, beta;
        float from_front[4], db[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = ys[row + i];
            beta[i] = betas[row + i];
            from_front[i] = db[i] = 0.f;
        }
        // what the tiles of columns have added: lane 16 g + i of the first wave the tiles i, i + 16, .. of its four steps
        float to_back[4] = {}, dot = 0.f;
        if (half == 0)
            for (int tile = r; tile < at.tiles(); tile += 16) {
                const float* const parts = at.parts(k, tile);
                const f32x4v d4 = at4(parts + row), f4 = at4(parts + C + row), l4 = at4(parts + 2 * C + row);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    db[i] += d4[i];
                    from_front[i] += f4[i];
                    to_back[i] += l4[i];
                }
                dot += parts[3 * C];
            }
        const int late = zero_here();
        const u16 *const Q = at.Q(k) + late, *const K = at.K(k) + late;
#pragma unroll
        for (int m = 0; m < kParts; ++m) {
            if (kP > 1 || m % 2 == 0) one_by_one();
            const f32x4v q4 = dq[m].total(), s4 = from_dS[m].total(), r4 = from_dR[m].total();
            const int d = key_column(m / kEach, m % kEach) + r + late;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float q = 0.f;
#pragma unroll
                for (int p = kP - 1; p >= 0; --p)
                    q += __uint_as_float((uint32_t)Q[p * C * DKP + fragment_at(w, DKP / 32, d / 32) + 8 * (4 * g + i + d % 32 / 8 * 16) + d % 8] << 16);
                dq_sum[m][i] = a.scale * y[i] * q4[i];
                dk_sum[m][i] = es[row + i] * s4[i] - y[i] * beta[i] * r4[i];
                from_front[i] = fmaf(q, dq_sum[m][i], from_front[i]);
            }
        }
        // q.k for the first wave, k.k for the second
        Sum dots[4];
        const u16* const own = half == 0 ? Q : K;
#pragma unroll
        for (int s = 0; s < DKP / 32; ++s) {
            if (kP > 1 || s % 4 == 0) one_by_one();
            bf16x8 fa[kP];
            fragment<kP>(fa, own + fragment_at(w, DKP / 32, s) + 8 * lane, C * DKP);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8 fb[kP];
                fragment<kP>(fb, K + fragment_at(j, DKP / 32, s) + 8 * lane, C * DKP);
                multiply(dots[j], fa, fb);
            }
        }
        // dP is scale D (dO U'); dA is -b D (dR U'), and D (dR U') k.k is taken from db
        float by[4];
        double G4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            by[i] = half == 0 ? a.scale : -beta[i];
            G4[i] = Gs[row + i];
        }
        const float of_beta = half == 0 ? 0.f : -1.f;
        float in_front[4] = {};     // pairs of the lane's steps with all steps of the tiles in front of this one
        float* const square = half == 0 ? Ps : As;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4v dots4 = dots[j].total(), pairs4 = pairs[j].total();
            const double G = Gs[16 * j + r];
            float over = 0.f;       // pairs that the decay at step 16 j + r lies between, of the lane's steps
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int step = row + i, other = 16 * j + r;
                const bool there = other <= step - half && step < n;        // the first wave has the diagonal too
                const float decayed = there ? expf((float)(G4[i] - G)) * pairs4[i] : 0.f, v = decayed * by[i];
                db[i] = fmaf(of_beta * decayed, dots4[i], db[i]);
                const float pair = other < step ? v * dots4[i] : 0.f;
                square[step * kRow + other] = v;
                // over the steps in front of 16 j + r: the 16 of the tile by shifts along the row of lanes
                float sum = row16_shifted<1>(pair);
                sum += row16_shifted<1>(sum);
                sum += row16_shifted<2>(sum);
                sum += row16_shifted<4>(sum);
                sum += row16_shifted<8>(sum);
                if (other <= step) over += in_front[i] + sum;
                in_front[i] += row16_sum(pair);
            }
            over += __shfl_xor(over, 16);
            over += __shfl_xor(over, 32);
            if (g == 0) overs[wave][16 * j + r] = over;
        }
        dot = row16_sum(dot);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = row16_sum(from_front[i]), l = row16_sum(to_back[i]), d = row16_sum(db[i]);
            if (r == 0) {
                fronts[half][row + i] = f;
                dbs[half][row + i] = d;
                if (half == 0) backs[row + i] = l;
            }
        }
        const float last = ys[C - 1];
        __syncthreads();
        bf16x8 both[2][3], dPa[2][3], dPt[2][3];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int from = 32 * s + 8 * g;
            split8<3>(at4(As + mine * kRow + from) + down4(As + from * kRow + mine, kRow), at4(As + mine * kRow + from + 4) + down4(As + (from + 4) * kRow + mine, kRow), both[s]);
            split8<3>(at4(Ps + mine * kRow + from), at4(Ps + mine * kRow + from + 4), dPa[s]);
            split8<3>(down4(Ps + from * kRow + mine, kRow), down4(Ps + (from + 4) * kRow + mine, kRow), dPt[s]);
        }
        if (wave == 0) {
            double from = (double)fronts[0][lane] + fronts[1][lane], to = backs[lane], dg = 0.0;
#pragma unroll
            for (int i = 0; i < kGradientWaves; ++i) dg += overs[i][lane];
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const double after = __shfl_down(from, off), before = __shfl_up(to, off);
                if (lane + off < 64) from += after;
                if (lane >= off) to += before;
            }
            to = __shfl_up(to, 1);
            dg += from + (lane > 0 ? to : 0.0) + (double)last * dot;
            if (lane < rows) {
                if (a.dg) *(float*)row_of<F32>(a.dg, a.dg_t, a.dg_b, t0 + lane, b, k.h) = lane < n ? (float)dg : 0.f;
                *(float*)row_of<F32>(a.dbeta, a.dbeta_t, a.dbeta_b, t0 + lane, b, k.h) = lane < n ? dbs[0][lane] + dbs[1][lane] : 0.f;
            }
        }
        // keys and queries by columns, and what the heads in front have left, a tile at a time (two at a time spill 128 bytes of a lane instead of 36: 8 x 1024
        // steps bf16 291 us)
        const u16 *const KT = at.KT(k) + late, *const QT = at.QT(k) + late;
        float* const shared = at.shared(k) + late;
        T *const dq0 = (T*)row_of<E>(a.dq, a.dq_t, a.dq_b, t0 + late, b, (int64_t)hk * a.Dk), *const dk0 = (T*)row_of<E>(a.dk, a.dk_t, a.dk_b, t0 + late, b, (int64_t)hk * a.Dk);
        const bool more = hh + 1 < group;
#pragma unroll
        for (int m = 0; m < kParts; ++m) {
            one_by_one();
            const int first = key_column(m / kEach, m % kEach), d = first + r + late;
            bf16x8 kt[2][kP], qt[2][kP];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                fragment<kP>(kt[s], KT + fragment_at(first / 16, 2, s) + 8 * lane, C * DKP);
                fragment<kP>(qt[s], QT + fragment_at(first / 16, 2, s) + 8 * lane, C * DKP);
            }
            f32x4v q4 = kZero4, k4 = kZero4;
            if (hh > 0)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float* const part = shared + (row + i + late) * DKP + first + r;
                    q4[i] = part[0];
                    k4[i] = part[C * DKP];
                }
            Sum sq, sk;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                multiply(sq, dPa[s], kt[s]);
                multiply(sk, both[s], kt[s]);
                multiply(sk, dPt[s], qt[s]);
            }
            q4 += dq_sum[m] + sq.total();
            k4 += dk_sum[m] + sk.total();
            if (more) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float* const part = shared + (row + i + late) * DKP + d;
                    part[0] = q4[i];
                    part[C * DKP] = k4[i];
                }
            } else if (d < a.Dk) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (row + i >= rows) continue;
                    E::store(dq0 + (row + i + late) * a.dq_t + d, row + i < n ? q4[i] : 0.f);
                    E::store(dk0 + (row + i + late) * a.dk_t + d, row + i < n ? k4[i] : 0.f);
                }
            }
        }
        __syncthreads();
    }
}

// ---- host

// Steps one by one up to here, in blocks from there on.  Blocks of 4 to 16 steps, one by one of 4 / 8 / 12 / 16, us: one sequence of 16 heads of 128 x 128 bf16
// 17 and 12.2 / 17.0 / 23.8 / 30.3; 16 of them 42 and 16.8 / 27.1 / 37.2 / 46.7; 64 of them 115 and 55.3 / 92.0 / 130 / 168; four of 8 heads of 100 x 100 fp32
// 24.7 and 11.7 / 15.1 / 20.3 / 25.8.  Four and 64 of 8 heads of 64 x 64 bf16 14.9 and 11.9 / 13.4 / 18.7 / 23.6, 36 and 14.0 / 22.4 / 30.3 / 38.2; four of 4 heads of
// 256 x 256 bf16 22 and 14.5 / 23.7 / 33.3 / 42.7.  Where the states alone fill the card, wide keys in fp32 gain from more single steps: 32 sequences of 4 heads of
// 256 x 256 111 and 21.1 / 30.5 / 39.5 / 47.2.
constexpr int kFewSteps = 8;

int64_t blocks(int T) { return (T + C - 1) / C; }

template <class E, int DKP, bool BACK>
hipError_t prepare(const DeltaArgs& a, hipStream_t s)
{
    const size_t lds = std::max<size_t>(2 * C * kStaged<E, DKP> * E::kBytes, 3 * C * kRow * sizeof(float));
    const auto kernel = a.Dk % 4 == 0 ? delta_prepare_kernel<E, DKP, BACK, true> : delta_prepare_kernel<E, DKP, BACK, false>;
    const hipError_t e = allow_dynamic_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks(a.T) * a.B * a.heads)), dim3(kThreads), lds, s, a);
    return hipGetLastError();
}

// Two tiles of columns to a workgroup from as many as keep all compute units busy with half the workgroups.  One and two tiles, us, 1024 steps of 16 heads of
// 128 x 128 bf16: one sequence (64 workgroups of two) 55 and 81, two 56 and 80, three 75 and 82, four (256) 87 and 94, in fp32 180 and 152;
// with the gradient 475 and 460.  300 steps of 8 heads of 100 x 100, fp32, with the gradient: four sequences (128) 152 and 170, eight (256) 254 and 240.
// 16 heads of 64 x 64 bf16: four sequences (128) 58 and 74, eight (256) 86 and 92, with the gradient 482 and 464, in fp32 176 and 151.
// Keys of more than 128 columns leave no registers for two.
bool two_tiles(const DeltaArgs& a) { return a.Dv > kTile && (int64_t)a.B * a.heads * ((a.Dv + 2 * kTile - 1) / (2 * kTile)) >= 256; }

template <class Kernel>
hipError_t walk_by(Kernel kernel, const DeltaArgs& a, int tiles, size_t lds, hipStream_t s)
{
    const hipError_t e = allow_dynamic_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)a.B * a.heads * tiles)), dim3(kThreads), lds, s, a, tiles);
    return hipGetLastError();
}
template <class E, int DKP, int NT, bool STATES>
hipError_t walk(const DeltaArgs& a, hipStream_t s)
{
    const size_t lds = NT * kTile * (3 * (DKP + 8) + 9 * kSteps) * sizeof(u16);
    return walk_by(delta_walk_kernel<E, DKP, NT, STATES>, a, (a.Dv + NT * kTile - 1) / (NT * kTile), lds, s);
}
template <class E, int DKP, int NT>
hipError_t walk_back(const DeltaArgs& a, hipStream_t s)
{
    const size_t lds = NT * kTile * (3 * (DKP + 8) + (9 + kPlanes<E>)*kSteps) * sizeof(u16);
    return walk_by(delta_walk_back_kernel<E, DKP, NT>, a, (a.Dv + NT * kTile - 1) / (NT * kTile), lds, s);
}

template <class E, int DKP>
hipError_t forward(const DeltaArgs& a, hipStream_t s)
{
    if (a.T <= kFewSteps) {
        const int tiles = (a.Dv + 31) / 32;
        hipLaunchKernelGGL((delta_step_kernel<E, DKP / 32>), dim3((unsigned)((int64_t)a.B * a.heads * tiles)), dim3(256), 0, s, a, tiles);
        return hipGetLastError();
    }
    const hipError_t e = prepare<E, DKP, false>(a, s);
    if (e != hipSuccess) return e;
    if constexpr (DKP <= 128)
        if (two_tiles(a)) return a.states ? walk<E, DKP, 2, true>(a, s) : walk<E, DKP, 2, false>(a, s);
    return a.states ? walk<E, DKP, 1, true>(a, s) : walk<E, DKP, 1, false>(a, s);
}

template <class E, int DKP>
hipError_t backward(const DeltaArgs& a, hipStream_t s)
{
    hipError_t e = a.T > 0 ? prepare<E, DKP, true>(a, s) : hipSuccess;
    if (e != hipSuccess) return e;
    const int tiles = (a.Dv + kTile - 1) / kTile;
    e = DKP <= 128 && two_tiles(a) ? walk_back<E, DKP, DKP <= 128 ? 2 : 1>(a, s) : walk_back<E, DKP, 1>(a, s);
    if (e != hipSuccess || a.T == 0) return e;
    hipLaunchKernelGGL((delta_update_kernel<E, DKP>), dim3((unsigned)(blocks(a.T) * a.B * a.heads * tiles)), dim3(kThreads), 0, s, a, tiles);
    constexpr int kRows = DKP < kRowsAtOnce ? DKP : kRowsAtOnce;
    const size_t lds = std::max<size_t>((6 * kRows + 3 * C) * kWideRow * sizeof(u16), 2 * C * kRow * sizeof(float));
    const auto kernel = a.Dv % 4 == 0 ? delta_gradient_kernel<E, DKP, true> : delta_gradient_kernel<E, DKP, false>;
    e = allow_dynamic_lds((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks(a.T) * a.B * a.key_heads)), dim3(kGradientThreads), lds, s, a);
    return hipGetLastError();
}

template <class E, int DKP>
size_t bytes_of(const DeltaArgs& a, bool back)
{
    return back ? Place<E, DKP, true>(a).bytes() : a.T <= kFewSteps ? 0 : Place<E, DKP, false>(a).bytes();
}
template <class E>
size_t bytes_by_width(const DeltaArgs& a, bool back)
{
    return a.Dk <= 64 ? bytes_of<E, 64>(a, back) : a.Dk <= 128 ? bytes_of<E, 128>(a, back) : bytes_of<E, 256>(a, back);
}

}  // namespace

// what either type asks for
size_t delta_workspace_bytes(int T, int B, int heads, int key_heads, int Dk, int Dv, bool back)
{
    DeltaArgs a = {};
    a.T = T; a.B = B; a.heads = heads; a.key_heads = key_heads; a.Dk = Dk; a.Dv = Dv;
    return std::max<size_t>(256, std::max(bytes_by_width<F32>(a, back), bytes_by_width<Bf16>(a, back)));
}

// a grid's threads have to stay under 2^32 (the blocks' gradient has twice as many to a workgroup; its workspace, 74 KB and more a block and head, ends in front of that)
bool delta_fits(int T, int B, int heads, int Dk, int Dv)
{
    const int64_t of_state = (int64_t)B * heads * ((Dv + kTile - 1) / kTile);
    return (int64_t)B * heads < (1 << 24) && of_state < (1 << 24) && blocks(T) * of_state < (1 << 24);
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
