// Scores over the vocabulary: log probabilities of given tokens with rank, entropy and the top alternatives, the distillation
// loss from a teacher's top logits, and the gradients of both by the logits.
//
//     d_j = l_j - max l     S = sum exp(d_j)     log p_j = d_j - log S     entropy = log S - sum exp(d_j) d_j / S
//     gradient: dl_j = dlogprob (1_t - p_j) - dentropy p_j (log p_j + entropy)
//
//     x = l / heat, s = softmax(x), t_j the teacher's share of word j of its list, t_r what it leaves for all others, s_r theirs
//     loss = heat^2 (sum_j t_j (log t_j - log s_j) + t_r (log t_r - log s_r))
//     gradient: dl_j = dloss heat (s_j - t_j) in the list, dloss heat s_j (1 - t_r / s_r) outside it
//
// A workgroup takes a row or a segment of it with its logits in registers, so that the maximum, the sums and the alternatives
// read them once; where a row has several segments a second launch joins them.
//
// Weights are 2^(l k - o) with k = log2(e) / heat in fp32 and o = k max l rounded: one fused multiply-add and the hardware's exponential, its
// argument off by half a step of itself, which a weight of 2^-t turns into t 2^-25 of itself.  What k and o have been rounded by is the same for
// a whole row and is put right in 64 bits: with e = k* / k - 1 (k* the exact one) and c = o (1 + e) - k* max l the sum over exp(d) is
// 2^c (sum + e ln 2 mean), mean being the sum of weight times exponent.  (An exponential of the difference in fp32, with what its product loses put
// in, and every sum in 64 bits took 62.7 us for 4096 rows of 10 000 bf16.)  Rows whose o is 2^20 or more take the differences.
// A clamp of the exponent at -200, whose weight is 0, takes in minus infinity and, where such tokens do not exist, NaN.
// Up to eight weights are added in fp32, those sums in fp64; the largest logit's own, which is 1, and those of its equals are counted beside them, so that
// the log p of a token that has nearly all mass is as exact as the sum over the others.
//
// Top alternatives: threads in groups; the n-th largest of the groups' own largest logits is a border that n logits reach, and only n groups
// hold logits that reach it; these are put in order by counting who is in front of whom.  A logit and its index make one key, so
// no two are equal.
#include "common.h"
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>

namespace l355 {

namespace {

typedef unsigned long long u64;
constexpr int kThreads = 256;               // of the kernels that join and that make gradients
constexpr int kGroups = 256;                // of threads, in the choice of alternatives
constexpr int kSweep = 8192;                // logits of a workgroup in the gradients
constexpr float kNone = -__builtin_inff(), kNothing = -200.f;
constexpr double kLog2e = 1.4426950408889634, kLn2 = 0.6931471805599453;

// l - biggest; 0 for an infinite logit that is the biggest
__device__ __forceinline__ float below(float l, float biggest) { return l == biggest ? 0.f : l - biggest; }

// The exponents l k - o of a row, and what their rounding adds up to
struct Exponents {
    float k, o;
    double e, c;
    bool usual;             // k biggest is small enough for c to be what rounding leaves (64 bits hold it to 2^-32)
    __device__ __forceinline__ Exponents(double exact, float biggest)
    {
        k = (float)exact;
        o = k * biggest;
        usual = fabsf(o) < 0x1p20f;
        e = exact / (double)k - 1.0;
        c = (double)o * (1.0 + e) - exact * (double)biggest;
    }
    __device__ __forceinline__ float of(float l) const { return fmaxf(fmaf(l, k, -o), kNothing); }
    // NaN stays
    __device__ __forceinline__ float or_nan(float l) const
    {
        const float t = fmaf(l, k, -o);
        return t < kNothing ? kNothing : t;
    }
};
// exp(scale d) for d <= 0, rows that are not usual; NaN stays
__device__ __forceinline__ float far_weight(float d) { return expf(d); }
__device__ __forceinline__ float far_weight(float d, double scale) { return expf((float)(d * scale)); }

// Over the 64 lanes, in every lane, by moves between registers: neighbour, other pair of the quad, half-row mirror, row mirror, then
// the two rows of a half and the two halves.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int CTRL, class T>
__device__ __forceinline__ T moved_by(T v)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, moved<CTRL>(__builtin_bit_cast(uint32_t, v)));
    } else {
        const u32x2v w = __builtin_bit_cast(u32x2v, v);
        return __builtin_bit_cast(T, (u32x2v){moved<CTRL>(w[0]), moved<CTRL>(w[1])});
    }
}
// both of what lanes a row (ROWS) or a half apart hold
template <bool ROWS, class T>
__device__ __forceinline__ void both_of(T v, T& a, T& b)
{
    const auto swap = [](uint32_t x) { return ROWS ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false); };
    if constexpr (sizeof(T) == 4) {
        const auto s = swap(__builtin_bit_cast(uint32_t, v));
        a = __builtin_bit_cast(T, (uint32_t)s[0]);
        b = __builtin_bit_cast(T, (uint32_t)s[1]);
    } else {
        const u32x2v w = __builtin_bit_cast(u32x2v, v);
        const auto lo = swap(w[0]), hi = swap(w[1]);
        a = __builtin_bit_cast(T, (u32x2v){(uint32_t)lo[0], (uint32_t)hi[0]});
        b = __builtin_bit_cast(T, (u32x2v){(uint32_t)lo[1], (uint32_t)hi[1]});
    }
}
template <class T, class F>
__device__ __forceinline__ T wave_join(T v, F join)
{
    v = join(v, moved_by<0xB1>(v));
    v = join(v, moved_by<0x4E>(v));
    v = join(v, moved_by<0x141>(v));
    v = join(v, moved_by<0x140>(v));
    T a, b;
    both_of<true>(v, a, b);
    v = join(a, b);
    both_of<false>(v, a, b);
    return join(a, b);
}
__device__ __forceinline__ float wave_max(float v)
{
    return wave_join(v, [](float a, float b) { return fmaxf(a, b); });
}
template <class T>
__device__ __forceinline__ T wave_add(T v)
{
    return wave_join(v, [](T a, T b) { return a + b; });
}
// over the workgroup, in every thread
template <int WAVES>
struct Shared {
    float f[WAVES];
    double d[WAVES], d2[WAVES];
    int i[WAVES];
};
template <int WAVES>
__device__ __forceinline__ float group_max(float v, Shared<WAVES>& sh)
{
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) sh.f[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh.f[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = fmaxf(v, sh.f[w]);
    return v;
}
// three sums in one go
template <int WAVES>
__device__ __forceinline__ void group_add(double& a, double& b, int& c, Shared<WAVES>& sh)
{
    a = wave_add(a);
    b = wave_add(b);
    c = wave_add(c);
    if ((threadIdx.x & 63) == 0) {
        sh.d[threadIdx.x >> 6] = a;
        sh.d2[threadIdx.x >> 6] = b;
        sh.i[threadIdx.x >> 6] = c;
    }
    __syncthreads();
    a = sh.d[0];
    b = sh.d2[0];
    c = sh.i[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
        a += sh.d[w];
        b += sh.d2[w];
        c += sh.i[w];
    }
}

// W neighbouring logits of a thread as they come, 16 bytes.  A piece that would reach behind the row is its last W logits, of which those in front of
// the piece's own column belong to somebody else: so no load has a branch, and all of a thread's are under way together.  (With a branch for the
// last piece, which the compiler waits in, 2048 rows of 32 000 bf16 took 66 us.)
template <class E>
constexpr int kWide = E::kBytes == 2 ? 8 : 4;
template <class E>
struct Piece {
    static constexpr int W = kWide<E>;
    u32x4v raw;
    static __device__ __forceinline__ int column(int col, int V) { return max(0, min(col, V - W)); }
    __device__ __forceinline__ void load(const typename E::T* row, int col, int V)
    {
        if (V >= W) {
            raw = *(const u32x4v_any*)(row + column(col, V));
        } else {        // a vocabulary of less than a piece
            typename E::T e[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (i < V) e[i] = row[i];
                else E::store(e + i, kNone);
            }
            __builtin_memcpy(&raw, e, 16);
        }
    }
    // the values; what is somebody else's becomes minus infinity (`whole`: the row reaches behind the chunk that the piece is of)
    __device__ __forceinline__ void take(int col, int V, bool whole, float* v) const
    {
        if constexpr (E::kBytes == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = bf16_lo(raw[i]);
                v[2 * i + 1] = bf16_hi(raw[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(raw[i]);
        }
        if (!whole) {
            const int others = col - column(col, V);
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = i >= others ? v[i] : kNone;
        }
    }
};
// a byte for each of W tokens, and the same where it is left out: such a token's logit becomes minus infinity
template <class E>
struct Mask {
    static constexpr int W = kWide<E>;
    uint32_t word[W / 4];
    __device__ __forceinline__ void load(const uint8_t* allowed, int col, int V)
    {
        if (V >= W) {
            __builtin_memcpy(word, allowed + Piece<E>::column(col, V), W);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (i % 4 == 0) word[i / 4] = 0;
                if (i < V) word[i / 4] |= (uint32_t)allowed[i] << i % 4 * 8;
            }
        }
    }
    __device__ __forceinline__ void apply(float* v) const
    {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = word[i / 4] >> (i % 4 * 8) & 0xff ? v[i] : kNone;
    }
};
// A piece of results, of which those in front of col are somebody else's
template <class E>
__device__ __forceinline__ void store_piece(typename E::T* row, int col, int V, bool whole, const float* v)
{
    constexpr int W = kWide<E>;
    const int at = Piece<E>::column(col, V);
    if (whole || at == col) {
        if (V >= W) {
            store_n<E, W, true>(row + at, v);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i)
        if (at + i >= col && at + i < V) E::store(row + at + i, v[i]);
}

// that of one token, none where it does not exist
template <class E>
__device__ __forceinline__ float logit_of(const typename E::T* row, const uint8_t* allowed, int token)
{
    const float v = E::load(row + token);
    return v == v && (!allowed || allowed[token]) ? v : kNone;
}

// Key of a token: larger for a larger logit, then for a smaller index; 0 for one that does not exist (NaN among them).  -0 is 0.
__device__ __forceinline__ u64 key_of(float v, int col)
{
    if (!(v > kNone)) return 0;
    const uint32_t u = __float_as_uint(v + 0.f), ordered = u >> 31 ? ~u : u | 0x80000000u;
    return (u64)ordered << 32 | (uint32_t)~col;
}
__device__ __forceinline__ float logit_of_key(u64 key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int token_of_key(u64 key) { return (int)~(uint32_t)key; }

// LIST: the most keys that can reach the border: those of kScoreMaxTop groups
template <int LIST>
struct TopShared {
    u64 most[kGroups];
    int front[kGroups];     // groups that are in front of each
    u64 list[LIST];
    u64 first[kScoreMaxTop];
    u64 border;
    int count;
};
// The n largest keys of the workgroup, in order, in sh.first (0 where there are fewer).  `most`: the thread's largest key;
// each(f): calls f with its keys.
template <int THREADS, int LIST, class Each>
__device__ __forceinline__ void top_keys(int n, u64 most, TopShared<LIST>& sh, Each each)
{
    constexpr int kOf = THREADS / kGroups;      // neighbouring threads of a group: 1 or 4
    const int tid = threadIdx.x;
    u64 group = most;
#pragma unroll
    for (int off = 1; off < kOf; off <<= 1) group = max(group, __shfl_xor(group, off));
    if (tid % kOf == 0) sh.most[tid / kOf] = group;
    if (tid == 0) {
        sh.border = 0;
        sh.count = 0;
    }
    if (tid < n) sh.first[tid] = 0;
    if (tid < kGroups) sh.front[tid] = 0;
    __syncthreads();
    {       // each thread a part of the groups that may be in front of its own
        const u64 mine = sh.most[tid % kGroups];
        int front = 0;
#pragma unroll 32
        for (int i = 0; i < kGroups / kOf; ++i) front += sh.most[tid / kGroups * (kGroups / kOf) + i] > mine;
        if constexpr (kOf == 1) {
            if (mine && front == n - 1) sh.border = mine;
        } else {
            atomicAdd(sh.front + tid % kGroups, front);
            __syncthreads();
            if (tid < kGroups && mine && sh.front[tid] == n - 1) sh.border = mine;
        }
    }
    __syncthreads();
    const u64 border = sh.border;
    if (most && most >= border)
        each(border, [&](u64 key) {
            if (key && key >= border) sh.list[atomicAdd(&sh.count, 1)] = key;
        });
    __syncthreads();
    // a wave counts for one key after another how many of the list are in front of it, 64 of them at a time
    const int count = sh.count, lane = tid & 63;
    const u64 near = lane < count ? sh.list[lane] : 0;
    for (int i = tid >> 6; i < count; i += THREADS / 64) {
        const u64 key = sh.list[i];
        int place = __popcll(__ballot(near > key));
        for (int j = 64; j < count && place < n; j += 64) place += __popcll(__ballot(j + lane < count && sh.list[j + lane] > key));
        if (lane == 0 && place < n) sh.first[place] = key;
    }
    __syncthreads();
}

// What is known of a row or of a segment
struct Part {
    double sum, mean;       // sum of exp(d), sum of exp(d) d
    float biggest;
    int front;              // tokens in front of the given one
};

__device__ __forceinline__ void finish_row(const ScoreArgs& a, int m, const Part& p, bool given, float mine, const u64* first)
{
    const bool some = p.biggest > kNone;
    const double log_sum = some ? log(p.sum) : 0.0;
    if (threadIdx.x == 0) {
        const double entropy = some ? log_sum - p.mean / p.sum : 0.0;
        if (a.logprob) a.logprob[m] = !given ? 0.f : mine > kNone ? (float)((double)below(mine, p.biggest) - log_sum) : kNone;
        if (a.rank) a.rank[m] = given ? p.front : -1;
        if (a.entropy) a.entropy[m] = (float)entropy;
        if (a.stats) {
            float* const s = a.stats + 4 * (int64_t)m;
            s[0] = p.biggest;
            s[1] = (float)log_sum;
            s[2] = (float)entropy;
            s[3] = some ? (float)(1.0 / p.sum) : 0.f;
        }
    }
    if (first && (int)threadIdx.x < a.top_n) {
        const u64 key = first[threadIdx.x];
        const int64_t at = (int64_t)m * a.top_n + threadIdx.x;
        a.top_token[at] = key ? token_of_key(key) : -1;
        a.top_logprob[at] = key ? (float)((double)below(logit_of_key(key), p.biggest) - log_sum) : kNone;
    }
}

__device__ __forceinline__ Part* parts_of(void* ws) { return (Part*)ws; }
__device__ __forceinline__ u64* keys_of(void* ws, int M, int segs) { return (u64*)(parts_of(ws) + (int64_t)M * segs); }

// The largest number below v (of zero, the smallest negative one)
__device__ __forceinline__ float just_below(float v)
{
    if (v == 0.f) return __uint_as_float(0x80000001u);
    const uint32_t u = __float_as_uint(v);
    return v == kNone ? v : __uint_as_float(u >> 31 ? u + 1 : u - 1);
}

// Measured: 4096 rows of 10 000 bf16 27 us (24.4 without the count of the largest), 3.0 TB/s, the vector units 73 % of the busy cycles (an exponential a logit at a quarter of
// the rate); 700 rows of 10 000 fp32 13 us; with 20 alternatives 256 rows of 32 000 bf16 and a mask 16 us, one row of 10 000 with 5 alternatives
// 9.2, where the row's eight barriers and the choice of alternatives follow each other on one compute unit.
template <class E, int VPT, int THREADS, bool TOP>
__global__ __launch_bounds__(THREADS) void score_kernel(ScoreArgs a, int segs)
{
    constexpr int W = kWide<E>, kChunks = VPT / W, kChunk = THREADS * W, kList = kScoreMaxTop * THREADS / kGroups * VPT;
    __shared__ Shared<THREADS / 64> sh;
    extern __shared__ u64 top_lds[];
    const int m = (int)(blockIdx.x / segs), seg = (int)(blockIdx.x % segs), first = seg * VPT * THREADS, tid = threadIdx.x;
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    const uint8_t* const allowed = a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr;
    const int chunks = min(kChunks, (a.V - first + kChunk - 1) / kChunk);       // that the row has; the same in all threads
    Piece<E> piece[kChunks];
    Mask<E> mask[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (c < chunks) piece[c].load(row, first + (c * THREADS + tid) * W, a.V);
    if (allowed)
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            if (c < chunks) mask[c].load(allowed, first + (c * THREADS + tid) * W, a.V);
    float v[VPT], most[kChunks], biggest = kNone;
    const auto column = [&](int c) { return Piece<E>::column(first + (c * THREADS + tid) * W, a.V); };
    const int token = a.token ? a.token[m] : -1;
    const bool given = token >= 0 && token < a.V;
    // the given token's logit: from the thread that holds it, or where that is in another segment from memory
    __shared__ float given_logit;
    float mine = kNone;
    if (given && (token < first || token >= first + kChunks * kChunk)) mine = logit_of<E>(row, allowed, token);
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (c < chunks) {
            piece[c].take(first + (c * THREADS + tid) * W, a.V, first + (c + 1) * kChunk <= a.V, v + c * W);
            if (allowed) mask[c].apply(v + c * W);
            const int place = token - first - (c * THREADS + tid) * W;
            if (given && place >= 0 && place < W) {
                const int shift = first + (c * THREADS + tid) * W - column(c);
#pragma unroll
                for (int i = 0; i < W; ++i)
                    if (i == place + shift) given_logit = v[c * W + i] == v[c * W + i] ? v[c * W + i] : kNone;
            }
            most[c] = kNone;
#pragma unroll
            for (int i = 0; i < W; ++i) most[c] = fmaxf(most[c], v[c * W + i]);
            biggest = fmaxf(biggest, most[c]);
        }
    const float own = biggest;
    Part p;
    p.biggest = biggest = group_max(biggest, sh);
    if (given && token >= first && token < first + kChunks * kChunk) mine = given_logit;
    p.sum = p.mean = 0.0;
    int front = 0, ones = 0;
    const Exponents x(kLog2e, biggest);
    if (x.usual) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            if (c < chunks) {
                float sum = 0.f, mean = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float t = x.of(v[c * W + i]), w = __builtin_amdgcn_exp2f(t);
                    sum += w;
                    mean = fmaf(w, t, mean);
                }
                if (most[c] == biggest) {       // a row's largest is here: the others once more
                    sum = mean = 0.f;
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float t = x.of(v[c * W + i]), w = v[c * W + i] == biggest ? 0.f : __builtin_amdgcn_exp2f(t);
                        sum += w;
                        mean = fmaf(w, t, mean);
                        ones += v[c * W + i] == biggest;
                    }
                }
                p.sum += sum;
                p.mean += mean;
            }
        const double scale = exp2(x.c), s = p.sum, t = p.mean;
        p.sum = scale * (s + x.e * kLn2 * t) + ones;
        p.mean = scale * kLn2 * (t * (1.0 + x.e) + x.c * s);
    } else if (biggest > kNone) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            if (c < chunks)
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float d = below(v[c * W + i], biggest), w = v[c * W + i] > kNone ? far_weight(d) : 0.f;
                    p.sum += w;
                    p.mean += w > 0.f ? w * d : 0.f;
                }
    }
    if (given) {
        // equal logits count in front of the token, so that there the border is just below it; the chunk that holds the token one by one
        const float before = just_below(mine);
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            if (c < chunks) {
                const int col = column(c);
                const float border = mine > kNone && col + W <= token ? before : mine;
#pragma unroll
                for (int i = 0; i < W; ++i) front += v[c * W + i] > border;
                if (mine > kNone && col < token && token < col + W)
#pragma unroll
                    for (int i = 0; i < W; ++i) front += v[c * W + i] == mine && col + i < token;
            }
    }
    group_add(p.sum, p.mean, front, sh);
    p.front = front;
    TopShared<kList>& top = *(TopShared<kList>*)top_lds;
    if constexpr (TOP) {
        int at = 0;
#pragma unroll
        for (int c = kChunks - 1; c >= 0; --c)
            if (c < chunks)
#pragma unroll
                for (int i = W - 1; i >= 0; --i) at = v[c * W + i] == own ? column(c) + i : at;
        top_keys<THREADS>(a.top_n, key_of(own, at), top, [&](u64 border, auto take) {
            const float least = border ? logit_of_key(border) : kNone;
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
                if (c < chunks)
#pragma unroll
                    for (int i = 0; i < W; ++i)
                        if (v[c * W + i] >= least) take(key_of(v[c * W + i], column(c) + i));
        });
    }
    if (segs == 1) {
        finish_row(a, m, p, given, mine, TOP ? top.first : nullptr);
        return;
    }
    if (tid == 0) parts_of(a.ws)[blockIdx.x] = p;
    if constexpr (TOP)
        if (tid < a.top_n) keys_of(a.ws, a.M, segs)[(int64_t)blockIdx.x * a.top_n + tid] = top.first[tid];
}

constexpr int kMostSegments = 128;          // of a row
constexpr int kJoinList = kMostSegments * kScoreMaxTop;
template <class E, bool TOP>
__global__ __launch_bounds__(kThreads) void score_join_kernel(ScoreArgs a, int segs)
{
    __shared__ Shared<kThreads / 64> sh;
    extern __shared__ u64 top_lds[];
    const int m = blockIdx.x, tid = threadIdx.x;
    Part p = {0.0, 0.0, kNone, 0};
    if (tid < segs) p = parts_of(a.ws)[(int64_t)m * segs + tid];
    const float biggest = group_max(p.biggest, sh);
    if (p.biggest > kNone) {
        const double d = below(p.biggest, biggest), f = exp(d);
        p.mean = f > 0.0 ? f * (p.mean + p.sum * d) : 0.0;
        p.sum *= f;
    }
    group_add(p.sum, p.mean, p.front, sh);
    p.biggest = biggest;
    const int token = a.token ? a.token[m] : -1;
    const bool given = token >= 0 && token < a.V;
    const float mine = given ? logit_of<E>((const typename E::T*)a.logits + (int64_t)m * a.ld, a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr, token)
                             : kNone;
    TopShared<kJoinList>& top = *(TopShared<kJoinList>*)top_lds;
    if constexpr (TOP) {
        const u64* const keys = keys_of(a.ws, a.M, segs) + (int64_t)m * segs * a.top_n;
        const int count = segs * a.top_n;
        u64 most = 0;
        for (int i = tid; i < count; i += kThreads) most = max(most, keys[i]);
        top_keys<kThreads>(a.top_n, most, top, [&](u64, auto take) {
            for (int i = tid; i < count; i += kThreads) take(keys[i]);
        });
    }
    finish_row(a, m, p, given, mine, TOP ? top.first : nullptr);
}

// Bound by memory: 700 rows of 10 000 fp32 12 us for 56 MB, 4.7 TB/s.  Nothing is shared between threads, so a workgroup is a stretch of a row.
template <class E>
__global__ __launch_bounds__(kThreads) void score_gradient_kernel(ScoreArgs a, int segs)
{
    constexpr int W = kWide<E>;
    const int m = (int)(blockIdx.x / segs), first = (int)(blockIdx.x % segs) * kSweep, end = min(first + kSweep, a.V);
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    typename E::T* const to = (typename E::T*)a.dlogits + (int64_t)m * a.dlogits_ld;
    const uint8_t* const allowed = a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr;
    const float* const stats = a.stats + 4 * (int64_t)m;
    const float biggest = stats[0], log_sum = stats[1], entropy = stats[2];
    const int token = a.token ? a.token[m] : -1;
    const bool given = token >= 0 && token < a.V;
    const float dlogprob = given && a.dlogprob ? a.dlogprob[m] : 0.f, dentropy = a.dentropy ? a.dentropy[m] : 0.f;
    const Exponents x(kLog2e, biggest);
    // log p = ln 2 (t + c) - log S up to e t, which is below a step of it; p = 2^t 2^c / S; bracket = constant + t slope
    const float per_sum = (float)(exp2(x.c) * (double)stats[3]);
    const float slope = dentropy * (float)kLn2, constant = dlogprob + dentropy * (float)(kLn2 * x.c - (double)log_sum + (double)entropy);
    // the given token's, with 1 - p and log p + entropy as such: of both little is left where it is nearly sure, and neither may be what rounding leaves
    // of dlogprob
    const auto of_given = [&](float l, float p) {
        const float log_p = below(l, biggest) - log_sum;
        return (p > 0.f ? -p * (dentropy * (log_p + entropy)) : 0.f) - dlogprob * expm1f(log_p);
    };
    constexpr int kChunks = kSweep / kThreads / W, kChunk = kThreads * W;
    const int chunks = (end - first + kChunk - 1) / kChunk;
    Piece<E> piece[kChunks];
    Mask<E> mask[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (c < chunks) {
            const int col = first + (c * kThreads + (int)threadIdx.x) * W;
            piece[c].load(row, col, a.V);
            if (allowed) mask[c].load(allowed, col, a.V);
        }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (c >= chunks) continue;
        const int col = first + (c * kThreads + (int)threadIdx.x) * W, at = Piece<E>::column(col, a.V);
        const bool whole = first + (c + 1) * kChunk <= a.V;
        float v[W], g[W];
        piece[c].take(col, a.V, whole, v);
        if (allowed) mask[c].apply(v);
        if (x.usual) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float t = x.of(v[i]);
                g[i] = -(__builtin_amdgcn_exp2f(t) * per_sum) * fmaf(t, slope, constant);
            }
            if (at <= token && token < at + W)
#pragma unroll
                for (int i = 0; i < W; ++i)
                    if (at + i == token && v[i] > kNone) g[i] = of_given(v[i], __builtin_amdgcn_exp2f(x.of(v[i])) * per_sum);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const bool exists = v[i] > kNone;
                const float d = exists ? below(v[i], biggest) : kNone, p = exists ? far_weight(d) * stats[3] : 0.f;
                const float bracket = p > 0.f ? fmaf(dentropy, d - log_sum + entropy, dlogprob) : 0.f;
                g[i] = !exists ? 0.f : at + i == token ? of_given(v[i], p) : -p * bracket;
            }
        }
        store_piece<E>(to, col, a.V, whole, g);
    }
}

// ---- distillation

struct RestPart {
    double sum;             // of exp((l - biggest) / heat) over the words outside the list
    float biggest;
    int twice;              // a word may stand in the list twice
};
constexpr int kOfLane = kDistillMaxTop / 64;

// Word j of a row's list, as far as it counts: one that is outside the vocabulary, or an earlier one again, does not.
struct Listed {
    int token;
    bool counts;
    double logit;           // the teacher's, over the heat
};
__device__ __forceinline__ Listed listed(const DistillArgs& a, int m, int j)
{
    Listed w = {-1, false, 0.0};
    if (j < a.K) {
        w.token = a.top_token[m * a.top_token_ld + j];
        w.counts = w.token >= 0 && w.token < a.V;
        w.logit = (double)a.top_logit[m * a.top_logit_ld + j] / a.temperature;
    }
    return w;
}
// looks through the list in front of word j
__device__ __forceinline__ bool again(const DistillArgs& a, int m, int j, int token)
{
    bool found = false;
    for (int i = 0; i < j; ++i) found |= a.top_token[m * a.top_token_ld + i] == token;
    return found;
}
// the largest, NaN where one is
__device__ __forceinline__ float wave_max_or_nan(float v)
{
    const bool bad = __ballot(v != v) != 0;
    v = wave_max(v);
    return bad ? __builtin_nanf("") : v;
}

// The loss of a row, by one wave: lane i has words i, i + 64, ..
template <class E>
__device__ void finish_loss(const DistillArgs& a, int m, const RestPart& rest)
{
    const int lane = threadIdx.x & 63;
    const double heat = a.temperature, per = 1.0 / heat;
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    Listed w[kOfLane];
    float l[kOfLane], biggest = kNone, most = kNone;
    int count = 0;
#pragma unroll
    for (int i = 0; i < kOfLane; ++i) w[i] = listed(a, m, lane + 64 * i);
    const int turns = (a.K + 63) / 64;          // the same in all lanes
    if (rest.twice)
#pragma unroll
        for (int i = 0; i < kOfLane; ++i) w[i].counts = w[i].counts && !again(a, m, lane + 64 * i, w[i].token);
#pragma unroll
    for (int i = 0; i < kOfLane; ++i) {
        l[i] = w[i].counts ? E::load(row + w[i].token) : kNone;
        biggest = fmaxf(biggest, l[i]);
        count += w[i].counts;
    }
    biggest = fmaxf(wave_max(biggest), rest.biggest);
    count = wave_add(count);
    // the student
    const bool some_rest = rest.sum > 0.0 || rest.sum != rest.sum;
    const double rest_d = (double)below(rest.biggest, biggest) * per;
    double d[kOfLane], in_list = 0.0;
#pragma unroll
    for (int i = 0; i < kOfLane; ++i) {
        if (i >= turns) continue;
        d[i] = (double)below(l[i], biggest) * per;
        in_list += w[i].counts ? exp(d[i]) : 0.0;
    }
    in_list = wave_add(in_list);
    const double sum = biggest == kNone ? (double)__builtin_nanf("") : in_list + (some_rest ? rest.sum * exp(rest_d) : 0.0);        // no logits: 0 / 0
    const double log_sum = log(sum);
    // the log of the share of what is outside, which may be too small for a number of its own
    const double log_rest = some_rest ? log(rest.sum) + rest_d : (double)kNone;
    // the teacher
    double norm = 0.0, log_norm = 0.0, t_rest = 0.0, in_teacher = 0.0, loss = 0.0;
    if (a.teacher_lse) {
        norm = a.teacher_lse[m];
    } else {
#pragma unroll
        for (int i = 0; i < kOfLane; ++i) most = w[i].counts && !(w[i].logit * heat <= (double)most) ? (float)(w[i].logit * heat) : most;
        norm = (double)wave_max_or_nan(most) * per;
        double z = 0.0;
#pragma unroll
        for (int i = 0; i < kOfLane; ++i)
            if (i < turns) z += w[i].counts ? exp(w[i].logit - norm) : 0.0;
        log_norm = log(wave_add(z));
    }
#pragma unroll
    for (int i = 0; i < kOfLane; ++i) {
        if (i >= turns) continue;
        const double log_t = w[i].logit - norm - log_norm, t = w[i].counts ? exp(log_t) : 0.0;
        in_teacher += t;
        loss += w[i].counts && t != 0.0 ? t * (log_t - (d[i] - log_sum)) : 0.0;
    }
    loss = wave_add(loss);
    if (a.teacher_lse) {
        const double left = 1.0 - wave_add(in_teacher);
        t_rest = left < 0.0 || count == a.V ? 0.0 : left;       // a list of all words leaves nobody to have what rounding leaves of 1
        if (t_rest > 0.0 && !some_rest) {
            // Nor does a student to whom all others are minus infinity.  A share t_j is off by its logit's and lse's half steps of 2^-24, their sum by those
            // weighed; four times that, for an lse that was worked out in fp32.
            double size = 0.0;
#pragma unroll
            for (int i = 0; i < kOfLane; ++i) {
                const double t = w[i].counts ? exp(w[i].logit - norm) : 0.0;
                size += t != 0.0 ? t * fabs(w[i].logit) : 0.0;
            }
            if (t_rest <= 0x1p-22 * (wave_add(size) + fabs(norm) + 1.0)) t_rest = 0.0;
        }
    }
    if (lane != 0) return;
    // what a word outside the list gets, as a factor of its s; where that would leave the range of fp32 the logarithm of what is
    // taken from it over exp(d) instead, which is then above 1
    double factor = 1.0;
    if (!a.teacher_lse && count == 0) {
        factor = loss = 0.0;        // no teacher in this row
    } else if (t_rest != 0.0) {
        const double r = log(t_rest) - (log_rest - log_sum);
        loss += t_rest * r;
        // (words that are all minus infinity have no s to take it from)
        if (some_rest) factor = r < 40.0 ? 1.0 - exp(r) : r != r ? r : log(t_rest) - log_rest;
    }
    if (a.loss) a.loss[m] = (float)(loss * heat * heat);
    if (a.stats) {
        float* const s = a.stats + 4 * (int64_t)m;
        s[0] = biggest;
        s[1] = (float)(rest.twice ? -1.0 / sum : 1.0 / sum);       // its sign says whether a word may stand in the list twice
        s[2] = (float)factor;
        s[3] = (float)log_norm;
    }
}

// The words of the list leave the sum over the others by a bit each in LDS, so that the share of all others is a sum and not 1 less what the list has.
// Measured: 2048 rows of 32 000 bf16 41 us, 3.2 TB/s, vector units 83 % of the busy cycles; 700 rows of 10 000 fp32 14 us.
template <class E, int VPT, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_kernel(DistillArgs a, int segs)
{
    constexpr int W = kWide<E>, kChunks = VPT / W, kChunk = THREADS * W;
    __shared__ Shared<THREADS / 64> sh;
    __shared__ uint32_t in_list[VPT * THREADS / 32];
    __shared__ int twice;
    const int m = (int)(blockIdx.x / segs), seg = (int)(blockIdx.x % segs), first = seg * VPT * THREADS, tid = threadIdx.x;
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    const int chunks = min(kChunks, (a.V - first + kChunk - 1) / kChunk);
    Piece<E> piece[kChunks];
    float v[VPT], biggest = kNone;
    const int word = tid < a.K ? a.top_token[m * a.top_token_ld + tid] : -1, at = word - first;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (c < chunks) piece[c].load(row, first + (c * THREADS + tid) * W, a.V);
    for (int i = tid; i < VPT * THREADS / 32; i += THREADS) in_list[i] = 0;
    if (tid == 0) twice = 0;
    __syncthreads();
    if (word >= 0 && at >= 0 && at < VPT * THREADS && atomicOr(in_list + at / 32, 1u << at % 32) >> at % 32 & 1) twice = 1;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (c < chunks) {
            const int place = (c * THREADS + tid) * W, from = Piece<E>::column(first + place, a.V) - first;
            piece[c].take(first + place, a.V, first + (c + 1) * kChunk <= a.V, v + c * W);
            // a piece moved to the row's end may start anywhere, in the segment in front of this one too (what is there is somebody else's)
            const int bit = max(from, 0);
            const uint64_t two = in_list[bit / 32] | (uint64_t)in_list[min(bit / 32 + 1, VPT * THREADS / 32 - 1)] << 32;
            const uint32_t bits = (uint32_t)(two >> bit % 32) << (bit - from);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                v[c * W + i] = bits >> i & 1 ? kNone : v[c * W + i];
                biggest = fmaxf(biggest, v[c * W + i]);
            }
        }
    RestPart p = {0.0, group_max(biggest, sh), twice};
    double unused = 0.0;
    int none = 0;
    const Exponents x(kLog2e / a.temperature, p.biggest);
    if (x.usual) {
        double mean = 0.0;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            if (c < chunks) {
                float sum = 0.f, t_sum = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float t = x.or_nan(v[c * W + i]), w = __builtin_amdgcn_exp2f(t);
                    sum += w;
                    t_sum = fmaf(w, t, t_sum);
                }
                p.sum += sum;
                mean += t_sum;
            }
        p.sum = exp2(x.c) * (p.sum + x.e * kLn2 * mean);
    } else {
        const double per = 1.0 / a.temperature;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            if (c < chunks)
#pragma unroll
                for (int i = 0; i < W; ++i) p.sum += v[c * W + i] == kNone ? 0.f : far_weight(below(v[c * W + i], p.biggest), per);
    }
    group_add(p.sum, unused, none, sh);
    if (segs > 1) {
        if (tid == 0) ((RestPart*)a.ws)[blockIdx.x] = p;
    } else if (tid < 64) {
        finish_loss<E>(a, m, p);
    }
}

// 2048 rows of two segments 8.6 us: the loss's chain of logarithms and exponentials in 64 bits, a wave a row.
template <class E>
__global__ __launch_bounds__(kThreads) void distill_join_kernel(DistillArgs a, int segs)
{
    __shared__ Shared<kThreads / 64> sh;
    const int m = blockIdx.x;
    RestPart p = {0.0, kNone, 0};
    if ((int)threadIdx.x < segs) p = ((const RestPart*)a.ws)[(int64_t)m * segs + threadIdx.x];
    const float biggest = group_max(p.biggest, sh);
    const bool some = p.sum > 0.0 || p.sum != p.sum;
    double unused = 0.0;
    p.sum = some ? p.sum * exp((double)below(p.biggest, biggest) / a.temperature) : 0.0;
    group_add(p.sum, unused, p.twice, sh);
    p.biggest = biggest;
    if (threadIdx.x < 64) finish_loss<E>(a, m, p);
}

// Bound by memory: 2048 rows of 32 000 bf16 46.5 us for 262 MB, 5.6 TB/s (some of it from the last-level cache); 700 rows of 10 000 fp32 13 us.
template <class E>
__global__ __launch_bounds__(kThreads) void distill_gradient_kernel(DistillArgs a, int segs)
{
    constexpr int W = kWide<E>;
    __shared__ Shared<kThreads / 64> sh;
    const int m = (int)(blockIdx.x / segs), first = (int)(blockIdx.x % segs) * kSweep, end = min(first + kSweep, a.V);
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    typename E::T* const to = (typename E::T*)a.dlogits + (int64_t)m * a.dlogits_ld;
    const float* const stats = a.stats + 4 * (int64_t)m;
    constexpr int kChunks = kSweep / kThreads / W, kChunk = kThreads * W;
    const int chunks = (end - first + kChunk - 1) / kChunk;
    Piece<E> piece[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (c < chunks) piece[c].load(row, first + (c * kThreads + (int)threadIdx.x) * W, a.V);
    const float biggest = stats[0], factor = stats[2];
    const double per_sum = fabs((double)stats[1]), per = 1.0 / a.temperature;
    const float scale = (float)(a.dloss[m] * a.temperature);
    Listed w = listed(a, m, threadIdx.x);
    if (stats[1] < 0.f) w.counts = w.counts && !again(a, m, threadIdx.x, w.token);
    // a word of the list that lies in this segment: its logit is read in front of all writes, which may be to the same place
    const bool here = w.counts && w.token >= first && w.token < end;
    float mine = 0.f;
    double log_t = w.logit;
    if (a.teacher_lse) {
        log_t -= a.teacher_lse[m];
    } else {
        const float z = w.counts ? (float)(w.logit * a.temperature) : kNone;
        const bool bad = __syncthreads_or(z != z);
        const float most = group_max(z, sh);
        log_t -= (bad ? (double)__builtin_nanf("") : (double)most * per) + (double)stats[3];
    }
    if (here) {
        const double s = exp((double)below(E::load(row + w.token), biggest) * per) * per_sum;
        mine = (float)((double)scale * (s - exp(log_t)));
    }
    __syncthreads();
    const Exponents x(kLog2e * per, biggest);
    const bool far_rest = factor > 1.f || !x.usual;
    const float kept = (float)((double)scale * (factor > 1.f ? 1.0 : (double)factor) * per_sum * (x.usual ? exp2(x.c) : 1.0));
    // a weight 2^t is off by e ln 2 t of itself, e being what k has been rounded by, and that is as much as its argument's rounding may be
    const float off = (float)(x.e * kLn2);
    const auto weight = [&](float l) {
        const float t = x.or_nan(l), w = __builtin_amdgcn_exp2f(t);
        return fmaf(w * t, off, w);
    };
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (c >= chunks) continue;
        const int col = first + (c * kThreads + (int)threadIdx.x) * W;
        const bool whole = first + (c + 1) * kChunk <= a.V;
        float v[W];
        piece[c].take(col, a.V, whole, v);
        if (factor == 0.f) {        // nothing to anybody outside the list: no teacher, whatever the row holds, or the others have what is theirs
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = 0.f;
        } else if (!far_rest) {
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = kept * weight(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const double d = (double)below(v[i], biggest) * per;
                v[i] = kept * (x.usual ? weight(v[i]) : expf((float)d)) - (factor > 1.f ? scale * expf(fminf((float)(d + (double)factor), 0.f)) : 0.f);
            }
        }
        store_piece<E>(to, col, a.V, whole, v);
    }
    __syncthreads();
    if (here) E::store(to + w.token, mine);
}

// ---- host

// How rows are laid over workgroups
struct Lay {
    int threads, per_thread, segs;
};
Lay lay_of(int M, int V)
{
    // many rows: four waves to a row or a segment, whose waits others fill (2048 rows of 32 000 bf16 in two segments and joined 50 us, one to
    // sixteen waves 65); else sixteen, so that a row of up to 65 536 is one launch
    Lay l;
    l.threads = M >= 512 ? 256 : 1024;
    l.per_thread = 8;
    while (l.per_thread < 64 && l.threads * l.per_thread < V) l.per_thread *= 2;
    // longer rows in segments: of few rows, shorter ones
    l.segs = (V + l.threads * l.per_thread - 1) / (l.threads * l.per_thread);
    if (l.segs > 1)
        while (l.per_thread > 8 && (int64_t)M * l.segs < 256) {
            l.per_thread /= 2;
            l.segs = (V + l.threads * l.per_thread - 1) / (l.threads * l.per_thread);
        }
    return l;
}
static_assert(kSampleMaxVocabulary <= kMostSegments * 8 * 1024 && kMostSegments <= kThreads, "");

template <class E, int VPT, int THREADS, bool TOP>
hipError_t score(const ScoreArgs& a, int segs, hipStream_t s)
{
    const dim3 grid((unsigned)((int64_t)a.M * segs));
    const size_t lds = TOP ? sizeof(TopShared<kScoreMaxTop * THREADS / kGroups * VPT>) : 0;
    const auto kernel = score_kernel<E, VPT, THREADS, TOP>;
    hipError_t e = TOP ? allow_dynamic_lds((const void*)kernel, lds) : hipSuccess;
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(THREADS), lds, s, a, segs);
    if (segs > 1) {
        const auto join = score_join_kernel<E, TOP>;
        const size_t join_lds = TOP ? sizeof(TopShared<kJoinList>) : 0;
        e = TOP ? allow_dynamic_lds((const void*)join, join_lds) : hipSuccess;
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(join, dim3(a.M), dim3(kThreads), join_lds, s, a, segs);
    }
    return hipGetLastError();
}
template <class E, int VPT, int THREADS>
hipError_t distill(const DistillArgs& a, int segs, hipStream_t s)
{
    hipLaunchKernelGGL((distill_kernel<E, VPT, THREADS>), dim3((unsigned)((int64_t)a.M * segs)), dim3(THREADS), 0, s, a, segs);
    if (segs > 1) hipLaunchKernelGGL((distill_join_kernel<E>), dim3(a.M), dim3(kThreads), 0, s, a, segs);
    return hipGetLastError();
}
template <class E, int THREADS, bool TOP>
hipError_t score_by(const ScoreArgs& a, const Lay& l, hipStream_t s)
{
    switch (l.per_thread) {
    case 8: return score<E, 8, THREADS, TOP>(a, l.segs, s);
    case 16: return score<E, 16, THREADS, TOP>(a, l.segs, s);
    case 32: return score<E, 32, THREADS, TOP>(a, l.segs, s);
    default: return score<E, 64, THREADS, TOP>(a, l.segs, s);
    }
}
template <class E>
hipError_t score_of(const ScoreArgs& a, hipStream_t s)
{
    Lay l = lay_of(a.M, a.V);
    if (l.threads == 256) return a.top_n ? score_by<E, 256, true>(a, l, s) : score_by<E, 256, false>(a, l, s);
    return a.top_n ? score_by<E, 1024, true>(a, l, s) : score_by<E, 1024, false>(a, l, s);
}
template <class E, int THREADS>
hipError_t distill_by(const DistillArgs& a, const Lay& l, hipStream_t s)
{
    switch (l.per_thread) {
    case 8: return distill<E, 8, THREADS>(a, l.segs, s);
    case 16: return distill<E, 16, THREADS>(a, l.segs, s);
    case 32: return distill<E, 32, THREADS>(a, l.segs, s);
    default: return distill<E, 64, THREADS>(a, l.segs, s);
    }
}
template <class E>
hipError_t distill_of(const DistillArgs& a, hipStream_t s)
{
    const Lay l = lay_of(a.M, a.V);
    return l.threads == 256 ? distill_by<E, 256>(a, l, s) : distill_by<E, 1024>(a, l, s);
}

}  // namespace

// a grid's threads have to stay under 2^32
bool score_fits(int M, int V)
{
    return M >= 0 && V >= 1 && V <= kSampleMaxVocabulary && M < (1 << 22) && (int64_t)M * ((V + kSweep - 1) / kSweep) < (1 << 24) &&
           (int64_t)M * lay_of(M, V).segs * lay_of(M, V).threads < ((int64_t)1 << 32);
}
size_t score_workspace_bytes(int M, int V, int top_n)
{
    const int segs = lay_of(M, V).segs;
    return std::max<size_t>(256, segs == 1 ? 0 : (size_t)M * segs * (sizeof(Part) + sizeof(u64) * top_n));
}
size_t distill_workspace_bytes(int M, int V)
{
    const int segs = lay_of(M, V).segs;
    return std::max<size_t>(256, segs == 1 ? 0 : (size_t)M * segs * sizeof(RestPart));
}

hipError_t launch_score_forward(const ScoreArgs& a, hipStream_t s) { return a.bf16 ? score_of<Bf16>(a, s) : score_of<F32>(a, s); }
hipError_t launch_distill_forward(const DistillArgs& a, hipStream_t s) { return a.bf16 ? distill_of<Bf16>(a, s) : distill_of<F32>(a, s); }
hipError_t launch_score_backward(const ScoreArgs& a, hipStream_t s)
{
    const int segs = (a.V + kSweep - 1) / kSweep;
    const dim3 grid((unsigned)((int64_t)a.M * segs)), block(kThreads);
    if (a.bf16) hipLaunchKernelGGL(score_gradient_kernel<Bf16>, grid, block, 0, s, a, segs);
    else hipLaunchKernelGGL(score_gradient_kernel<F32>, grid, block, 0, s, a, segs);
    return hipGetLastError();
}
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s)
{
    const int segs = (a.V + kSweep - 1) / kSweep;
    const dim3 grid((unsigned)((int64_t)a.M * segs)), block(kThreads);
    if (a.bf16) hipLaunchKernelGGL(distill_gradient_kernel<Bf16>, grid, block, 0, s, a, segs);
    else hipLaunchKernelGGL(distill_gradient_kernel<F32>, grid, block, 0, s, a, segs);
    return hipGetLastError();
}

}  // namespace l355
