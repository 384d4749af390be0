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
// read them once; where a row has several segments a second launch joins them.  Terms are fp32, their sums fp64: the entropy
// of a row that is nearly sure is what is left of two sums.
//
// Top alternatives: the n-th largest of the 256 threads' own largest logits is a border that n logits reach, and only n threads
// hold logits that reach it; these are put in order by counting who is in front of whom.  A logit and its index make one key, so
// no two are equal.
#include "common.h"
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>

namespace l355 {

namespace {

typedef unsigned long long u64;
constexpr int kThreads = 256, kScoreWaves = kThreads / 64;
constexpr int kMostSegments = 64;           // of a row
constexpr int kSweep = 8192;                // logits of a workgroup in the gradients
constexpr float kNone = -__builtin_inff();

constexpr double kLog2e = 1.4426950408889634;

// exp(c d) for d <= 0: 2 to the power of d k, k = c log2 e as the sum of two floats, with what the product's rounding lost put in
// afterwards (without, d = -20 would be off by 1e-6).  Minus infinity gives 0, NaN stays.
struct Exp {
    float hi, lo;
    __device__ __forceinline__ explicit Exp(double c) : hi((float)(c * kLog2e)), lo((float)(c * kLog2e - (double)(float)(c * kLog2e))) {}
    __device__ __forceinline__ float operator()(float d) const
    {
        d = d < -1e30f ? -1e30f : d;
        const float t = d * hi, lost = fmaf(d, lo, fmaf(d, hi, -t)), x = __builtin_amdgcn_exp2f(t);
        return fmaf(x * lost, 0.6931471805599453f, x);
    }
};
// l - biggest; 0 for an infinite logit that is the biggest
__device__ __forceinline__ float below(float l, float biggest) { return l == biggest ? 0.f : l - biggest; }

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}
template <class T>
__device__ __forceinline__ T wave_add(T v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
// over the workgroup, in every thread
struct Shared {
    float f[kScoreWaves];
    double d[kScoreWaves];
    int i[kScoreWaves];
};
__device__ __forceinline__ float group_max(float v, Shared& sh)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.f[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(sh.f[0], sh.f[1]), fmaxf(sh.f[2], sh.f[3]));
}
__device__ __forceinline__ double group_add(double v, Shared& sh)
{
    v = wave_add(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.d[threadIdx.x >> 6] = v;
    __syncthreads();
    return (sh.d[0] + sh.d[1]) + (sh.d[2] + sh.d[3]);
}
__device__ __forceinline__ int group_add(int v, Shared& sh)
{
    v = wave_add(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.i[threadIdx.x >> 6] = v;
    __syncthreads();
    return (sh.i[0] + sh.i[1]) + (sh.i[2] + sh.i[3]);
}
static_assert(kScoreWaves == 4, "");

// W neighbouring logits from col on; what lies behind the row is minus infinity
template <class E>
constexpr int kWide = E::kBytes == 2 ? 8 : 4;
template <class E>
__device__ __forceinline__ void load_wide(const typename E::T* row, int col, int V, float* v)
{
    constexpr int W = kWide<E>;
    if (col + W <= V) {
        load_n<E, W, true>(row + col, v);
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = col + e < V ? E::load(row + col + e) : kNone;
    }
}
template <class E>
__device__ __forceinline__ void store_wide(typename E::T* row, int col, int V, const float* v)
{
    constexpr int W = kWide<E>;
    if (col + W <= V) {
        store_n<E, W, true>(row + col, v);
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
            if (col + e < V) E::store(row + col + e, v[e]);
    }
}
// a byte for each of them that does not exist becomes minus infinity, and so does NaN
template <class E>
__device__ __forceinline__ void leave_out(const uint8_t* allowed, int col, int V, float* v)
{
    constexpr int W = kWide<E>;
    if (allowed) {
        if (col + W <= V) {
            uint32_t word[W / 4];
            __builtin_memcpy(word, allowed + col, W);
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = word[e / 4] >> (e % 4 * 8) & 0xff ? v[e] : kNone;
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = col + e < V && allowed[col + e] ? v[e] : kNone;
        }
    }
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = v[e] == v[e] ? v[e] : kNone;
}
// that of one token, none where it does not exist
template <class E>
__device__ __forceinline__ float logit_of(const typename E::T* row, const uint8_t* allowed, int token)
{
    const float v = E::load(row + token);
    return v == v && (!allowed || allowed[token]) ? v : kNone;
}

// Key of a token: larger for a larger logit, then for a smaller index; 0 for one that does not exist.  -0 is 0.
__device__ __forceinline__ u64 key_of(float v, int col)
{
    if (v == kNone) return 0;
    const uint32_t u = __float_as_uint(v + 0.f), ordered = u >> 31 ? ~u : u | 0x80000000u;
    return (u64)ordered << 32 | (uint32_t)~col;
}
__device__ __forceinline__ float logit_of_key(u64 key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int token_of_key(u64 key) { return (int)~(uint32_t)key; }

struct TopShared {
    u64 most[kThreads];
    u64 list[kScoreMaxTop * 64];
    u64 first[kScoreMaxTop];
    u64 border;
    int count;
};
// The n largest keys of the workgroup, in order, in sh.first (0 where there are fewer).  `most`: the thread's largest key;
// each(f): calls f with its keys, at most 64.
template <class Each>
__device__ __forceinline__ void top_keys(int n, u64 most, TopShared& sh, Each each)
{
    const int tid = threadIdx.x;
    __syncthreads();
    sh.most[tid] = most;
    if (tid == 0) {
        sh.border = 0;
        sh.count = 0;
    }
    if (tid < n) sh.first[tid] = 0;
    __syncthreads();
    int front = 0;
#pragma unroll 8
    for (int i = 0; i < kThreads; ++i) front += sh.most[i] > most;
    if (most && front == n - 1) sh.border = most;
    __syncthreads();
    const u64 border = sh.border;
    if (most && most >= border)
        each([&](u64 key) {
            if (key && key >= border) sh.list[atomicAdd(&sh.count, 1)] = key;
        });
    __syncthreads();
    const int count = sh.count;
    for (int i = tid; i < count; i += kThreads) {
        const u64 key = sh.list[i];
        int place = 0;
        for (int j = 0; j < count; ++j) place += sh.list[j] > key;
        if (place < n) sh.first[place] = key;
    }
    __syncthreads();
}

// What is known of a row or of a segment
struct Part {
    double sum, mean;       // sum of exp(d), sum of exp(d) d
    float biggest;
    int front;              // tokens in front of the given one
};

__device__ __forceinline__ void finish_row(const ScoreArgs& a, int m, const Part& p, bool given, float mine, const TopShared* top)
{
    const bool some = p.biggest > kNone;
    const double log_sum = some ? log(p.sum) : 0.0;
    const double entropy = some ? log_sum - p.mean / p.sum : 0.0;
    if (threadIdx.x == 0) {
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
    if (top && (int)threadIdx.x < a.top_n) {
        const u64 key = top->first[threadIdx.x];
        const int64_t at = (int64_t)m * a.top_n + threadIdx.x;
        a.top_token[at] = key ? token_of_key(key) : -1;
        a.top_logprob[at] = key ? (float)((double)below(logit_of_key(key), p.biggest) - log_sum) : kNone;
    }
}

__device__ __forceinline__ Part* parts_of(void* ws) { return (Part*)ws; }
__device__ __forceinline__ u64* keys_of(void* ws, int M, int segs) { return (u64*)(parts_of(ws) + (int64_t)M * segs); }

template <class E, int VPT, bool TOP>
__global__ __launch_bounds__(kThreads) void score_kernel(ScoreArgs a, int segs)
{
    constexpr int W = kWide<E>;
    __shared__ Shared sh;
    __shared__ std::conditional_t<TOP, TopShared, int> top;
    const int m = (int)(blockIdx.x / segs), seg = (int)(blockIdx.x % segs), first = seg * VPT * kThreads;
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    const uint8_t* const allowed = a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr;
    const int token = a.token ? a.token[m] : -1;
    const bool given = token >= 0 && token < a.V;
    const float mine = given ? logit_of<E>(row, allowed, token) : kNone;
    float v[VPT], biggest = kNone;
#pragma unroll
    for (int c = 0; c < VPT / W; ++c) load_wide<E>(row, first + (c * kThreads + (int)threadIdx.x) * W, a.V, v + c * W);
#pragma unroll
    for (int c = 0; c < VPT / W; ++c) leave_out<E>(allowed, first + (c * kThreads + (int)threadIdx.x) * W, a.V, v + c * W);
#pragma unroll
    for (int i = 0; i < VPT; ++i) biggest = fmaxf(biggest, v[i]);
    const float own = biggest;
    const auto col_of = [&](int i) { return first + (i / W * kThreads + (int)threadIdx.x) * W + i % W; };
    Part p;
    p.biggest = biggest = group_max(biggest, sh);
    p.sum = p.mean = 0.0;
    int front = 0;
    if (biggest > kNone) {
        const Exp e(1.0);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const float d = below(v[i], biggest), x = e(d);
            p.sum += x;
            p.mean += x > 0.f ? x * d : 0.f;
        }
        if (given)
#pragma unroll
            for (int i = 0; i < VPT; ++i) front += v[i] > mine || (v[i] == mine && v[i] > kNone && col_of(i) < token);
    }
    p.sum = group_add(p.sum, sh);
    p.mean = group_add(p.mean, sh);
    p.front = group_add(front, sh);
    if constexpr (TOP) {
        int at = 0;
#pragma unroll
        for (int i = VPT - 1; i >= 0; --i) at = v[i] == own ? col_of(i) : at;
        top_keys(a.top_n, key_of(own, at), top, [&](auto take) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) take(key_of(v[i], col_of(i)));
        });
    }
    if (segs == 1) {
        if constexpr (TOP) finish_row(a, m, p, given, mine, &top);
        else finish_row(a, m, p, given, mine, nullptr);
        return;
    }
    if (threadIdx.x == 0) parts_of(a.ws)[blockIdx.x] = p;
    if constexpr (TOP)
        if ((int)threadIdx.x < a.top_n) keys_of(a.ws, a.M, segs)[(int64_t)blockIdx.x * a.top_n + threadIdx.x] = top.first[threadIdx.x];
}

template <class E, bool TOP>
__global__ __launch_bounds__(kThreads) void score_join_kernel(ScoreArgs a, int segs)
{
    __shared__ Shared sh;
    __shared__ std::conditional_t<TOP, TopShared, int> top;
    const int m = blockIdx.x, tid = threadIdx.x;
    Part p = {0.0, 0.0, kNone, 0};
    if (tid < segs) p = parts_of(a.ws)[(int64_t)m * segs + tid];
    const float biggest = group_max(p.biggest, sh);
    if (p.biggest > kNone) {
        const double d = below(p.biggest, biggest), f = exp(d);
        p.mean = f > 0.0 ? f * (p.mean + p.sum * d) : 0.0;
        p.sum *= f;
    }
    p.sum = group_add(p.sum, sh);
    p.mean = group_add(p.mean, sh);
    p.front = group_add(p.front, sh);
    p.biggest = biggest;
    const int token = a.token ? a.token[m] : -1;
    const bool given = token >= 0 && token < a.V;
    const float mine = given ? logit_of<E>((const typename E::T*)a.logits + (int64_t)m * a.ld, a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr, token)
                             : kNone;
    if constexpr (TOP) {
        const u64* const keys = keys_of(a.ws, a.M, segs) + (int64_t)m * segs * a.top_n;
        const int count = segs * a.top_n;       // at most 64 for each thread
        u64 most = 0;
        for (int i = tid; i < count; i += kThreads) most = max(most, keys[i]);
        top_keys(a.top_n, most, top, [&](auto take) {
            for (int i = tid; i < count; i += kThreads) take(keys[i]);
        });
        finish_row(a, m, p, given, mine, &top);
    } else {
        finish_row(a, m, p, given, mine, nullptr);
    }
}
static_assert(kMostSegments * kScoreMaxTop <= 64 * kThreads, "");

template <class E>
__global__ __launch_bounds__(kThreads) void score_gradient_kernel(ScoreArgs a, int segs)
{
    constexpr int W = kWide<E>;
    const int m = (int)(blockIdx.x / segs), first = (int)(blockIdx.x % segs) * kSweep, end = min(first + kSweep, a.V);
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    typename E::T* const to = (typename E::T*)a.dlogits + (int64_t)m * a.dlogits_ld;
    const uint8_t* const allowed = a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr;
    const float* const stats = a.stats + 4 * (int64_t)m;
    const float biggest = stats[0], log_sum = stats[1], entropy = stats[2], per_sum = stats[3];
    const int token = a.token ? a.token[m] : -1;
    const bool given = token >= 0 && token < a.V;
    const float dlogprob = given && a.dlogprob ? a.dlogprob[m] : 0.f, dentropy = a.dentropy ? a.dentropy[m] : 0.f;
    const Exp e(1.0);
#pragma unroll 2
    for (int col = first + (int)threadIdx.x * W; col < end; col += kThreads * W) {
        float v[W];
        load_wide<E>(row, col, a.V, v);
        leave_out<E>(allowed, col, a.V, v);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float d = below(v[i], biggest), p = e(d) * per_sum;
            float g = dlogprob;
            if (a.dentropy) g = p > 0.f ? fmaf(dentropy, d - log_sum + entropy, g) : 0.f;
            g *= -p;
            if (col + i == token) g += dlogprob;
            v[i] = v[i] > kNone ? g : 0.f;
        }
        store_wide<E>(to, col, a.V, v);
    }
}

// ---- distillation

struct RestPart {
    double sum;             // of exp((l - biggest) / heat) over the words outside the list
    float biggest;
};

// Word j of a row's list.  A word that is outside the vocabulary, or an earlier one again, does not count.
struct Listed {
    int token;
    bool counts;
    double logit;           // the teacher's, over the heat
};
__device__ __forceinline__ Listed listed(const DistillArgs& a, int m, int* tokens)
{
    const int j = threadIdx.x;
    Listed w = {-1, false, 0.0};
    if (j < a.K) {
        w.token = a.top_token[m * a.top_token_ld + j];
        w.counts = w.token >= 0 && w.token < a.V;
        w.logit = (double)a.top_logit[m * a.top_logit_ld + j] / (double)a.temperature;
    }
    tokens[j] = w.token;
    __syncthreads();
    for (int i = 0; i < j && j < a.K; ++i) w.counts &= tokens[i] != w.token;
    return w;
}
__device__ __forceinline__ float group_max_or_nan(float v, Shared& sh)
{
    const double n = group_add(v != v ? 1.0 : 0.0, sh);
    v = group_max(v, sh);
    return n > 0.0 ? __builtin_nanf("") : v;
}

template <class E>
__device__ void finish_loss(const DistillArgs& a, int m, RestPart rest, Shared& sh, int* tokens)
{
    const Listed w = listed(a, m, tokens);
    const double heat = a.temperature, per = 1.0 / heat;
    const float l = w.counts ? E::load((const typename E::T*)a.logits + (int64_t)m * a.ld + w.token) : kNone;
    const float biggest = fmaxf(group_max(l, sh), rest.biggest);
    // the student
    const double d = (double)below(l, biggest) * per;
    const double in_list = group_add(w.counts ? exp(d) : 0.0, sh);
    const double outside = rest.sum > 0.0 || rest.sum != rest.sum ? rest.sum * exp((double)below(rest.biggest, biggest) * per) : 0.0;
    const double sum = biggest == kNone ? (double)__builtin_nanf("") : in_list + outside, log_sum = log(sum);      // no logits: 0 / 0
    // the log of the share of what is outside, which may be too small for a number of its own
    const double log_rest = rest.sum > 0.0 || rest.sum != rest.sum ? log(rest.sum) + (double)below(rest.biggest, biggest) * per : (double)kNone;
    // the teacher
    const int count = group_add((int)w.counts, sh);
    double norm = 0.0, t_rest = 0.0, log_t = (double)kNone, log_norm = 0.0;
    if (a.teacher_lse) {
        norm = a.teacher_lse[m];
        log_t = w.logit - norm;
    } else {
        const float most = group_max_or_nan(w.counts ? (float)(w.logit * heat) : kNone, sh);
        log_norm = log(group_add(w.counts ? exp(w.logit - (double)most * per) : 0.0, sh));
        log_t = w.logit - (double)most * per - log_norm;
    }
    const double t = w.counts ? exp(log_t) : 0.0;
    if (a.teacher_lse) {
        const double left = 1.0 - group_add(t, sh);
        t_rest = left < 0.0 ? 0.0 : left;
    }
    double loss = group_add(w.counts && t != 0.0 ? t * (log_t - (d - log_sum)) : 0.0, sh);
    if (threadIdx.x != 0) return;
    // what a word outside the list gets, as a factor of its s; where that would leave the range of fp32 the logarithm of what is
    // taken from it over exp(d) instead, which is then above 1
    double factor = 1.0;
    if (!a.teacher_lse && count == 0) {
        factor = loss = 0.0;        // no teacher in this row
    } else if (t_rest != 0.0) {
        loss += t_rest * (log(t_rest) - (log_rest - log_sum));
        const double r = log(t_rest) - (log_rest - log_sum);
        factor = r < 40.0 ? 1.0 - exp(r) : r != r ? r : log(t_rest) - log_rest;
    }
    if (a.loss) a.loss[m] = (float)(loss * heat * heat);
    if (a.stats) {
        float* const s = a.stats + 4 * (int64_t)m;
        s[0] = biggest;
        s[1] = (float)(1.0 / sum);
        s[2] = (float)factor;
        s[3] = (float)log_norm;
    }
}

template <class E, int VPT>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a, int segs)
{
    constexpr int W = kWide<E>;
    __shared__ Shared sh;
    __shared__ int tokens[kThreads];
    __shared__ uint32_t in_list[VPT * kThreads / 32];
    const int m = (int)(blockIdx.x / segs), seg = (int)(blockIdx.x % segs), first = seg * VPT * kThreads, tid = threadIdx.x;
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    for (int i = tid; i < VPT * kThreads / 32; i += kThreads) in_list[i] = 0;
    float v[VPT], biggest = kNone;
#pragma unroll
    for (int c = 0; c < VPT / W; ++c) load_wide<E>(row, first + (c * kThreads + tid) * W, a.V, v + c * W);
    __syncthreads();
    if (tid < a.K) {
        const int at = a.top_token[m * a.top_token_ld + tid] - first;
        if (at >= 0 && at < VPT * kThreads) atomicOr(in_list + at / 32, 1u << at % 32);
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < VPT / W; ++c) {
        const int at = (c * kThreads + tid) * W;
        const uint32_t bits = in_list[at / 32] >> at % 32;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v[c * W + i] = bits >> i & 1 ? kNone : v[c * W + i];
            biggest = fmaxf(biggest, v[c * W + i]);
        }
    }
    RestPart p;
    p.biggest = group_max(biggest, sh);
    double sum = 0.0;
    const Exp e(1.0 / (double)a.temperature);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const float x = e(below(v[i], p.biggest));
        sum += v[i] == kNone ? 0.f : x;
    }
    p.sum = group_add(sum, sh);
    if (segs == 1) finish_loss<E>(a, m, p, sh, tokens);
    else if (tid == 0) ((RestPart*)a.ws)[blockIdx.x] = p;
}

template <class E>
__global__ __launch_bounds__(kThreads) void distill_join_kernel(DistillArgs a, int segs)
{
    __shared__ Shared sh;
    __shared__ int tokens[kThreads];
    const int m = blockIdx.x;
    RestPart p = {0.0, kNone};
    if ((int)threadIdx.x < segs) p = ((const RestPart*)a.ws)[(int64_t)m * segs + threadIdx.x];
    const float biggest = group_max(p.biggest, sh);
    const bool some = p.sum > 0.0 || p.sum != p.sum;
    p.sum = group_add(some ? p.sum * exp((double)below(p.biggest, biggest) / (double)a.temperature) : 0.0, sh);
    p.biggest = biggest;
    finish_loss<E>(a, m, p, sh, tokens);
}

template <class E>
__global__ __launch_bounds__(kThreads) void distill_gradient_kernel(DistillArgs a, int segs)
{
    constexpr int W = kWide<E>;
    __shared__ Shared sh;
    __shared__ int tokens[kThreads];
    const int m = (int)(blockIdx.x / segs), first = (int)(blockIdx.x % segs) * kSweep, end = min(first + kSweep, a.V);
    const typename E::T* const row = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    typename E::T* const to = (typename E::T*)a.dlogits + (int64_t)m * a.dlogits_ld;
    const float* const stats = a.stats + 4 * (int64_t)m;
    const float biggest = stats[0], per_sum = stats[1], factor = stats[2];
    const float scale = a.dloss[m] * a.temperature;
    const Listed w = listed(a, m, tokens);
    const double per = 1.0 / (double)a.temperature;
    const Exp e(per), one(1.0);
    // a word of the list that lies in this segment: its logit is read in front of all writes, which may be to the same place
    const bool here = w.counts && w.token >= first && w.token < end;
    float mine = 0.f;
    double log_t = w.logit;
    if (a.teacher_lse) log_t -= a.teacher_lse[m];
    else log_t -= (double)group_max_or_nan(w.counts ? (float)(w.logit * (double)a.temperature) : kNone, sh) * per + (double)stats[3];
    if (here) {
        const double s = exp((double)below(E::load(row + w.token), biggest) * per) * (double)per_sum;
        mine = (float)((double)scale * (s - exp(log_t)));
    }
    __syncthreads();
    const float kept = scale * (factor > 1.f ? 1.f : factor) * per_sum, fper = (float)per;
#pragma unroll 2
    for (int col = first + (int)threadIdx.x * W; col < end; col += kThreads * W) {
        float v[W];
        load_wide<E>(row, col, a.V, v);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float d = below(v[i], biggest);
            v[i] = kept * e(d);
            if (factor > 1.f) v[i] -= scale * one(fminf(fmaf(d, fper, factor), 0.f));
        }
        store_wide<E>(to, col, a.V, v);
    }
    __syncthreads();
    if (here) E::store(to + w.token, mine);
}

// ---- host

int segments(int V, int per_thread) { return (V + per_thread * kThreads - 1) / (per_thread * kThreads); }
// Logits of a thread: as few as keep 1024 workgroups busy, as many as leave a row 64 segments
int per_thread(int M, int V)
{
    int n = 8;
    while (n < 64 && ((int64_t)M * segments(V, n) > 1024 || segments(V, n) > kMostSegments) && segments(V, n) > 1) n *= 2;
    return n;
}

template <class E, int VPT>
hipError_t score(const ScoreArgs& a, hipStream_t s)
{
    const int segs = segments(a.V, VPT);
    const dim3 grid((unsigned)((int64_t)a.M * segs)), block(kThreads);
    if (a.top_n) hipLaunchKernelGGL((score_kernel<E, VPT, true>), grid, block, 0, s, a, segs);
    else hipLaunchKernelGGL((score_kernel<E, VPT, false>), grid, block, 0, s, a, segs);
    if (segs > 1) {
        if (a.top_n) hipLaunchKernelGGL((score_join_kernel<E, true>), dim3(a.M), block, 0, s, a, segs);
        else hipLaunchKernelGGL((score_join_kernel<E, false>), dim3(a.M), block, 0, s, a, segs);
    }
    return hipGetLastError();
}
template <class E, int VPT>
hipError_t distill(const DistillArgs& a, hipStream_t s)
{
    const int segs = segments(a.V, VPT);
    hipLaunchKernelGGL((distill_kernel<E, VPT>), dim3((unsigned)((int64_t)a.M * segs)), dim3(kThreads), 0, s, a, segs);
    if (segs > 1) hipLaunchKernelGGL((distill_join_kernel<E>), dim3(a.M), dim3(kThreads), 0, s, a, segs);
    return hipGetLastError();
}
template <class E>
hipError_t score_of(const ScoreArgs& a, hipStream_t s)
{
    switch (per_thread(a.M, a.V)) {
    case 8: return score<E, 8>(a, s);
    case 16: return score<E, 16>(a, s);
    case 32: return score<E, 32>(a, s);
    default: return score<E, 64>(a, s);
    }
}
template <class E>
hipError_t distill_of(const DistillArgs& a, hipStream_t s)
{
    switch (per_thread(a.M, a.V)) {
    case 8: return distill<E, 8>(a, s);
    case 16: return distill<E, 16>(a, s);
    case 32: return distill<E, 32>(a, s);
    default: return distill<E, 64>(a, s);
    }
}

}  // namespace

// a grid's threads have to stay under 2^32
bool score_fits(int M, int V)
{
    return M >= 0 && V >= 1 && V <= kSampleMaxVocabulary && M < (1 << 22) && (int64_t)M * ((V + kSweep - 1) / kSweep) < (1 << 24);
}
size_t score_workspace_bytes(int M, int V, int top_n)
{
    const int segs = segments(V, per_thread(M, V));
    return std::max<size_t>(256, segs == 1 ? 0 : (size_t)M * segs * (sizeof(Part) + sizeof(u64) * top_n));
}
size_t distill_workspace_bytes(int M, int V)
{
    const int segs = segments(V, per_thread(M, V));
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
