// The draw of one token per row of logits from given random numbers: temperature, then the top_k likeliest, then the shortest
// prefix of those that holds top_p of their mass, then those within min_p of the likeliest.
//
//     w_j = exp((l_j - max l) / temperature), as a whole number of 2^-S
//     order: logit descending, index ascending; what top_k and top_p keep is everything up to one token, the border
//     token = first index, ascending, at which the running sum over the kept exceeds u times their sum
//
// Weights are evaluated in 64 bits and summed as 64-bit whole numbers: a sum has the same bits in every order, so atomics and
// the cut of the work do not change who is drawn.
//
// A workgroup per row; each wave has a run of neighbouring tokens, 256 at a time (four to a lane), which every step reads again
// from the caches (kept in registers, 32 a lane, the unrolled steps spilled).  A border is found by a histogram over 2048 bins of the logit's distance to the
// largest one - of counts for top_k, of masses for top_p - and the tokens of the bin in which it lies are compared one by one
// (kList of them; more than that, in rows of equal or of very far logits, by the digits of the logit's bit pattern).
//
// Bound: the vector units' 64-bit arithmetic (about 17 instructions a weight) and the barriers between the steps.
#include "elem.h"
#include "lm_ops.h"

namespace l355 {

namespace {

typedef unsigned long long u64;
constexpr int kBins = 2048, kList = 512, kTable = 1024;
constexpr int kChunk = 256;         // tokens of a wave at a time

// Bits of a value in ascending order; both zeros are one value.  Every number above minus infinity has a key above 0.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

struct Shared {
    union {
        u64 mass[kBins];
        unsigned count[kBins];
    };
    double table[kTable];           // 2^(k / 1024)
    u64 list_weight[kList];
    uint32_t list_key[kList];
    int list_index[kList];
    u64 part[16];
    u64 found_before;
    unsigned found_digit, listed;
    uint32_t border_key;
    int border_index;
};

// The weight of a token as a whole number: 2^(y / 1024) 2^S with y = (l - top) 1024 log2(e) / temperature, y = n + r,
// 2^(n / 1024) by table and exponent, 2^(r / 1024) by its series to the third power (r at most a half: 6e-16).
struct Weights {
    const double* table;
    double top, scale;
    uint32_t top_key;
    int bits;                       // S, at most 51: adding 2^52 rounds to a whole number in the low bits
    bool infinite;                  // the largest logit is plus infinity and has all mass
    __device__ __forceinline__ u64 whole(uint32_t key) const
    {
        if (infinite) return key == top_key ? 1ull << bits : 0ull;
        const double y = fmax(((double)value_of(key) - top) * scale, -1024.0 * 1074.0);
        const double n = rint(y), r = y - n;
        const int i = (int)n;
        constexpr double c1 = 6.769015435155716e-4 /* ln 2 / 1024 */, c2 = c1 * c1 / 2, c3 = c1 * c1 * c1 / 6;
        const double p = fma(fma(fma(c3, r, c2), r, c1), r, 1.0);
        const double v = __builtin_amdgcn_ldexp(table[i & (kTable - 1)] * p, (i >> 10) + bits);
        return (u64)__double_as_longlong(v + 0x1p52) & 0xfffffffffffffull;
    }
};

// One row as a workgroup of WAVES waves sees it
template <class E, int VEC>
struct Row {
    const typename E::T* logits;
    const uint8_t* allowed;
    int V, first, chunks, lane;     // first: of the wave's tokens

    __device__ __forceinline__ int index(int chunk, int e) const { return first + chunk * kChunk + lane * 4 + e; }
    // keys of four neighbouring tokens; 0: masked (what it holds is not looked at), NaN, minus infinity or behind the row
    __device__ __forceinline__ void load(int chunk, uint32_t (&k)[4]) const
    {
        const int j = index(chunk, 0);
        float v[4];
        uint32_t mask = 0x01010101u;
        if (VEC == 4) {
            if (j < V) {            // V is a multiple of four
                load_n<E, 4>(logits + j, v);
                if (allowed) mask = *(const uint32_t*)(allowed + j);
            } else {
                mask = 0;
            }
        } else {
            mask = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < V) {
                    v[e] = E::load(logits + j + e);
                    mask |= (allowed ? (uint32_t)allowed[j + e] : 1u) << (8 * e);
                }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) k[e] = (mask >> (8 * e) & 255u) && v[e] > -__builtin_inff() ? key_of(v[e]) : 0u;
    }
    // f(chunk, keys) for the wave's tokens in their order
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
#pragma unroll 2
        for (int c = 0; c < chunks; ++c) {
            uint32_t k[4];
            load(c, k);
            f(c, k);
        }
    }
};

__device__ __forceinline__ u64 wave_total(u64 v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}
__device__ __forceinline__ u64 wave_front(u64 v, int lane)     // sum over the lanes in front
{
    u64 incl = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 up = __shfl_up(incl, off, 64);
        if (lane >= off) incl += up;
    }
    return incl - v;
}
// Sum over the waves in front of this one and over all of them, of a value that every lane of a wave has
template <int WAVES>
__device__ __forceinline__ u64 join(u64 v, Shared& sh, u64* total)
{
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.part[wave] = v;
    __syncthreads();
    u64 front = 0, all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const u64 p = sh.part[i];
        if (i < wave) front += p;
        all += p;
    }
    *total = all;
    return front;
}

// The first bin from `last` down to 0 or, DOWN = false, from 0 up, at which base + the sum so far reaches `want`, and the sum in
// front of it.  Behind a barrier; all threads.
template <int WAVES, bool MASS, bool DOWN>
__device__ __forceinline__ void crossing(Shared& sh, u64 base, double want, unsigned* bin, u64* before)
{
    constexpr int kEach = kBins / (64 * WAVES);
    u64 v[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = threadIdx.x * kEach + i, b = DOWN ? kBins - 1 - at : at;
        v[i] = MASS ? sh.mass[b] : sh.count[b];
        sum += v[i];
    }
    const int lane = threadIdx.x & 63;
    const u64 inside = wave_front(sum, lane);
    u64 total;
    u64 front = base + join<WAVES>(__shfl(inside + sum, 63, 64), sh, &total) + inside;
    if ((double)front < want && (double)(front + sum) >= want) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if ((double)front < want && (double)(front + v[i]) >= want) {
                const int at = threadIdx.x * kEach + i;
                sh.found_digit = DOWN ? kBins - 1 - at : at;
                sh.found_before = front;
            }
            front += v[i];
        }
    }
    __syncthreads();
    *bin = sh.found_digit;
    *before = sh.found_before;
}

// The first token in index order at which the running sum of weight(key, index) exceeds `past` (counts: reaches past + 1), given
// each wave's sum.  One wave finds it and calls found(index, key).
template <int WAVES, class R, class W, class F>
__device__ __forceinline__ void in_order(const R& row, u64 front, u64 mine, double past, W weight, F found)
{
    if (!((double)front <= past && (double)(front + mine) > past)) return;
    bool done = false;
    row.each([&](int c, const uint32_t (&k)[4]) {
        if (done) return;
        u64 w[4], sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = weight(k[e], row.index(c, e));
            sum += w[e];
        }
        const u64 chunk = wave_total(sum);
        if ((double)(front + chunk) > past) {
            u64 run = front + wave_front(sum, row.lane);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if ((double)run <= past && (double)(run + w[e]) > past) found(row.index(c, e), k[e]);
                run += w[e];
            }
            done = true;
        }
        front += chunk;
    });
}

constexpr int kDigitShift[3] = {21, 10, 0};
constexpr unsigned kDigitMask[3] = {2047u, 2047u, 1023u};

// What stays is every token in front of (key, index) in the order, and that token
struct Border {
    uint32_t key;
    int index;
    __device__ __forceinline__ bool keeps(uint32_t k, int j) const { return k > key || (k == key && j <= index); }
};

// The border among the tokens that `old` keeps: the first token at which the sum of their counts or masses reaches `want`
// (MASS: share * the sum of all, at least 1).
template <int WAVES, bool MASS, class R>
__device__ __forceinline__ Border find_border(const R& row, const Weights& w, Shared& sh, float top, float bins_per_unit, const Border& old, double want)
{
    constexpr int kThreads = 64 * WAVES;
    const int tid = threadIdx.x;
    auto weight = [&](uint32_t k) -> u64 { return MASS ? w.whole(k) : 1ull; };
    // a larger distance never has a smaller bin: difference, product and conversion are monotone
    auto bin_of = [&](uint32_t k) -> unsigned { return k == w.top_key ? 0u : (unsigned)fminf((top - value_of(k)) * bins_per_unit, (float)(kBins - 1)); };
    auto clear = [&]() {
        for (int i = tid; i < kBins; i += kThreads) {
            if (MASS) sh.mass[i] = 0;
            else sh.count[i] = 0;
        }
        if (tid == 0) sh.listed = 0;
    };
    auto add = [&](unsigned b, uint32_t k) {
        if (MASS) atomicAdd(&sh.mass[b], weight(k));
        else atomicAdd(&sh.count[b], 1u);
    };
    __syncthreads();
    clear();
    __syncthreads();
    row.each([&](int c, const uint32_t (&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k[e] && old.keeps(k[e], row.index(c, e))) add(bin_of(k[e]), k[e]);
    });
    __syncthreads();
    if (MASS) {
        u64 sum = 0, total;
        for (int i = tid; i < kBins; i += kThreads) sum += sh.mass[i];
        join<WAVES>(wave_total(sum), sh, &total);
        want = fmax(want * (double)total, 1.0);     // the likeliest token always stays
    }
    unsigned bin;
    u64 before;
    crossing<WAVES, MASS, false>(sh, 0, want, &bin, &before);
    // the tokens of that bin
    row.each([&](int c, const uint32_t (&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = row.index(c, e);
            if (k[e] && old.keeps(k[e], j) && bin_of(k[e]) == bin) {
                const unsigned at = atomicAdd(&sh.listed, 1u);
                if (at < kList) {
                    sh.list_key[at] = k[e];
                    sh.list_index[at] = j;
                    sh.list_weight[at] = weight(k[e]);
                }
            }
        }
    });
    __syncthreads();
    const unsigned listed = sh.listed;
    if (listed <= kList) {
        // each against all: the sum in front of it in the order
        for (unsigned i = tid; i < listed; i += kThreads) {
            const uint32_t k = sh.list_key[i];
            const int j = sh.list_index[i];
            u64 front = before;
            for (unsigned o = 0; o < listed; ++o) {
                const uint32_t ko = sh.list_key[o];
                if (ko > k || (ko == k && sh.list_index[o] < j)) front += sh.list_weight[o];
            }
            if ((double)front < want && (double)(front + sh.list_weight[i]) >= want) {
                sh.border_key = k;
                sh.border_index = j;
            }
        }
        __syncthreads();
        return Border{sh.border_key, sh.border_index};
    }
    // many: digit by digit of the key, then by index among equal ones
    uint32_t prefix = 0;
    for (int d = 0; d < 3; ++d) {
        __syncthreads();
        clear();
        __syncthreads();
        row.each([&](int c, const uint32_t (&k)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (k[e] && old.keeps(k[e], row.index(c, e)) && bin_of(k[e]) == bin && (d == 0 || k[e] >> kDigitShift[d - 1] == prefix >> kDigitShift[d - 1]))
                    add((k[e] >> kDigitShift[d]) & kDigitMask[d], k[e]);
        });
        __syncthreads();
        unsigned digit;
        crossing<WAVES, MASS, true>(sh, before, want, &digit, &before);
        prefix |= digit << kDigitShift[d];
    }
    const double nth = ceil((want - (double)before) / (double)weight(prefix));      // 1: the first of the equal ones
    auto equal = [&](uint32_t k, int j) -> u64 { return k == prefix && old.keeps(k, j); };
    u64 count = 0, total;
    row.each([&](int c, const uint32_t (&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) count += equal(k[e], row.index(c, e));
    });
    const u64 mine = wave_total(count), front = join<WAVES>(mine, sh, &total);
    in_order<WAVES>(row, front, mine, fmin(nth, (double)total) - 1.0, equal, [&](int j, uint32_t) { sh.border_index = j; });
    __syncthreads();
    return Border{prefix, sh.border_index};
}

template <class E, int WAVES, int VEC>
__global__ __launch_bounds__(64 * WAVES) void sample_kernel(SampleArgs a, int bits)
{
    __shared__ Shared sh;
    const int m = blockIdx.x, tid = threadIdx.x;
    Row<E, VEC> row;
    row.logits = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    row.allowed = a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr;
    row.V = a.V;
    row.lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), all_chunks = (a.V + kChunk - 1) / kChunk, each = (all_chunks + WAVES - 1) / WAVES;
    row.first = wave * each * kChunk;
    row.chunks = max(0, min(each, all_chunks - wave * each));
    const float heat = a.temperature ? a.temperature[m] : 1.f;
    const bool greedy = !(heat > 0.f);
    const int top_k = a.top_k ? a.top_k[m] : 0;
    const double top_p = a.top_p ? (double)a.top_p[m] : 1.0, min_p = a.min_p ? fmin((double)a.min_p[m], 1.0) : 0.0;
    for (int i = tid; i < kTable; i += 64 * WAVES) sh.table[i] = exp2((double)i / kTable);

    // largest key, the first token that has it, and how many tokens there are
    u64 best = 0;                   // key, then the index from the back
    unsigned there = 0;
    row.each([&](int c, const uint32_t (&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const u64 v = (u64)k[e] << 32 | (unsigned)(0x7fffffff - row.index(c, e));
            best = k[e] && v > best ? v : best;
            there += k[e] != 0;
        }
    });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        const u64 o = __shfl_xor(best, off, 64);
        best = o > best ? o : best;
        there += __shfl_xor(there, off, 64);
    }
    if (row.lane == 0) {
        sh.part[wave] = best;
        sh.list_weight[wave] = there;
    }
    __syncthreads();
    u64 tokens = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        best = sh.part[i] > best ? sh.part[i] : best;
        tokens += sh.list_weight[i];
    }
    if (tokens == 0 || greedy) {
        if (tid == 0) {
            a.token[m] = tokens ? 0x7fffffff - (int)(unsigned)best : -1;
            if (a.prob) a.prob[m] = tokens ? 1.f : 0.f;
            if (a.kept) a.kept[m] = tokens ? 1 : 0;
        }
        return;
    }
    const float top = value_of((uint32_t)(best >> 32));
    Weights w;
    w.table = sh.table;
    w.top = (double)top;
    w.scale = 1024.0 * 1.4426950408889634 / (double)heat;
    w.top_key = (uint32_t)(best >> 32);
    w.bits = bits;
    w.infinite = top == __builtin_inff();
    const double one = (double)(1ull << bits);
    // 64 bins to a factor of e, over 32 of them; a weight behind that is below 2^-46
    const float bins_per_unit = fminf(64.f / heat, 0x1p100f);

    Border border = {0u, -1};       // all
    if (top_k > 0 && (u64)top_k < tokens) border = find_border<WAVES, false>(row, w, sh, top, bins_per_unit, border, (double)top_k);
    if (top_p < 1.0) border = find_border<WAVES, true>(row, w, sh, top, bins_per_unit, border, top_p);

    const double least = min_p * one;
    auto kept_weight = [&](uint32_t k, int j, bool* kept) -> u64 {
        if (k == 0 || !border.keeps(k, j)) return 0;
        const u64 v = w.whole(k);
        if ((double)v < least) return 0;
        *kept = true;
        return v;
    };
    u64 mass = 0, total, all_kept;
    unsigned kept = 0;
    __syncthreads();
    row.each([&](int c, const uint32_t (&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            bool here = false;
            mass += kept_weight(k[e], row.index(c, e), &here);
            kept += here;
        }
    });
    const u64 mine = wave_total(mass);
    // both sums in one exchange: a row has at most 2^20 tokens
    join<WAVES>(wave_total(kept), sh, &all_kept);
    const u64 front = join<WAVES>(mine, sh, &total);
    const double want = fmin(fmax((double)a.u[m], 0.0), 0x1.fffffep-1) * (double)total;
    in_order<WAVES>(
        row, front, mine, want,
        [&](uint32_t k, int j) {
            bool here;
            return kept_weight(k, j, &here);
        },
        [&](int j, uint32_t k) {
            a.token[m] = j;
            if (a.prob) a.prob[m] = (float)((double)w.whole(k) / (double)total);
        });
    if (tid == 0 && a.kept) a.kept[m] = (int)all_kept;
}

template <class E, int VEC>
void sample(const SampleArgs& a, int bits, hipStream_t s)
{
    const dim3 grid(a.M);
    // four waves up to 2048 tokens: fewer to wait for at each of some twenty barriers
    if (a.V <= 2048) hipLaunchKernelGGL((sample_kernel<E, 4, VEC>), grid, dim3(256), 0, s, a, bits);
    else hipLaunchKernelGGL((sample_kernel<E, 16, VEC>), grid, dim3(1024), 0, s, a, bits);
}

}  // namespace

size_t sample_workspace_bytes(int, int) { return 256; }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s)
{
    int bits = 62;          // V weights of at most 1 stay below 2^62
    for (int v = a.V; v > 1; v = (v + 1) / 2) --bits;
    bits = bits < 51 ? bits : 51;
    const bool fours = a.V % 4 == 0 && a.ld % 4 == 0 && ((uintptr_t)a.logits & (a.bf16 ? 7 : 15)) == 0 && a.allowed_ld % 4 == 0 && ((uintptr_t)a.allowed & 3) == 0;
    if (a.bf16) {
        if (fours) sample<Bf16, 4>(a, bits, s);
        else sample<Bf16, 1>(a, bits, s);
    } else {
        if (fours) sample<F32, 4>(a, bits, s);
        else sample<F32, 1>(a, bits, s);
    }
    return hipGetLastError();
}

}  // namespace l355
