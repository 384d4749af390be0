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
// A workgroup per row; each wave has a run of neighbouring tokens, 256 at a time (four to a lane).  Every step reads them again,
// from LDS where the row fits there (HELD: masks and NaN done), else from the caches (in registers, 32 a lane, the unrolled
// steps spilled).  A border is found by a histogram over 2048 bins of the logit's distance to the largest one - of counts for
// top_k, of masses for top_p - and the tokens of the bin in which it lies are compared one by one (kList of them; more than
// that, in rows of equal or of very far logits, by the digits of the logit's bit pattern).  The token is found in two steps:
// the wave in whose run the sum is passed, then that run cut over all threads.
//
// Bound: the row's one compute unit, in steps that wait for each other at sixteen barriers; a batch takes what its slowest rows
// take.  256 rows of 32 000 bf16: 9.8 us greedy, 19.6 without a filter, 21.7 with top_k 50, 33 with top_p 0.95, 29 with both, 36 to
// 38 with mixed settings and masks (vector instructions fill 55 % of the busy cycles there); one row of 10 000 with both 17.0.
#include "common.h"
#include "elem.h"
#include "lm_ops.h"

namespace l355 {

namespace {

typedef unsigned long long u64;
constexpr int kBins = 2048, kList = 512, kTable = 1024;
constexpr int kChunk = 256;         // tokens of a wave at a time
constexpr int kAhead = 2;           // ... and of these so many are requested at once from memory
constexpr float kInf = __builtin_inff();
// A row is held where it fits beside Shared, up to 28 672 fp32 and 57 344 bf16 tokens.  us held and read again from the caches,
// top_k 50 and top_p 0.95: one row of 10 000 fp32 17.0 and 20.8, 28 000 24.2 and 31.5, of 57 344 bf16 37.7 and 51.0, 512 rows of 4000
// 27.1 and 31.0, of 28 000 55 and 79, 2048 rows of 2000 42.8 and 48.1; with mixed settings 36.0 and 40.3 there.
constexpr size_t kHeldBytes = 112 << 10;
// chunks of each of `waves` runs over a row
__host__ __device__ constexpr int chunks_of(int V, int waves) { return ((V + kChunk - 1) / kChunk + waves - 1) / waves; }

// Bits of a value in ascending order; both zeros are one value
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key ^ ((uint32_t)((int)~key >> 31) | 0x80000000u)); }

struct Shared {
    union {
        u64 mass[kBins];
        unsigned count[kBins];
    };
    double table[kTable];           // 2^(k / 1024)
    u64 list_weight[kList], list_front[kList];
    float list_value[kList];
    int list_index[kList];
    u64 part[2][16], kept[16];
    float gathered[16][128];        // of each wave: what each_kept waits with
    u64 found_before;
    unsigned found_bin, listed;
    float border_value;
    int border_index;
};

// The weight of a token as a whole number: 2^(y / 1024) 2^S with y = (l - top) 1024 log2(e) / temperature, y = n + r,
// 2^(n / 1024) by table and exponent, 2^(r / 1024) by its series to the third power (r at most a half: 6e-16).
struct Weights {
    const double* table;
    double scale, shift;            // y = l scale + shift
    float top;
    int bits;                       // S, at most 51: adding 2^52 rounds to a whole number in the low bits
    // No branch in here: the chains of several tokens run side by side.  Of minus infinity or NaN it is anything.
    __device__ __forceinline__ u64 whole(float v) const
    {
        const double y = fma((double)v, scale, shift), n = rint(y), r = y - n;
        int i;                      // the instruction's own saturation: a weight too far down becomes 0
        asm("v_cvt_i32_f64 %0, %1" : "=v"(i) : "v"(n));
        constexpr double c1 = 6.769015435155716e-4 /* ln 2 / 1024 */, c2 = c1 * c1 / 2, c3 = c1 * c1 * c1 / 6;
        const double p = fma(fma(fma(c3, r, c2), r, c1), r, 1.0);
        const double x = __builtin_amdgcn_ldexp(table[i & (kTable - 1)] * p, (i >> 10) + bits);
        const u64 w = (u64)__double_as_longlong(x + 0x1p52) & 0xfffffffffffffull;
        return v == top ? 1ull << bits : w;     // exactly one, plus infinity among them
    }
    // of those of four tokens that `wanted` has, 0 of the others
    __device__ __forceinline__ void whole4(const float (&l)[4], const bool (&wanted)[4], u64 (&v)[4]) const
    {
        if (__any(wanted[0] || wanted[1] || wanted[2] || wanted[3])) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = whole(l[e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = wanted[e] ? v[e] : 0ull;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = 0ull;
        }
    }
};

typedef uint32_t u32_byte __attribute__((aligned(1)));

// One row as a workgroup sees it.  A token that is masked (what it holds is not looked at), NaN or behind the row is minus infinity.
template <class E, bool HELD>
struct Row {
    const typename E::T* logits;
    const uint8_t* allowed;
    typename E::T* held;
    int V, first, chunks, lane;     // first: of the wave's tokens

    __device__ __forceinline__ int index(int chunk, int e) const { return first + chunk * kChunk + lane * 4 + e; }
    __device__ __forceinline__ float one(int j) const
    {
        if (HELD) return E::load(held + j);
        return j < V ? from_memory(j) : -kInf;
    }
    __device__ __forceinline__ float from_memory(int j) const { return !allowed || allowed[j] ? fmaxf(E::load(logits + j), -kInf) : -kInf; }
    __device__ __forceinline__ void load(int chunk, float (&v)[4]) const
    {
        const int j = index(chunk, 0);
        if (j + 4 <= V) {           // in one access each, wherever the row starts
            load_n<E, 4, true>(logits + j, v);
            if (allowed) {
                const uint32_t mask = *(const u32_byte*)(allowed + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mask >> (8 * e) & 255u ? v[e] : -kInf;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaxf(v[e], -kInf);      // NaN gives way
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = j + e < V ? from_memory(j + e) : -kInf;
        }
    }
    template <class F>
    __device__ __forceinline__ void each_from_memory(F f) const
    {
        for (int c0 = 0; c0 < chunks; c0 += kAhead) {
            float v[kAhead][4];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) load(c0 + i < chunks ? c0 + i : 1 << 21, v[i]);    // (behind every row: nothing is read)
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (c0 + i < chunks) f(c0 + i, v[i]);
        }
    }
    // f(chunk, values) for the wave's tokens in their order
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        if constexpr (HELD) {
            for (int c = 0; c < chunks; ++c) {
                float v[4];
                load_n<E, 4>(held + index(c, 0), v);
                f(c, v);
            }
        } else {
            each_from_memory(f);
        }
    }
};

template <int CTRL>
__device__ __forceinline__ u64 moved(u64 v)     // by register moves between lanes; 0 where none comes from
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xF, 0xF, true);
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 of_lane(u64 v, int lane)
{
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
// Sum over the lanes up to this one; *total: over all (rows of sixteen lanes by shifts of 1, 2, 4 and 8, then the rows)
__device__ __forceinline__ u64 wave_scan(u64 v, u64* total)
{
    v += moved<0x111>(v);
    v += moved<0x112>(v);
    v += moved<0x114>(v);
    v += moved<0x118>(v);
    const u64 r0 = of_lane(v, 15), r1 = r0 + of_lane(v, 31), r2 = r1 + of_lane(v, 47);
    *total = r2 + of_lane(v, 63);
    const int lane = threadIdx.x & 63;
    return v + (lane < 16 ? 0ull : lane < 32 ? r0 : lane < 48 ? r1 : r2);
}
__device__ __forceinline__ u64 wave_total(u64 v)
{
    u64 total;
    wave_scan(v, &total);
    return total;
}
// Sum over the waves in front of this one and over all of them, of a value that every lane of a wave has.  Its barrier is the only
// one: what the next join writes is the other half of `part`, and this half again only behind the next one's barrier.
template <int WAVES>
__device__ __forceinline__ u64 join(u64 v, Shared& sh, int& turn, u64* total)
{
    const int wave = threadIdx.x >> 6;
    u64* const part = sh.part[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    u64 front = 0, all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const u64 p = part[i];
        if (i < wave) front += p;
        all += p;
    }
    *total = all;
    return front;
}

// The first bin from 0 up (DOWN: from the last down) at which base + the sum so far reaches `want`, and the sum in front of it.
// SHARE: `want` comes as a share of the bins' sum and becomes that part of it, at least 1 (the likeliest token always stays).
// Behind a barrier; all threads.  Nobody reads the bins after it.
template <int WAVES, bool MASS, bool DOWN, bool SHARE>
__device__ __forceinline__ void crossing(Shared& sh, int& turn, u64 base, double& want, unsigned* bin, u64* before)
{
    constexpr int kEach = kBins / (64 * WAVES);
    u64 v[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = threadIdx.x * kEach + i, b = DOWN ? kBins - 1 - at : at;
        v[i] = MASS ? sh.mass[b] : sh.count[b];
        sum += v[i];
    }
    u64 mine, total;
    const u64 inside = wave_scan(sum, &mine) - sum;
    u64 front = base + join<WAVES>(mine, sh, turn, &total) + inside;
    if (SHARE) want = fmax(want * (double)total, 1.0);
    if ((double)front < want && (double)(front + sum) >= want) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if ((double)front < want && (double)(front + v[i]) >= want) {
                const int at = threadIdx.x * kEach + i;
                sh.found_bin = DOWN ? kBins - 1 - at : at;
                sh.found_before = front;
            }
            front += v[i];
        }
    }
    __syncthreads();
    *bin = sh.found_bin;
    *before = sh.found_before;
}

// The first token in index order at which the running sum of weight(value, index) exceeds `past`, given each wave's sum over its
// run: found(index, weight) is called by the thread that has it.  All threads.
template <int WAVES, class R, class W, class F>
__device__ __forceinline__ void in_order(const R& row, Shared& sh, int& turn, u64 front, u64 mine, double past, W weight, F found)
{
    if ((double)front <= past && (double)(front + mine) > past && row.lane == 0) {
        sh.border_index = row.first;
        sh.found_bin = row.chunks * kChunk;
        sh.found_before = front;
    }
    __syncthreads();
    const int n = sh.found_bin, share = (n + 64 * WAVES - 1) / (64 * WAVES), j0 = sh.border_index + min(threadIdx.x * share, n);
    const int each = min(share, sh.border_index + n - j0);
    u64 run = sh.found_before, sum = 0, wave_sum, total;
    for (int i = 0; i < each; ++i) sum += weight(row.one(j0 + i), j0 + i);
    const u64 upto = wave_scan(sum, &wave_sum);
    run += join<WAVES>(wave_sum, sh, turn, &total) + upto - sum;
    if ((double)run <= past && (double)(run + sum) > past)
        for (int i = 0; i < each; ++i) {
            const u64 w = weight(row.one(j0 + i), j0 + i);
            if ((double)run <= past && (double)(run + w) > past) found(j0 + i, w);
            run += w;
        }
}

constexpr int kDigitShift[3] = {21, 10, 0};
constexpr unsigned kDigitMask[3] = {2047u, 2047u, 1023u};

// What stays is every token in front of (value, index) in the order, and that token
struct Border {
    float value;
    int index;
    __device__ __forceinline__ bool keeps(float v, int j) const { return v > value || (v == value && j <= index); }
};

// f(value, there) for the wave's tokens that the border keeps, in any order, 64 of them at a time: a border mostly leaves a few
// tokens in every 256, whose weights would cost as much as those of all (one row of 10 000 words 18.1 us so, 256 rows of 32 000
// bf16 with mixed settings 40.9; gathered 16.6 and 34.8).  All lanes call f; `there` says whether a lane has one.
template <class R, class F>
__device__ __forceinline__ void each_kept(const R& row, const Border& border, float* gathered, F f)
{
    int n = 0;
    auto in_order_of_this_wave = []() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    row.each([&](int c, const float (&l)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool mine = border.keeps(l[e], row.index(c, e));
            const u64 all = __ballot(mine);
            if (all == 0) continue;
            if (mine) gathered[n + __popcll(all & ((1ull << row.lane) - 1))] = l[e];
            n += __popcll(all);
            if (n < 64) continue;
            in_order_of_this_wave();
            n -= 64;
            const float v = gathered[n + row.lane];
            in_order_of_this_wave();
            f(v, true);
        }
    });
    if (n == 0) return;
    in_order_of_this_wave();
    const bool there = row.lane < n;
    f(gathered[there ? row.lane : 0], there);
}

template <int WAVES>
__device__ __forceinline__ void clear_bins(Shared& sh)
{
    for (int i = threadIdx.x; i < kBins; i += 64 * WAVES) sh.mass[i] = 0;
}

// The border among the tokens that `old` keeps: the first token at which the sum of their counts or masses reaches `want`
// (MASS: share * the sum of all, at least 1).  Bins and `listed` are zero, a barrier behind, and are left so for the next
// barrier.
template <int WAVES, bool MASS, class R>
__device__ __forceinline__ Border find_border(const R& row, const Weights& w, Shared& sh, int& turn, float bins_per_unit, const Border& old, double want)
{
    constexpr int kThreads = 64 * WAVES;
    const int tid = threadIdx.x;
    auto weight = [&](float v) -> u64 { return MASS ? w.whole(v) : 1ull; };
    // a larger distance never has a smaller bin: difference, product and conversion are monotone (infinity less itself has bin 0)
    auto bin_of = [&](float v) -> unsigned { return (unsigned)fminf(fmaxf((w.top - v) * bins_per_unit, 0.f), (float)(kBins - 1)); };
    if (MASS && old.value > -kInf) {
        each_kept(row, old, sh.gathered[tid >> 6], [&](float v, bool there) {
            const u64 x = weight(v);
            if (there) atomicAdd(&sh.mass[bin_of(v)], x);
        });
    } else {
        row.each([&](int c, const float (&l)[4]) {
            bool mine[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[e] = old.keeps(l[e], row.index(c, e));
            u64 v[4];
            if (MASS) w.whole4(l, mine, v);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (mine[e]) {
                    if (MASS) atomicAdd(&sh.mass[bin_of(l[e])], v[e]);
                    else atomicAdd(&sh.count[bin_of(l[e])], 1u);
                }
        });
    }
    __syncthreads();
    unsigned bin;
    u64 before;
    crossing<WAVES, MASS, false, MASS>(sh, turn, 0, want, &bin, &before);
    clear_bins<WAVES>(sh);
    // the tokens of that bin
    row.each([&](int c, const float (&l)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = row.index(c, e);
            if (bin_of(l[e]) == bin && old.keeps(l[e], j)) {
                const unsigned at = atomicAdd(&sh.listed, 1u);
                if (at < kList) {
                    sh.list_value[at] = l[e];
                    sh.list_index[at] = j;
                    sh.list_weight[at] = weight(l[e]);
                    sh.list_front[at] = before;
                }
            }
        }
    });
    __syncthreads();
    const int listed = (int)min(sh.listed, (unsigned)kList + 1);
    if (listed <= kList) {
        // each against all, several threads to each: the sum in front of it in the order
        const int parts = kThreads / max(listed, 1), i = tid / max(parts, 1), part = tid % max(parts, 1);
        const int step = max(parts, 1), rounds = parts > 0 ? 1 : (listed + kThreads - 1) / kThreads;
        for (int k = 0; k < rounds; ++k) {
            const int me = i + k * kThreads;
            if (me < listed) {
                const float v = sh.list_value[me];
                const int j = sh.list_index[me];
                u64 front = 0;
                for (int o = part; o < listed; o += step) {
                    const float vo = sh.list_value[o];
                    const u64 wo = sh.list_weight[o];
                    front += vo > v || (vo == v && sh.list_index[o] < j) ? wo : 0ull;
                }
                if (front) atomicAdd(&sh.list_front[me], front);
            }
        }
        __syncthreads();
        for (int k = tid; k < listed; k += kThreads) {
            const u64 front = sh.list_front[k];
            if ((double)front < want && (double)(front + sh.list_weight[k]) >= want) {
                sh.border_value = sh.list_value[k];
                sh.border_index = sh.list_index[k];
            }
        }
        if (tid == 0) sh.listed = 0;            // everybody has read it
        __syncthreads();
        return {sh.border_value, sh.border_index};
    }
    // many: digit by digit of the bit pattern, then by index among equal ones
    uint32_t prefix = 0;
    for (int d = 0; d < 3; ++d) {
        __syncthreads();
        row.each([&](int c, const float (&l)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t k = key_of(l[e]);
                if (bin_of(l[e]) == bin && old.keeps(l[e], row.index(c, e)) && (d == 0 || k >> kDigitShift[d - 1] == prefix >> kDigitShift[d - 1])) {
                    const unsigned b = (k >> kDigitShift[d]) & kDigitMask[d];
                    if (MASS) atomicAdd(&sh.mass[b], weight(l[e]));
                    else atomicAdd(&sh.count[b], 1u);
                }
            }
        });
        __syncthreads();
        unsigned digit;
        crossing<WAVES, MASS, true, false>(sh, turn, before, want, &digit, &before);
        clear_bins<WAVES>(sh);
        prefix |= digit << kDigitShift[d];
    }
    const float value = value_of(prefix);
    const double nth = ceil((want - (double)before) / (double)weight(value));       // 1: the first of the equal ones
    auto equal = [&](float v, int j) -> u64 { return v == value && old.keeps(v, j); };
    u64 count = 0, total;
    row.each([&](int c, const float (&l)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) count += equal(l[e], row.index(c, e));
    });
    const u64 mine = wave_total(count), front = join<WAVES>(mine, sh, turn, &total);
    if (tid == 0) sh.listed = 0;
    int* const at = (int*)sh.list_index;
    in_order<WAVES>(row, sh, turn, front, mine, fmin(nth, (double)total) - 1.0, equal, [&](int j, u64) { at[0] = j; });
    __syncthreads();
    return {value, at[0]};
}

template <class E, int WAVES, bool HELD>
__global__ __launch_bounds__(64 * WAVES) void sample_kernel(SampleArgs a, int bits)
{
    __shared__ Shared sh;
    extern __shared__ __attribute__((aligned(16))) uint8_t held_row[];
    const int m = blockIdx.x, tid = threadIdx.x;
    int turn = 1;                   // part[0] is used here
    Row<E, HELD> row;
    row.held = (typename E::T*)held_row;
    row.logits = (const typename E::T*)a.logits + (int64_t)m * a.ld;
    row.allowed = a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr;
    row.V = a.V;
    row.lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    row.chunks = chunks_of(a.V, WAVES);
    row.first = wave * row.chunks * kChunk;
    const float heat = a.temperature ? a.temperature[m] : 1.f;
    const bool greedy = !(heat > 0.f);
    const int top_k = a.top_k ? a.top_k[m] : 0;
    const double top_p = a.top_p ? (double)a.top_p[m] : 1.0, min_p = a.min_p ? fmin((double)a.min_p[m], 1.0) : 0.0;
    for (int i = tid; i < kTable; i += 64 * WAVES) sh.table[i] = exp2((double)i / kTable);
    clear_bins<WAVES>(sh);
    if (tid == 0) sh.listed = 0;

    // the largest logit, and how many tokens there are
    float best = -kInf;
    int there = 0;
    row.each_from_memory([&](int c, const float (&l)[4]) {
        if (HELD) store_n<E, 4>(row.held + row.index(c, 0), l);     // a value of the type, or minus infinity
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            best = fmaxf(best, l[e]);
            there += __popcll(__ballot(l[e] > -kInf));
        }
    });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) best = fmaxf(best, __shfl_xor(best, off, 64));
    if (row.lane == 0) sh.part[0][wave] = (u64)__float_as_uint(best) << 32 | (unsigned)there;
    __syncthreads();
    int tokens = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const u64 p = sh.part[0][i];
        best = fmaxf(best, __uint_as_float((uint32_t)(p >> 32)));
        tokens += (int)(unsigned)p;
    }
    if (tokens == 0) {
        if (tid == 0) {
            a.token[m] = -1;
            if (a.prob) a.prob[m] = 0.f;
            if (a.kept) a.kept[m] = 0;
        }
        return;
    }
    if (greedy) {
        int first = 0x7fffffff;
        row.each([&](int c, const float (&l)[4]) {
#pragma unroll
            for (int e = 3; e >= 0; --e)
                if (l[e] == best) first = min(first, row.index(c, e));
        });
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) first = min(first, __shfl_xor(first, off, 64));
        if (row.lane == 0) sh.list_index[wave] = first;
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int i = 0; i < WAVES; ++i) first = min(first, sh.list_index[i]);
            a.token[m] = first;
            if (a.prob) a.prob[m] = 1.f;
            if (a.kept) a.kept[m] = 1;
        }
        return;
    }
    Weights w;
    w.table = sh.table;
    w.top = best;
    w.scale = 1024.0 * 1.4426950408889634 / (double)heat;
    w.shift = best == kInf ? -0x1p1000 : -(double)best * w.scale;      // plus infinity: everything else is far below
    w.bits = bits;
    // Masses: 64 bins to a factor of e, over 32 of them; a weight behind that is below 2^-46.  Counts: 64 to a unit of the logit
    // whatever the temperature (by the weights a cold row's last bin held hundreds: 256 rows of 1000 with mixed settings took 31 us).
    constexpr float kCountBins = 64.f;
    const float mass_bins = fminf(64.f / heat, 0x1p100f);

    Border border = {-kInf, -1};    // all
    if (top_k > 0 && top_k < tokens) border = find_border<WAVES, false>(row, w, sh, turn, kCountBins, border, (double)top_k);
    if (top_p < 1.0) border = find_border<WAVES, true>(row, w, sh, turn, mass_bins, border, top_p);

    const u64 least = (u64)ceil(fmax(min_p, 0.0) * (double)(1ull << bits));
    u64 mass = 0, total;
    unsigned kept = 0;
    if (border.value > -kInf) {
        each_kept(row, border, sh.gathered[wave], [&](float v, bool there) {
            const u64 x = w.whole(v);
            const bool stays = there && x >= least;
            mass += stays ? x : 0ull;
            kept += __popcll(__ballot(stays));
        });
    } else {
        row.each([&](int c, const float (&l)[4]) {
            u64 v[4];
            bool keep[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) keep[e] = border.keeps(l[e], row.index(c, e));
            w.whole4(l, keep, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool stays = keep[e] && v[e] >= least;
                mass += stays ? v[e] : 0ull;
                kept += __popcll(__ballot(stays));
            }
        });
    }
    const u64 mine = wave_total(mass);
    if (row.lane == 0) sh.kept[wave] = kept;
    const u64 front = join<WAVES>(mine, sh, turn, &total);
    if (tid == 0 && a.kept) {
        for (int i = 1; i < WAVES; ++i) kept += (unsigned)sh.kept[i];
        a.kept[m] = (int)kept;
    }
    const double want = fmin(fmax((double)a.u[m], 0.0), 0x1.fffffep-1) * (double)total;
    in_order<WAVES>(
        row, sh, turn, front, mine, want,
        [&](float v, int j) -> u64 {
            const u64 x = w.whole(v);
            return border.keeps(v, j) && x >= least ? x : 0ull;
        },
        [&](int j, u64 v) {
            a.token[m] = j;
            if (a.prob) a.prob[m] = (float)((double)v / (double)total);
        });
}

template <class E, int WAVES>
hipError_t sample(const SampleArgs& a, int bits, hipStream_t s)
{
    const size_t held = (size_t)WAVES * chunks_of(a.V, WAVES) * kChunk * E::kBytes;
    if (held > kHeldBytes) {
        hipLaunchKernelGGL((sample_kernel<E, WAVES, false>), dim3(a.M), dim3(64 * WAVES), 0, s, a, bits);
        return hipGetLastError();
    }
    const hipError_t e = allow_dynamic_lds((const void*)sample_kernel<E, WAVES, true>, held);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((sample_kernel<E, WAVES, true>), dim3(a.M), dim3(64 * WAVES), held, s, a, bits);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t s)
{
    int bits = 62;          // V weights of at most 1 stay below 2^62
    for (int v = a.V; v > 1; v = (v + 1) / 2) --bits;
    bits = bits < 51 ? bits : 51;
    // four waves up to 2048 tokens: fewer to wait for at each barrier
    if (a.V <= 2048) return a.bf16 ? sample<Bf16, 4>(a, bits, s) : sample<F32, 4>(a, bits, s);
    return a.bf16 ? sample<Bf16, 16>(a, bits, s) : sample<F32, 16>(a, bits, s);
}

}  // namespace l355
