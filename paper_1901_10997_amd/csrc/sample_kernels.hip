// The draw of one token per row of logits from given random numbers: temperature, then the top_k likeliest, then the shortest
// prefix of those that holds top_p of their mass, then those within min_p of the likeliest.
//
//     w_j = exp((l_j - max l) / temperature), as a whole number of 2^-S
//     order: logit descending, index ascending.  Everything that is kept is: keys above a border key, and of the tokens on
//     the border key the first few by index; so a filter is a search for its border, by digits of the logit's bit pattern
//     with a histogram of counts (top_k) or of masses (top_p)
//     token = first index, ascending, at which the running sum over the kept exceeds u times their sum
//
// Weights are evaluated in 64 bits and summed as 64-bit whole numbers: a sum has the same bits in every order, so atomics and
// the cut of the work do not change who is drawn.
#include "elem.h"
#include "lm_ops.h"

namespace l355 {

namespace {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;
constexpr int kBins = 2048;
typedef unsigned long long u64;

// Bits of a value in ascending order; both zeros are one value.  Every number above minus infinity has a key above 0.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// One row as the kernel sees it
template <class E>
struct Row {
    const typename E::T* logits;
    const uint8_t* allowed;
    // key of token j; 0: masked (what it holds is not looked at), NaN or minus infinity
    __device__ __forceinline__ uint32_t key(int j) const
    {
        if (allowed && !allowed[j]) return 0u;
        const float v = E::load(logits + j);
        return v > -__builtin_inff() ? key_of(v) : 0u;
    }
};

struct Weights {
    double top, heat, one;      // largest logit, temperature, the whole number that stands for 1
    uint32_t top_key;
    __device__ __forceinline__ double of(uint32_t key) const
    {
        return key == top_key ? 1.0 : exp(((double)value_of(key) - top) / heat);
    }
    __device__ __forceinline__ u64 whole(uint32_t key) const { return (u64)rint(of(key) * one); }
};

struct Shared {
    union {
        u64 mass[kBins];
        unsigned count[kBins];
    };
    u64 part[kSampleWaves];
    u64 found_before;
    unsigned found_digit;
    int found_index;
};

// Sum over the threads in front of this one, and over all of them
__device__ __forceinline__ u64 scan(u64 v, Shared& sh, u64* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 incl = v;
    for (int off = 1; off < 64; off <<= 1) {
        const u64 up = __shfl_up(incl, off, 64);
        if (lane >= off) incl += up;
    }
    __syncthreads();
    if (lane == 63) sh.part[wave] = incl;
    __syncthreads();
    u64 before = 0, all = 0;
    for (int i = 0; i < kSampleWaves; ++i) {
        if (i < wave) before += sh.part[i];
        all += sh.part[i];
    }
    *total = all;
    return before + incl - v;
}
__device__ __forceinline__ u64 block_max(u64 v, Shared& sh)
{
    for (int off = 32; off >= 1; off >>= 1) {
        const u64 o = __shfl_xor(v, off, 64);
        v = o > v ? o : v;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int i = 0; i < kSampleWaves; ++i) v = sh.part[i] > v ? sh.part[i] : v;
    return v;
}

constexpr int kDigitShift[3] = {21, 10, 0};
constexpr unsigned kDigitMask[3] = {2047u, 2047u, 1023u};

// From the highest bin down, the first at which base + the sum so far reaches `want`: the bin, and the sum in front of it.
// Called by all threads behind a barrier; two bins each.
template <bool MASS>
__device__ __forceinline__ void crossing(Shared& sh, u64 base, double want, unsigned* digit, u64* before)
{
    const int hi = kBins - 1 - 2 * threadIdx.x, lo = hi - 1;
    const u64 a = MASS ? sh.mass[hi] : sh.count[hi], b = MASS ? sh.mass[lo] : sh.count[lo];
    u64 total;
    const u64 front = base + scan(a + b, sh, &total);
    if ((double)front < want && (double)(front + a + b) >= want) {
        const bool first = (double)(front + a) >= want;
        sh.found_digit = first ? hi : lo;
        sh.found_before = first ? front : front + a;
    }
    __syncthreads();
    *digit = sh.found_digit;
    *before = sh.found_before;
    __syncthreads();
}

template <class E>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a, int whole_bits)
{
    __shared__ Shared sh;
    const int m = blockIdx.x, tid = threadIdx.x, V = a.V;
    const Row<E> row = {(const typename E::T*)a.logits + (int64_t)m * a.ld, a.allowed ? a.allowed + (int64_t)m * a.allowed_ld : nullptr};
    const float heat = a.temperature ? a.temperature[m] : 1.f;
    const int top_k = !(heat > 0.f) ? 1 : a.top_k && a.top_k[m] > 0 ? a.top_k[m] : V;
    const double top_p = a.top_p ? (double)a.top_p[m] : 1.0, min_p = a.min_p ? fmin((double)a.min_p[m], 1.0) : 0.0;

    // largest key and how many tokens there are
    uint32_t top = 0;
    unsigned there = 0;
    for (int j = tid; j < V; j += kSampleThreads) {
        const uint32_t k = row.key(j);
        top = max(top, k);
        there += k != 0;
    }
    u64 tokens;
    scan(there, sh, &tokens);
    top = (uint32_t)block_max(top, sh);
    if (tokens == 0) {
        if (tid == 0) {
            a.token[m] = -1;
            if (a.prob) a.prob[m] = 0.f;
            if (a.kept) a.kept[m] = 0;
        }
        return;
    }
    Weights w;
    w.top_key = top;
    w.top = (double)value_of(top);
    w.heat = heat > 0.f ? (double)heat : 1.0;
    w.one = (double)(1ull << whole_bits);

    // kept: key > border, and the first `on_border` tokens of that key
    uint32_t border = 0;
    u64 on_border = 0;
    if ((u64)top_k < tokens) {
        uint32_t prefix = 0;
        u64 before = 0;
        for (int d = 0; d < 3; ++d) {
            for (int i = tid; i < kBins; i += kSampleThreads) sh.count[i] = 0;
            __syncthreads();
            for (int j = tid; j < V; j += kSampleThreads) {
                const uint32_t k = row.key(j);
                if (k && (d == 0 || k >> kDigitShift[d - 1] == prefix >> kDigitShift[d - 1]))
                    atomicAdd(&sh.count[(k >> kDigitShift[d]) & kDigitMask[d]], 1u);
            }
            __syncthreads();
            unsigned digit;
            crossing<false>(sh, before, (double)top_k, &digit, &before);
            prefix |= digit << kDigitShift[d];
        }
        border = prefix;
        on_border = (u64)top_k - before;
    }
    if (top_p < 1.0) {
        uint32_t prefix = 0;
        u64 before = 0;
        double want = 0.0;
        for (int d = 0; d < 3; ++d) {
            for (int i = tid; i < kBins; i += kSampleThreads) sh.mass[i] = 0;
            __syncthreads();
            auto mine = [&](uint32_t k) { return d == 0 || k >> kDigitShift[d - 1] == prefix >> kDigitShift[d - 1]; };
            auto add = [&](uint32_t k, u64 times) { atomicAdd(&sh.mass[(k >> kDigitShift[d]) & kDigitMask[d]], w.whole(k) * times); };
            for (int j = tid; j < V; j += kSampleThreads) {
                const uint32_t k = row.key(j);
                if (k > border && mine(k)) add(k, 1);
            }
            if (tid == 0 && border && mine(border)) add(border, on_border);
            __syncthreads();
            if (d == 0) {
                u64 total;
                scan(sh.mass[2 * tid] + sh.mass[2 * tid + 1], sh, &total);
                want = fmax(top_p * (double)total, 1.0);    // the likeliest token always stays
            }
            unsigned digit;
            crossing<true>(sh, before, want, &digit, &before);
            prefix |= digit << kDigitShift[d];
        }
        const double steps = ceil((want - (double)before) / (double)w.whole(prefix));
        if (prefix != border) on_border = ~0ull;
        on_border = (double)on_border > steps ? (u64)steps : on_border;
        border = prefix;
    }
    // Of the tokens on the border key only the first ones: the index of the last of them.  From here on a thread has a run
    // of neighbouring tokens.
    const int each = (V + kSampleThreads - 1) / kSampleThreads, j0 = min(tid * each, V), j1 = min(j0 + each, V);
    int last = V;
    if (border) {
        u64 equal = 0, all;
        for (int j = j0; j < j1; ++j) equal += row.key(j) == border;
        const u64 front = scan(equal, sh, &all);
        if (all > on_border) {
            if (front < on_border && front + equal >= on_border) {
                u64 n = front;
                for (int j = j0; j < j1; ++j)
                    if (row.key(j) == border && ++n == on_border) sh.found_index = j;
            }
            __syncthreads();
            last = sh.found_index;
            __syncthreads();
        }
    }
    auto kept_weight = [&](int j) -> double {       // below 0: not kept
        const uint32_t k = row.key(j);
        if (k == 0 || k < border || (k == border && j > last)) return -1.0;
        const double v = w.of(k);
        return v >= min_p ? v : -1.0;
    };
    u64 mass = 0, kept = 0, all_kept, total;
    for (int j = j0; j < j1; ++j) {
        const double v = kept_weight(j);
        if (v >= 0.0) {
            mass += (u64)rint(v * w.one);
            ++kept;
        }
    }
    scan(kept, sh, &all_kept);
    const u64 front = scan(mass, sh, &total);
    const double want = fmin(fmax((double)a.u[m], 0.0), 0x1.fffffep-1) * (double)total;
    if ((double)front <= want && (double)(front + mass) > want) {
        u64 run = front;
        for (int j = j0; j < j1; ++j) {
            const double v = kept_weight(j);
            if (v < 0.0) continue;
            run += (u64)rint(v * w.one);
            if ((double)run > want) {
                a.token[m] = j;
                if (a.prob) a.prob[m] = (float)(v * w.one / (double)total);
                break;
            }
        }
    }
    if (tid == 0 && a.kept) a.kept[m] = (int)all_kept;
}

}  // namespace

size_t sample_workspace_bytes(int, int) { return 256; }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s)
{
    int bits = 62;          // V weights of at most 1 stay below 2^62
    for (int v = a.V; v > 1; v = (v + 1) / 2) --bits;
    if (a.bf16) hipLaunchKernelGGL(sample_kernel<Bf16>, dim3(a.M), dim3(kSampleThreads), 0, s, a, bits);
    else hipLaunchKernelGGL(sample_kernel<F32>, dim3(a.M), dim3(kSampleThreads), 0, s, a, bits);
    return hipGetLastError();
}

}  // namespace l355
