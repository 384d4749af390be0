// Gated linear recurrence: the cell of the paper's Section 4 with gates that read the input only (no W_h), so that the
// recurrence is linear in the state and time can be cut into pieces:
//
//     c_t = f_t c_{t-1} + i_t g_t          a run of steps maps the state in front of it to  A c + S,  A = prod f
//     h_t = o_t tanh(c_t)
//     gradient: e_t = f_t delta_t (what reaches c_{t-1}),  delta_t = dh_t o_t (1 - tanh^2 c_t) + e_{t+1}
//               a run of steps maps the e behind it to  A e + U  with the same A
//
// One thread takes a run of consecutive steps of one or two neighbouring units with their pre-activations in registers;
// the waves of a workgroup take consecutive runs of the same units (a tile), pass (A, S) through LDS and go on to the next
// tile with the state in registers.  Where batch and width alone give too few workgroups, time is also cut into segments: a
// first launch leaves the segments' (A, S) in the workspace, the second starts each segment from the product of those in
// front of it.  The final state may overwrite the first one, and workgroups of the second launch may start when others have
// ended: so the first launch puts the first state into its segment's S, and beside them where the segment that starts from it
// finds it.
#include "device_math.h"
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>
#include <type_traits>

namespace l355 {

namespace {

constexpr int kScanWaves = 4;                       // waves of a workgroup
constexpr int kRun = 8;                             // steps of a thread in the forward pass; the gradient's are kScanSteps
constexpr int kScanTarget = 1024;                   // workgroups aimed at where time is cut: four on each compute unit

// one or two neighbouring elements as loaded
template <class E, int UPT>
using Raw = std::conditional_t<UPT == 2, uint32_t, typename E::T>;
template <class E, int UPT>
__device__ __forceinline__ void unpack(Raw<E, UPT> r, float (&v)[UPT])
{
    if constexpr (UPT == 2) {
        v[0] = bf16_lo(r);
        v[1] = bf16_hi(r);
    } else if constexpr (E::kBytes == 2) {
        v[0] = __uint_as_float((uint32_t)r << 16);
    } else {
        v[0] = r;
    }
}

// What one workgroup works on, the same in all of its threads but for the unit
struct Place {
    int b, seg, len, unit;      // unit: first of the thread's, clamped into the layer
    bool live;                  // the thread's units exist
    int tile0, tile1;           // tiles of the segment
};

template <int UPT>
__device__ __forceinline__ Place place_of(const ScanArgs& a, int groups, int tiles, int tiles_per_seg, int first_seg = 0)
{
    Place p;
    const unsigned blk = blockIdx.x, per_b = (unsigned)groups;
    const unsigned g = blk % per_b, rest = blk / per_b;
    p.b = (int)(rest % (unsigned)a.B);
    p.seg = first_seg + (int)(rest / (unsigned)a.B);
    p.len = a.lengths ? min(max(a.lengths[p.b], 0), a.T) : a.T;
    const int unit = (int)(g * 64 + (threadIdx.x & 63)) * UPT;
    p.live = unit < a.H;
    p.unit = p.live ? unit : a.H - UPT;
    p.tile0 = p.seg * tiles_per_seg;
    p.tile1 = min(p.tile0 + tiles_per_seg, tiles);
    return p;
}

// position in memory of step s < len
__device__ __forceinline__ int at_step(const ScanArgs& a, int len, int s) { return a.reverse ? len - 1 - s : s; }

// (A, S) of a segment.  ws: [segments][B][H][2]
__device__ __forceinline__ float* slot(const ScanArgs& a, const Place& p, int seg, int u) { return a.ws + (((int64_t)seg * a.B + p.b) * a.H + p.unit + u) * 2; }

// A product of forget gates is zero only if one of them is: where it would underflow it stays the smallest number, so that an
// infinite state in front of it (or gradient behind it) stays infinite, as it does step by step, and does not become 0 * infinity.
// What a finite one adds through such a product is below 2^-21.
constexpr float kLeast = 0x1p-149f;
__device__ __forceinline__ float product_of(float a, float b)
{
    const float p = a * b;
    return p == 0.f && a != 0.f && b != 0.f ? kLeast : p;
}
// that of a run, once it has come out as zero
template <int N, class F>
__device__ __forceinline__ float product_of_run(int on, F gate)
{
    bool zero = false;
#pragma unroll
    for (int j = 0; j < N; ++j) zero |= j < on && gate(j) == 0.f;
    return zero ? 0.f : kLeast;
}

// State in front of a segment, or gradient behind it: the (A, S) of `n` segments (first, first + step, ..) applied to `v`.
// Each wave joins a part of them, eight requested at a time (one after the other their loads took longer than the segment);
// the parts meet in LDS.  Called by the whole workgroup.
template <int UPT>
__device__ __forceinline__ void through_segments(const ScanArgs& a, const Place& p, int first, int n, int step, float (&part_a)[kScanWaves][64 * UPT],
                                                 float (&part_s)[kScanWaves][64 * UPT], float (&v)[UPT])
{
    if (n <= 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int k0 = n * wave / kScanWaves, k1 = n * (wave + 1) / kScanWaves;
    float A[UPT], S[UPT];
#pragma unroll
    for (int u = 0; u < UPT; ++u) {
        A[u] = 1.f;
        S[u] = 0.f;
    }
    for (int k = k0; k < k1; k += 8) {
        float w[8][2 * UPT];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float* const q = slot(a, p, first + min(k + i, k1 - 1) * step, 0);
#pragma unroll
            for (int u = 0; u < 2 * UPT; ++u) w[i][u] = q[u];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (k + i >= k1) break;
#pragma unroll
            for (int u = 0; u < UPT; ++u) {
                S[u] = fmaf(w[i][2 * u], S[u], w[i][2 * u + 1]);
                A[u] = product_of(A[u], w[i][2 * u]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < UPT; ++u) {
        part_a[wave][u * 64 + lane] = A[u];
        part_s[wave][u * 64 + lane] = S[u];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kScanWaves; ++w)
#pragma unroll
        for (int u = 0; u < UPT; ++u) v[u] = fmaf(part_a[w][u * 64 + lane], v[u], part_s[w][u * 64 + lane]);
}

// Forward.  The next tile is requested as soon as this one's pre-activations have become gates, so that its way from memory
// is covered by the runs' joining, the second half of the arithmetic and the stores.
// SUMMARY: only the segment's (A, S), into the workspace.
template <class E, int UPT, bool SUMMARY>
__global__ __launch_bounds__(64 * kScanWaves) void scan_forward_kernel(ScanArgs a, int groups, int tiles, int tiles_per_seg, int segs)
{
    using T = typename E::T;
    using R = Raw<E, UPT>;
    constexpr int kTile = kRun * kScanWaves;
    __shared__ float run_a[2][kScanWaves][64 * UPT], run_s[2][kScanWaves][64 * UPT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place p = place_of<UPT>(a, groups, tiles, tiles_per_seg);
    const T* const P = (const T*)a.P + (int64_t)p.b * a.P_b;        // the same in all lanes; a lane adds its unit
    T* const h = (T*)a.h + (int64_t)p.b * a.h_b;
    const int64_t P_step = a.reverse ? -a.P_t : a.P_t, h_step = a.reverse ? -a.h_t : a.h_t;
    float carry[UPT], whole[UPT];
#pragma unroll
    for (int u = 0; u < UPT; ++u) {
        carry[u] = 0.f;
        whole[u] = 1.f;
    }
    if (!SUMMARY && a.c0 && p.seg == 0)
#pragma unroll
        for (int u = 0; u < UPT; ++u) carry[u] = segs > 1 ? slot(a, p, segs - 1, u)[0] : a.c0[(int64_t)p.b * a.H + p.unit + u];
    R pf[kRun], pi[kRun], pg[kRun], po[kRun];
    auto request = [&](int tile) {
        const int s0 = tile * kTile + wave * kRun, on = min(p.len - s0, kRun);
        if (tile >= p.tile1 || on <= 0) return;
        const T* q = P + at_step(a, p.len, s0) * a.P_t;
#pragma unroll
        for (int j = 0; j < kRun; ++j) {               // steps behind the end read the last one again: no branch between loads
            pf[j] = *(const R*)(q + p.unit);
            pi[j] = *(const R*)(q + a.H + p.unit);
            pg[j] = *(const R*)(q + 3 * (int64_t)a.H + p.unit);
            if (!SUMMARY) po[j] = *(const R*)(q + 2 * (int64_t)a.H + p.unit);
            q += j + 1 < on ? P_step : 0;
        }
    };
    request(p.tile0);
    if (!SUMMARY) through_segments<UPT>(a, p, 0, p.seg, 1, run_a[1], run_s[1], carry);
    int turn = 0;
    for (int tile = p.tile0; tile < p.tile1; ++tile, turn ^= 1) {
        const int s0 = tile * kTile + wave * kRun;
        const int on = min(max(p.len - s0, 0), kRun);               // steps of the run that the sequence has
        float f[kRun][UPT], b[kRun][UPT], o[kRun][UPT], A[UPT], S[UPT];
#pragma unroll
        for (int u = 0; u < UPT; ++u) {
            A[u] = 1.f;
            S[u] = 0.f;
        }
        // FULL: a run without a branch, which all but the last of a sequence are
        auto gates = [&](auto full) {
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                if (!decltype(full)::value && j >= on) continue;
                float i[UPT], g[UPT];
                unpack<E, UPT>(pf[j], f[j]);
                unpack<E, UPT>(pi[j], i);
                unpack<E, UPT>(pg[j], g);
                if (!SUMMARY) unpack<E, UPT>(po[j], o[j]);
#pragma unroll
                for (int u = 0; u < UPT; ++u) {
                    f[j][u] = sigmoidf_fast(f[j][u]);
                    b[j][u] = sigmoidf_fast(i[u]) * tanhf_exact(g[u]);
                    if (!SUMMARY) o[j][u] = sigmoidf_fast(o[j][u]);
                    S[u] = fmaf(f[j][u], S[u], b[j][u]);
                    A[u] *= f[j][u];
                }
            }
        };
        if (on == kRun) gates(std::true_type());
        else gates(std::false_type());
#pragma unroll
        for (int u = 0; u < UPT; ++u)
            if (A[u] == 0.f) A[u] = product_of_run<kRun>(on, [&](int j) { return f[j][u]; });
        request(tile + 1);
#pragma unroll
        for (int u = 0; u < UPT; ++u) {
            run_a[turn][wave][u * 64 + lane] = A[u];
            run_s[turn][wave][u * 64 + lane] = S[u];
        }
        // One barrier is enough (the other buffer is written next, and everybody has read it in front of this one), and a bare
        // one: that of __syncthreads() waits for the loads under way too.
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
        float in[UPT];
#pragma unroll
        for (int w = 0; w < kScanWaves; ++w)
#pragma unroll
            for (int u = 0; u < UPT; ++u) {
                if (w == wave) in[u] = carry[u];
                carry[u] = fmaf(run_a[turn][w][u * 64 + lane], carry[u], run_s[turn][w][u * 64 + lane]);
                if (SUMMARY) whole[u] = product_of(whole[u], run_a[turn][w][u * 64 + lane]);
            }
        if (SUMMARY) continue;
        if (a.states && s0 % kScanSteps == 0 && s0 < a.T && p.live)
#pragma unroll
            for (int u = 0; u < UPT; ++u)
                a.states[((int64_t)(s0 / kScanSteps) * a.B + p.b) * a.H + p.unit + u] = in[u];
        auto outputs = [&](auto full) {
            T* q = h + at_step(a, p.len, s0) * a.h_t + p.unit;
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                float out[UPT];
                if (decltype(full)::value || j < on) {
#pragma unroll
                    for (int u = 0; u < UPT; ++u) {
                        in[u] = fmaf(f[j][u], in[u], b[j][u]);
                        out[u] = o[j][u] * tanhf_exact(in[u]);
                    }
                    if (p.live) store_n<E, UPT>(q, out);
                    q += h_step;
                } else if (s0 + j < a.T) {
#pragma unroll
                    for (int u = 0; u < UPT; ++u) out[u] = 0.f;
                    if (p.live) store_n<E, UPT>(h + (s0 + j) * a.h_t + p.unit, out);
                }
            }
        };
        if (on == kRun) outputs(std::true_type());
        else outputs(std::false_type());
    }
    if (wave != 0 || !p.live) return;
#pragma unroll
    for (int u = 0; u < UPT; ++u) {
        if (SUMMARY) {
            float* const w = slot(a, p, p.seg, u);
            if (p.seg == 0 && a.c0) {
                const float c0 = a.c0[(int64_t)p.b * a.H + p.unit + u];
                slot(a, p, segs - 1, u)[0] = c0;            // whose own is not needed
                carry[u] = fmaf(whole[u], c0, carry[u]);
                whole[u] = 0.f;
            }
            w[0] = whole[u];
            w[1] = carry[u];
        } else if (a.cT && p.tile1 == tiles) {
            a.cT[(int64_t)p.b * a.H + p.unit + u] = carry[u];
        }
    }
}

// Gradient: tiles from the last to the first.  The states inside a run of kScanSteps steps are computed again from the one
// the forward kept in front of it.  What does not depend on the gradient behind the run - that of the output gate, and
// dh o (1 - tanh^2 c) - is finished (the first: stored) before the runs are joined, so that five values a step wait in registers.
template <class E, bool SUMMARY>
__global__ __launch_bounds__(64 * kScanWaves) void scan_backward_kernel(ScanArgs a, int groups, int tiles, int tiles_per_seg, int segs)
{
    using T = typename E::T;
    __shared__ float run_a[2][kScanWaves][64], run_s[2][kScanWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place p = place_of<1>(a, groups, tiles, tiles_per_seg, SUMMARY ? 1 : 0);      // nothing precedes segment 0
    const T* const P = (const T*)a.P + (int64_t)p.b * a.P_b;
    const T* const dh = (const T*)a.dh + (int64_t)p.b * a.dh_b;
    T* const dP = (T*)a.dP + (int64_t)p.b * a.dP_b;
    const int64_t H = a.H, P_step = a.reverse ? -a.P_t : a.P_t, dh_step = a.reverse ? -a.dh_t : a.dh_t, dP_step = a.reverse ? -a.dP_t : a.dP_t;
    const bool last = p.seg == segs - 1 && a.dcT;
    float carry[1] = {SUMMARY || !last ? 0.f : segs > 1 ? slot(a, p, 0, 0)[0] : a.dcT[(int64_t)p.b * a.H + p.unit]}, whole = 1.f;
    if (!SUMMARY) through_segments<1>(a, p, segs - 1, segs - 1 - p.seg, -1, run_a[1], run_s[1], carry);
    int turn = 0;
    for (int tile = p.tile1 - 1; tile >= p.tile0; --tile, turn ^= 1) {
        const int s0 = (tile * kScanWaves + wave) * kScanSteps;
        const int on = min(max(p.len - s0, 0), kScanSteps);
        float f[kScanSteps], i[kScanSteps], g[kScanSteps], c[kScanSteps], u[kScanSteps];
        float A = 1.f, U = 0.f;
        // FULL: a run without a branch, which all but the last of a sequence are
        auto load_run = [&](auto full) {
            constexpr bool FULL = decltype(full)::value;
            float o[kScanSteps], d[kScanSteps];
            float state = a.states[((int64_t)(s0 / kScanSteps) * a.B + p.b) * H + p.unit];
            const int first = at_step(a, p.len, s0);
            const T *q = P + first * a.P_t, *r = dh + first * a.dh_t;
#pragma unroll
            for (int j = 0; j < kScanSteps; ++j) {
                f[j] = E::load(q + p.unit);
                i[j] = E::load(q + H + p.unit);
                g[j] = E::load(q + 3 * H + p.unit);
                o[j] = E::load(q + 2 * H + p.unit);
                d[j] = E::load(r + p.unit);
                if (FULL || j + 1 < on) {
                    q += P_step;
                    r += dh_step;
                }
            }
            T* to = dP + first * a.dP_t + 2 * H + p.unit;
#pragma unroll
            for (int j = 0; j < kScanSteps; ++j) {
                if (!FULL && j >= on) continue;
                f[j] = sigmoidf_fast(f[j]);
                i[j] = sigmoidf_fast(i[j]);
                g[j] = tanhf_exact(g[j]);
                c[j] = state;       // in front of the step
                state = fmaf(f[j], state, i[j] * g[j]);
                const float og = sigmoidf_fast(o[j]), t = tanhf_exact(state), through = d[j] * og;
                u[j] = through * fmaf(-t, t, 1.f);
                if (!SUMMARY && p.live) E::store(to, through * t * (1.f - og));
                to += dP_step;
            }
#pragma unroll
            for (int j = kScanSteps - 1; j >= 0; --j) {
                if (!FULL && j >= on) continue;
                U = f[j] * (u[j] + U);
                A *= f[j];
            }
        };
        if (on == kScanSteps) load_run(std::true_type());
        else if (on > 0) load_run(std::false_type());
        if (A == 0.f) A = product_of_run<kScanSteps>(on, [&](int j) { return f[j]; });
        run_a[turn][wave][lane] = A;
        run_s[turn][wave][lane] = U;
        __syncthreads();        // one is enough: the other buffer is written next, and everybody has read it in front of this one
        float e = 0.f;
#pragma unroll
        for (int w = kScanWaves - 1; w >= 0; --w) {
            if (w == wave) e = carry[0];
            carry[0] = fmaf(run_a[turn][w][lane], carry[0], run_s[turn][w][lane]);
            if (SUMMARY) whole = product_of(whole, run_a[turn][w][lane]);
        }
        if (SUMMARY) continue;
        auto store_run = [&](auto full) {
            constexpr bool FULL = decltype(full)::value;
            T* q = dP + at_step(a, p.len, s0 + (FULL ? kScanSteps : on) - 1) * a.dP_t + p.unit;
#pragma unroll
            for (int j = kScanSteps - 1; j >= 0; --j) {
                if (FULL || j < on) {
                    const float delta = u[j] + e, di = delta * i[j];
                    e = f[j] * delta;
                    if (p.live) {
                        E::store(q, e * c[j] * (1.f - f[j]));
                        E::store(q + H, di * g[j] * (1.f - i[j]));
                        E::store(q + 3 * H, di * fmaf(-g[j], g[j], 1.f));
                    }
                    q -= dP_step;
                } else if (s0 + j < a.T && p.live) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) E::store(dP + (s0 + j) * a.dP_t + k * H + p.unit, 0.f);
                }
            }
        };
        if (on == kScanSteps) store_run(std::true_type());
        else store_run(std::false_type());
    }
    if (wave != 0 || !p.live) return;
    if (SUMMARY) {
        float* const w = slot(a, p, p.seg, 0);
        const float dcT = last ? a.dcT[(int64_t)p.b * a.H + p.unit] : 0.f;
        w[0] = last ? 0.f : whole;
        w[1] = fmaf(whole, dcT, carry[0]);
        if (last) slot(a, p, 0, 0)[0] = dcT;                // whose own is not needed
    } else if (a.dc0 && p.seg == 0) {
        a.dc0[(int64_t)p.b * H + p.unit] = carry[0];
    }
}

// One step: a thread per state
template <class E>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a)
{
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= (int64_t)a.B * a.H) return;
    const int b = (int)(n / a.H), unit = (int)(n % a.H);
    const typename E::T* const q = (const typename E::T*)a.P + (int64_t)b * a.P_b + unit;
    const bool on = !a.lengths || a.lengths[b] > 0;
    float c = a.c0 ? a.c0[n] : 0.f, h = 0.f;
    if (a.states) a.states[n] = c;
    if (on) {
        c = fmaf(sigmoidf_fast(E::load(q)), c, sigmoidf_fast(E::load(q + a.H)) * tanhf_exact(E::load(q + 3 * (int64_t)a.H)));
        h = sigmoidf_fast(E::load(q + 2 * (int64_t)a.H)) * tanhf_exact(c);
    }
    E::store((typename E::T*)a.h + (int64_t)b * a.h_b + unit, h);
    if (a.cT) a.cT[n] = c;
}

struct Cut {
    int groups, tiles, per_seg, segs;
};
// How a layer of `H` units with `upt` of them per thread, and tiles of `steps` steps, is cut: not from `whole` workgroups on, nor
// for fewer than `least` tiles.
Cut cut_of(int T, int B, int H, int upt, int steps, int whole, int least)
{
    Cut c;
    c.groups = (H + 64 * upt - 1) / (64 * upt);
    c.tiles = (T + steps - 1) / steps;
    const int64_t wgs = std::max<int64_t>(1, (int64_t)c.groups * B);
    const int segs = wgs >= whole || c.tiles < least ? 1 : (int)std::min<int64_t>(std::max<int64_t>(1, kScanTarget / wgs), std::max(1, c.tiles));
    c.per_seg = std::max(1, (c.tiles + segs - 1) / segs);
    c.segs = std::max(1, (c.tiles + c.per_seg - 1) / c.per_seg);
    return c;
}
// The summaries read three quarters of the pre-activations once more in the forward pass, and everything in the gradient's, so
// cutting pays while a tile is a chain of waits: up to three workgroups for four compute units forward, one for two back; some
// more where sequences have lengths of their own and the longest alone would hold its workgroups.  us without and with the cut at
// 1500 units, fp32, batch 6, 8 and 12 (144, 192, 288 workgroups): forward of 300 steps 27 and 26, 29 and 31, 36 and 45; gradient
// of 1500 steps at batch 4 (96) 165 and 118 to bf16, 121 and 118 to fp32, at batch 6 136 and 177; with lengths, forward of 300
// steps at batch 8 28 and 25, at batch 12 32 and 34, gradient at batch 8 37 and 41.  Of few tiles the second launch costs more
// than it gives (64 steps, batch 1: 5.3 and 6.9).  Of many the chain grows longer, and that of a bf16 sequence has half as
// much to read: us without and with the cut at 188 to 192 workgroups (201 units at batch 47, 1500 at 16) 300 steps 22.5 and 21.6,
// 36.5 and 36.7, 1500 steps 103 and 79, 155 and 131, 4000 steps 266 and 196, 386 and 347; at 208 (1024 at 26) 55.7 and 59.6 for 520
// steps, 144 and 143, 375 and 383; at 240 (1500 at 20) 61 and 66, 156 and 159, 394 and 425.  fp32 at 188 to 192 (201 at 47, 1500 at 8)
// 1500 steps 119 and 110, 123 and 118, 4000 steps 292 and 286, 300 and 326; at 208 (1024 at 13) 113 and 122, 278 and 344; at 240 (1500
// at 10) 128 and 143, 313 and 405.  With lengths, at 240 workgroups (256 at 60, fp32) 300 steps 26.2 and 25.4, 1500 111 and 108.
Cut forward_cut(int T, int B, int H, int upt, bool lengths, bool bf16)
{
    constexpr int kTile = kRun * kScanWaves, kManyTiles = 16;
    return cut_of(T, B, H, upt, kTile, lengths ? 256 : T <= (kManyTiles - 1) * kTile ? 176 : bf16 ? 208 : 192, 4);
}
Cut backward_cut(int T, int B, int H, bool lengths) { return cut_of(T, B, H, 1, kScanSteps * kScanWaves, lengths ? 176 : 128, 3); }

}  // namespace

// the largest of the cuts: one or two units per thread, forward or back, with lengths or without, of either type
size_t scan_workspace_bytes(int T, int B, int H)
{
    int segs = 1;
    for (const bool lengths : {false, true}) {
        segs = std::max(segs, backward_cut(T, B, H, lengths).segs);
        for (const bool bf16 : {false, true})
            for (const int upt : {1, 2}) segs = std::max(segs, forward_cut(T, B, H, upt, lengths, bf16).segs);
    }
    return segs < 2 ? 256 : (size_t)segs * B * H * 2 * sizeof(float);
}

// a grid's threads have to stay under 2^32
bool scan_fits(int T, int B, int H)
{
    const Cut c = forward_cut(T, B, H, 1, true, true);
    return (int64_t)c.groups * B * c.segs < (1 << 24);
}

template <class E, int UPT>
static void forward(const ScanArgs& a, hipStream_t s)
{
    const Cut c = forward_cut(a.T, a.B, a.H, UPT, a.lengths != nullptr, a.bf16);
    const dim3 grid((unsigned)c.groups * a.B * c.segs), block(64 * kScanWaves);
    const dim3 but_last((unsigned)c.groups * a.B * (c.segs - 1));      // nothing follows the last segment
    if (c.segs > 1) hipLaunchKernelGGL((scan_forward_kernel<E, UPT, true>), but_last, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
    hipLaunchKernelGGL((scan_forward_kernel<E, UPT, false>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
}

hipError_t launch_scan_forward(const ScanArgs& a, hipStream_t s)
{
    if (a.T == 1) {
        const dim3 grid((unsigned)(((int64_t)a.B * a.H + 255) / 256)), block(256);
        if (a.bf16) hipLaunchKernelGGL(scan_step_kernel<Bf16>, grid, block, 0, s, a);
        else hipLaunchKernelGGL(scan_step_kernel<F32>, grid, block, 0, s, a);
        return hipGetLastError();
    }
    // two bf16 units per thread where every row of units starts on a word; a layer of up to 64 units fills a wave without
    const bool words = a.bf16 && a.H > 64 && !((a.H | a.P_t | a.P_b | a.h_t | a.h_b) & 1) && !(((uintptr_t)a.P | (uintptr_t)a.h) & 3);
    if (words) forward<Bf16, 2>(a, s);
    else if (a.bf16) forward<Bf16, 1>(a, s);
    else forward<F32, 1>(a, s);
    return hipGetLastError();
}

hipError_t launch_scan_backward(const ScanArgs& a, hipStream_t s)
{
    const Cut c = backward_cut(a.T, a.B, a.H, a.lengths != nullptr);
    const dim3 grid((unsigned)c.groups * a.B * c.segs), but_first((unsigned)c.groups * a.B * (c.segs - 1)), block(64 * kScanWaves);
    if (a.bf16) {
        if (c.segs > 1) hipLaunchKernelGGL((scan_backward_kernel<Bf16, true>), but_first, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
        hipLaunchKernelGGL((scan_backward_kernel<Bf16, false>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
    } else {
        if (c.segs > 1) hipLaunchKernelGGL((scan_backward_kernel<F32, true>), but_first, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
        hipLaunchKernelGGL((scan_backward_kernel<F32, false>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
    }
    return hipGetLastError();
}

}  // namespace l355
