// Gated linear recurrence: the cell of the paper's Section 4 with gates that read the input only (no W_h), so that the
// recurrence is linear in the state and time can be cut into pieces:
//
//     c_t = f_t c_{t-1} + i_t g_t          a run of steps maps the state in front of it to  A c + S,  A = prod f
//     h_t = o_t tanh(c_t)
//     gradient: e_t = f_t delta_t (what reaches c_{t-1}),  delta_t = dh_t o_t (1 - tanh^2 c_t) + e_{t+1}
//               a run of steps maps the e behind it to  A e + U  with the same A
//
// One thread takes kScanSteps consecutive steps of one or two neighbouring units with all of their pre-activations in
// registers; the waves of a workgroup take consecutive runs of steps of the same units (a tile), pass (A, S) through LDS and
// go on to the next tile with the state in registers.  Where batch and width alone give too few workgroups, time is also cut
// into segments: a first launch leaves every segment's (A, S) in the workspace, the second starts each segment from the
// product of those in front of it.
#include "device_math.h"
#include "elem.h"
#include "lm_ops.h"

#include <algorithm>

namespace l355 {

namespace {

constexpr int kScanWaves = 4;                               // waves of a workgroup
constexpr int kTileSteps = kScanSteps * kScanWaves;         // steps of a tile
constexpr int kScanTarget = 1024;                           // workgroups aimed at: four on each compute unit

// What one workgroup works on, the same in all of its threads but for the unit
struct Place {
    int b, seg, len, unit;      // unit: first of the thread's, clamped into the layer
    bool live;                  // the thread's units exist
    int tile0, tile1;           // tiles of the segment
};

template <int UPT>
__device__ __forceinline__ Place place_of(const ScanArgs& a, int groups, int tiles, int tiles_per_seg)
{
    Place p;
    const unsigned blk = blockIdx.x, per_b = (unsigned)groups;
    const unsigned g = blk % per_b, rest = blk / per_b;
    p.b = (int)(rest % (unsigned)a.B);
    p.seg = (int)(rest / (unsigned)a.B);
    p.len = a.lengths ? min(max(a.lengths[p.b], 0), a.T) : a.T;
    const int unit = (int)(g * 64 + (threadIdx.x & 63)) * UPT;
    p.live = unit < a.H;
    p.unit = p.live ? unit : a.H - UPT;
    p.tile0 = p.seg * tiles_per_seg;
    p.tile1 = min(p.tile0 + tiles_per_seg, tiles);
    return p;
}

// position in memory of step s < len
__device__ __forceinline__ int64_t at_step(const ScanArgs& a, int len, int s) { return a.reverse ? len - 1 - s : s; }

// State in front of a segment, or gradient behind it: the (A, S) of the segments in between applied to `v`.
// ws: [segments][B][H][2]
template <int UPT>
__device__ __forceinline__ void through_segments(const ScanArgs& a, const Place& p, int from, int to, int step, float (&v)[UPT])
{
    for (int s = from; s != to; s += step) {
        const float* const w = a.ws + (((int64_t)s * a.B + p.b) * a.H + p.unit) * 2;
#pragma unroll
        for (int u = 0; u < UPT; ++u) v[u] = fmaf(w[2 * u], v[u], w[2 * u + 1]);
    }
}

// SUMMARY: only the segment's (A, S), into the workspace.
template <class E, int UPT, bool SUMMARY>
__global__ __launch_bounds__(64 * kScanWaves) void scan_forward_kernel(ScanArgs a, int groups, int tiles, int tiles_per_seg)
{
    __shared__ float run_a[2][kScanWaves][64 * UPT], run_s[2][kScanWaves][64 * UPT];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Place p = place_of<UPT>(a, groups, tiles, tiles_per_seg);
    const typename E::T* const P = (const typename E::T*)a.P + (int64_t)p.b * a.P_b + p.unit;
    typename E::T* const h = (typename E::T*)a.h + (int64_t)p.b * a.h_b + p.unit;
    float carry[UPT], whole[UPT];
#pragma unroll
    for (int u = 0; u < UPT; ++u) {
        carry[u] = !SUMMARY && a.c0 ? a.c0[(int64_t)p.b * a.H + p.unit + u] : 0.f;
        whole[u] = 1.f;
    }
    if (!SUMMARY) through_segments<UPT>(a, p, 0, p.seg, 1, carry);
    int turn = 0;
    for (int tile = p.tile0; tile < p.tile1; ++tile, turn ^= 1) {
        const int s0 = tile * kTileSteps + wave * kScanSteps;
        float f[kScanSteps][UPT], b[kScanSteps][UPT], o[kScanSteps][UPT];
        const bool any = s0 < p.len;
        if (any) {
#pragma unroll
            for (int j = 0; j < kScanSteps; ++j) {     // steps behind the end read the last one again: no branch between loads
                const typename E::T* const q = P + at_step(a, p.len, min(s0 + j, p.len - 1)) * a.P_t;
                float i[UPT], g[UPT];
                load_n<E, UPT>(q, f[j]);
                load_n<E, UPT>(q + a.H, i);
                if (!SUMMARY) load_n<E, UPT>(q + 2 * (int64_t)a.H, o[j]);
                load_n<E, UPT>(q + 3 * (int64_t)a.H, g);
                const bool on = s0 + j < p.len;
#pragma unroll
                for (int u = 0; u < UPT; ++u) {
                    f[j][u] = on ? sigmoidf_fast(f[j][u]) : 1.f;
                    b[j][u] = on ? sigmoidf_fast(i[u]) * tanhf_exact(g[u]) : 0.f;
                }
            }
        }
        float A[UPT], S[UPT];
#pragma unroll
        for (int u = 0; u < UPT; ++u) {
            A[u] = 1.f;
            S[u] = 0.f;
        }
        if (any) {
#pragma unroll
            for (int j = 0; j < kScanSteps; ++j)
#pragma unroll
                for (int u = 0; u < UPT; ++u) {
                    S[u] = fmaf(f[j][u], S[u], b[j][u]);
                    A[u] *= f[j][u];
                }
        }
#pragma unroll
        for (int u = 0; u < UPT; ++u) {
            run_a[turn][wave][u * 64 + lane] = A[u];
            run_s[turn][wave][u * 64 + lane] = S[u];
        }
        __syncthreads();        // one is enough: the other buffer is written next, and everybody has read it in front of this one
        float in[UPT];
#pragma unroll
        for (int w = 0; w < kScanWaves; ++w)
#pragma unroll
            for (int u = 0; u < UPT; ++u) {
                if (w == wave) in[u] = carry[u];
                carry[u] = fmaf(run_a[turn][w][u * 64 + lane], carry[u], run_s[turn][w][u * 64 + lane]);
                if (SUMMARY) whole[u] *= run_a[turn][w][u * 64 + lane];
            }
        if (SUMMARY) continue;
        if (a.states && s0 < a.T && p.live)
#pragma unroll
            for (int u = 0; u < UPT; ++u)
                a.states[((int64_t)(s0 / kScanSteps) * a.B + p.b) * a.H + p.unit + u] = in[u];
#pragma unroll
        for (int j = 0; j < kScanSteps; ++j) {
            const int s = s0 + j;
            if (s >= a.T) break;
            float out[UPT];
            const bool on = s < p.len;
#pragma unroll
            for (int u = 0; u < UPT; ++u) {
                out[u] = 0.f;
                if (on) {
                    in[u] = fmaf(f[j][u], in[u], b[j][u]);
                    out[u] = sigmoidf_fast(o[j][u]) * tanhf_exact(in[u]);
                }
            }
            if (p.live) store_n<E, UPT>(h + (on ? at_step(a, p.len, s) : (int64_t)s) * a.h_t, out);
        }
    }
    if (wave != 0 || !p.live) return;
#pragma unroll
    for (int u = 0; u < UPT; ++u) {
        if (SUMMARY) {
            float* const w = a.ws + (((int64_t)p.seg * a.B + p.b) * a.H + p.unit + u) * 2;
            w[0] = whole[u];
            w[1] = carry[u];
        } else if (a.cT && p.tile1 == tiles) {
            a.cT[(int64_t)p.b * a.H + p.unit + u] = carry[u];
        }
    }
}

// Gradient: tiles from the last to the first.  The states inside a run of kScanSteps steps are computed again from the one
// the forward kept in front of it.
template <class E, bool SUMMARY>
__global__ __launch_bounds__(64 * kScanWaves) void scan_backward_kernel(ScanArgs a, int groups, int tiles, int tiles_per_seg, int segs)
{
    __shared__ float run_a[2][kScanWaves][64], run_s[2][kScanWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Place p = place_of<1>(a, groups, tiles, tiles_per_seg);
    const typename E::T* const P = (const typename E::T*)a.P + (int64_t)p.b * a.P_b + p.unit;
    const typename E::T* const dh = (const typename E::T*)a.dh + (int64_t)p.b * a.dh_b + p.unit;
    typename E::T* const dP = (typename E::T*)a.dP + (int64_t)p.b * a.dP_b + p.unit;
    const int64_t H = a.H;
    float carry[1] = {!SUMMARY && a.dcT ? a.dcT[(int64_t)p.b * a.H + p.unit] : 0.f}, whole = 1.f;
    if (!SUMMARY) through_segments<1>(a, p, segs - 1, p.seg, -1, carry);
    int turn = 0;
    for (int tile = p.tile1 - 1; tile >= p.tile0; --tile, turn ^= 1) {
        const int s0 = tile * kTileSteps + wave * kScanSteps;
        float f[kScanSteps], i[kScanSteps], o[kScanSteps], g[kScanSteps], d[kScanSteps], c[kScanSteps];
        const bool any = s0 < p.len;
        float A = 1.f, U = 0.f;
        if (any) {
            float state = a.states[((int64_t)(s0 / kScanSteps) * a.B + p.b) * H + p.unit];
#pragma unroll
            for (int j = 0; j < kScanSteps; ++j) {
                const int64_t pos = at_step(a, p.len, min(s0 + j, p.len - 1));
                const typename E::T* const q = P + pos * a.P_t;
                f[j] = E::load(q);
                i[j] = E::load(q + H);
                o[j] = E::load(q + 2 * H);
                g[j] = E::load(q + 3 * H);
                d[j] = E::load(dh + pos * a.dh_t);
            }
#pragma unroll
            for (int j = 0; j < kScanSteps; ++j) {
                f[j] = sigmoidf_fast(f[j]);
                i[j] = sigmoidf_fast(i[j]);
                o[j] = sigmoidf_fast(o[j]);
                g[j] = tanhf_exact(g[j]);
                c[j] = state;       // in front of the step
                state = fmaf(f[j], state, i[j] * g[j]);
            }
#pragma unroll
            for (int j = kScanSteps - 1; j >= 0; --j) {
                if (s0 + j < p.len) {
                    const float t = tanhf_exact(fmaf(f[j], c[j], i[j] * g[j]));
                    U = f[j] * fmaf(d[j] * o[j], fmaf(-t, t, 1.f), U);
                    A *= f[j];
                }
            }
        }
        run_a[turn][wave][lane] = A;
        run_s[turn][wave][lane] = U;
        __syncthreads();
        float e = 0.f;
#pragma unroll
        for (int w = kScanWaves - 1; w >= 0; --w) {
            if (w == wave) e = carry[0];
            carry[0] = fmaf(run_a[turn][w][lane], carry[0], run_s[turn][w][lane]);
            if (SUMMARY) whole *= run_a[turn][w][lane];
        }
        if (SUMMARY) continue;
#pragma unroll
        for (int j = kScanSteps - 1; j >= 0; --j) {
            const int s = s0 + j;
            if (s >= a.T) continue;
            float df = 0.f, di = 0.f, dout = 0.f, dg = 0.f;
            const bool on = s < p.len;
            if (on) {
                const float t = tanhf_exact(fmaf(f[j], c[j], i[j] * g[j]));
                const float delta = fmaf(d[j] * o[j], fmaf(-t, t, 1.f), e);
                e = f[j] * delta;
                df = e * c[j] * (1.f - f[j]);
                di = delta * g[j] * i[j] * (1.f - i[j]);
                dout = d[j] * t * o[j] * (1.f - o[j]);
                dg = delta * i[j] * fmaf(-g[j], g[j], 1.f);
            }
            if (p.live) {
                typename E::T* const q = dP + (on ? at_step(a, p.len, s) : (int64_t)s) * a.dP_t;
                E::store(q, df);
                E::store(q + H, di);
                E::store(q + 2 * H, dout);
                E::store(q + 3 * H, dg);
            }
        }
    }
    if (wave != 0 || !p.live) return;
    if (SUMMARY) {
        float* const w = a.ws + (((int64_t)p.seg * a.B + p.b) * H + p.unit) * 2;
        w[0] = whole;
        w[1] = carry[0];
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
// How a layer of `H` units with `upt` of them per thread is cut
Cut cut_of(int T, int B, int H, int upt)
{
    Cut c;
    c.groups = (H + 64 * upt - 1) / (64 * upt);
    c.tiles = (T + kTileSteps - 1) / kTileSteps;
    const int64_t wgs = std::max<int64_t>(1, (int64_t)c.groups * B);
    int segs = (int)std::min<int64_t>(std::max<int64_t>(1, kScanTarget / wgs), std::max(1, c.tiles));
    c.per_seg = std::max(1, (c.tiles + segs - 1) / segs);
    c.segs = std::max(1, (c.tiles + c.per_seg - 1) / c.per_seg);
    return c;
}

}  // namespace

// the larger of the two cuts: one or two units per thread
size_t scan_workspace_bytes(int T, int B, int H)
{
    const int segs = std::max(cut_of(T, B, H, 1).segs, cut_of(T, B, H, 2).segs);
    return segs < 2 ? 256 : (size_t)segs * B * H * 2 * sizeof(float);
}

// a grid's threads have to stay under 2^32
bool scan_fits(int T, int B, int H)
{
    const Cut c = cut_of(T, B, H, 1);
    return (int64_t)c.groups * B * c.segs < (1 << 24);
}

template <class E, int UPT>
static void forward(const ScanArgs& a, hipStream_t s)
{
    const Cut c = cut_of(a.T, a.B, a.H, UPT);
    const dim3 grid((unsigned)c.groups * a.B * c.segs), block(64 * kScanWaves);
    if (c.segs > 1) hipLaunchKernelGGL((scan_forward_kernel<E, UPT, true>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg);
    hipLaunchKernelGGL((scan_forward_kernel<E, UPT, false>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg);
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
    const Cut c = cut_of(a.T, a.B, a.H, 1);
    const dim3 grid((unsigned)c.groups * a.B * c.segs), block(64 * kScanWaves);
    if (a.bf16) {
        if (c.segs > 1) hipLaunchKernelGGL((scan_backward_kernel<Bf16, true>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
        hipLaunchKernelGGL((scan_backward_kernel<Bf16, false>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
    } else {
        if (c.segs > 1) hipLaunchKernelGGL((scan_backward_kernel<F32, true>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
        hipLaunchKernelGGL((scan_backward_kernel<F32, false>), grid, block, 0, s, a, c.groups, c.tiles, c.per_seg, c.segs);
    }
    return hipGetLastError();
}

}  // namespace l355
