// C entries of the operators around the cells: the checks of their arguments, in front of anything that reaches the device.
#include "../../include/lstm355.h"
#include "common.h"
#include "lm_ops.h"

#include <cstdio>

using namespace l355;

static_assert(LSTM_SCAN_STEPS == kScanSteps, "");

namespace {

int bad(const char* entry, const char* what)
{
    char msg[256];
    std::snprintf(msg, sizeof msg, "%s: %s", entry, what);
    return op_error(LSTM_ERR_ARG, msg);
}
// Every call that reaches the device goes through here: the runtime allocates on the host, and so does the table of kernels
// with their LDS sizes, and no exception may leave a C entry.
template <class A>
int launched(const char* entry, hipError_t (*launch)(const A&, hipStream_t), const A& a, void* stream) noexcept
{
    char msg[256];
    try {
        const hipError_t e = launch(a, (hipStream_t)stream);
        if (e == hipSuccess) return LSTM_OK;
        std::snprintf(msg, sizeof msg, "%s: %s", entry, hipGetErrorString(e));
        return op_error(e == hipErrorOutOfMemory ? LSTM_ERR_NOMEM : LSTM_ERR_LAUNCH, msg);
    } catch (...) {
        std::snprintf(msg, sizeof msg, "%s: host allocation failed", entry);
        return op_error(LSTM_ERR_NOMEM, msg);
    }
}
int small(const char* entry, size_t got, size_t need)
{
    char msg[256];
    std::snprintf(msg, sizeof msg, "%s: workspace of %zu bytes, %zu are needed", entry, got, need);
    return op_error(LSTM_ERR_NOMEM, msg);
}
bool is_type(int dtype) { return dtype == LSTM_F32 || dtype == LSTM_BF16; }
bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool of_type(const void* p, int dtype) { return aligned(p, dtype == LSTM_BF16 ? 2 : 4); }
bool floats(std::initializer_list<const void*> all)
{
    for (const void* p : all)
        if (!aligned(p, 4)) return false;
    return true;
}
// Offsets are 64 bits wide; a stride beyond 2^40 elements is a mistake and could overflow them.
constexpr int64_t kMaxStride = (int64_t)1 << 40;
bool stride_ok(int64_t s, int64_t least) { return s >= least && s <= kMaxStride; }

// The least that a workspace has to hold.  The product and the draw ask for no more, and touch none of it.
constexpr size_t kLeastWorkspace = 256;

const char kType[] = "unknown dtype", kSize[] = "a size is negative or too large", kNull[] = "a required pointer is NULL";
const char kAlign[] = "a pointer is not aligned to its element type";

int check_scan(const char* entry, int T, int B, int H, int dtype, int reverse, const void* P, int64_t P_t, int64_t P_b, const void* ws,
               size_t ws_bytes)
{
    if (T < 0 || B < 0 || H < 1 || H > (1 << 26) || T > (1 << 30) || !scan_fits(T, B, H)) return bad(entry, kSize);
    if (!is_type(dtype)) return bad(entry, kType);
    if (reverse != 0 && reverse != 1) return bad(entry, "reverse must be 0 or 1");
    if (T > 0 && B > 0 && !P) return bad(entry, kNull);
    if (!stride_ok(P_t, 0) || !stride_ok(P_b, 0)) return bad(entry, "a stride of P is negative or too large");
    if (!of_type(P, dtype)) return bad(entry, kAlign);
    const size_t need = scan_workspace_bytes(T, B, H);
    if (ws_bytes < need) return small(entry, ws_bytes, need);
    if (!ws) return bad(entry, kNull);
    if (!aligned(ws, 16)) return bad(entry, "the workspace is not 16-byte aligned");
    return LSTM_OK;
}
// T x B rows of `width` elements, t and b apart, that must not share any
bool apart(int T, int B, int64_t t, int64_t b, int64_t width)
{
    if (T == 0) return true;
    if (!stride_ok(t, T > 1 ? width : 0) || !stride_ok(b, B > 1 ? width : 0)) return false;
    if (T == 1 || B == 1) return true;
    // i rows along the fewer ones are as far as j along the others and `rest` elements: rows meet where that is within a row of
    // j or of j + 1 of them.  Where one dimension lies within a step of the other this ends at its first i.
    const bool steps_fewer = T < B;
    const int64_t few = steps_fewer ? T : B, many = steps_fewer ? B : T, s_few = steps_fewer ? t : b, s_many = steps_fewer ? b : t;
    if (s_many >= (few - 1) * (__int128)s_few + width) return true;
    int64_t j = 0, rest = 0;
    for (int64_t i = 1; i < few; ++i) {
        j += s_few / s_many;
        rest += s_few % s_many;
        if (rest >= s_many) {
            rest -= s_many;
            ++j;
        }
        if (j >= many) break;
        if (rest < width || (j + 1 < many && s_many - rest < width)) return false;
    }
    return true;
}
// a matrix of `cols` columns: NULL is fine
bool matrix_ok(const void* p, int64_t ld, int rows, int cols, int dtype)
{
    return !p || (of_type(p, dtype) && stride_ok(ld, rows > 1 ? cols : 0));
}
bool eight_bits_ok(const void* p, int64_t ld, int cols) { return aligned(p, 16) && ld % 16 == 0 && stride_ok(ld, cols); }
int blocks_of(int n) { return (n + kScaleCols - 1) / kScaleCols; }

}  // namespace

extern "C" {

size_t lstm_scan_workspace_bytes(int T, int B, int H)
{
    return T < 0 || B < 0 || H < 1 || H > (1 << 26) || T > (1 << 30) || !scan_fits(T, B, H) ? 0 : scan_workspace_bytes(T, B, H);
}

int lstm_scan_forward(int T, int B, int H, int dtype, int reverse, const void* P, int64_t P_t, int64_t P_b,
                      const int32_t* lengths, const float* c0, void* h, int64_t h_t, int64_t h_b, float* cT, float* states,
                      void* workspace, size_t workspace_bytes, void* stream)
{
    static const char entry[] = "lstm_scan_forward";
    if (const int rc = check_scan(entry, T, B, H, dtype, reverse, P, P_t, P_b, workspace, workspace_bytes)) return rc;
    if (B == 0) return LSTM_OK;
    if (T > 0 && !h) return bad(entry, kNull);
    if (!apart(T, B, h_t, h_b, H)) return bad(entry, "rows of h overlap");
    if (!of_type(h, dtype) || !floats({lengths, c0, cT, states})) return bad(entry, kAlign);
    ScanArgs a = {};
    a.T = T; a.B = B; a.H = H; a.bf16 = dtype == LSTM_BF16; a.reverse = reverse;
    a.P = P; a.P_t = P_t; a.P_b = P_b; a.lengths = lengths; a.c0 = c0;
    a.h = h; a.h_t = h_t; a.h_b = h_b; a.cT = cT; a.states = states; a.ws = (float*)workspace;
    return launched(entry, launch_scan_forward, a, stream);
}

int lstm_scan_backward(int T, int B, int H, int dtype, int reverse, const void* P, int64_t P_t, int64_t P_b,
                       const int32_t* lengths, const float* states, const void* dh, int64_t dh_t, int64_t dh_b,
                       const float* dcT, void* dP, int64_t dP_t, int64_t dP_b, float* dc0, void* workspace,
                       size_t workspace_bytes, void* stream)
{
    static const char entry[] = "lstm_scan_backward";
    if (const int rc = check_scan(entry, T, B, H, dtype, reverse, P, P_t, P_b, workspace, workspace_bytes)) return rc;
    if (B == 0) return LSTM_OK;
    if (T > 0 && (!states || !dh || !dP)) return bad(entry, kNull);
    if (!stride_ok(dh_t, 0) || !stride_ok(dh_b, 0)) return bad(entry, "a stride of dh is negative or too large");
    if (!apart(T, B, dP_t, dP_b, 4 * (int64_t)H)) return bad(entry, "rows of dP overlap");
    if (!of_type(dh, dtype) || !of_type(dP, dtype) || !floats({lengths, states, dcT, dc0})) return bad(entry, kAlign);
    ScanArgs a = {};
    a.T = T; a.B = B; a.H = H; a.bf16 = dtype == LSTM_BF16; a.reverse = reverse;
    a.P = P; a.P_t = P_t; a.P_b = P_b; a.lengths = lengths; a.states = const_cast<float*>(states);
    a.dh = dh; a.dh_t = dh_t; a.dh_b = dh_b; a.dcT = dcT;
    a.dP = dP; a.dP_t = dP_t; a.dP_b = dP_b; a.dc0 = dc0; a.ws = (float*)workspace;
    return launched(entry, launch_scan_backward, a, stream);
}

int lstm_rmsnorm_forward(int M, int N, int dtype, const void* x, int64_t x_ld, const void* residual, int64_t residual_ld,
                         const float* weight, float eps, void* sum, int64_t sum_ld, void* y, int64_t y_ld, uint8_t* y8,
                         int64_t y8_ld, float* y8_scale, int64_t y8_scale_ld, float* rstd, void* stream)
{
    static const char entry[] = "lstm_rmsnorm_forward";
    if (M < 0 || M >= (1 << 24) || N < 1) return bad(entry, kSize);
    if (N > kNormMaxCols) return bad(entry, "rows of more than 16384 columns");
    if (!is_type(dtype)) return bad(entry, kType);
    if (!(eps >= 0.f)) return bad(entry, "eps must be >= 0");
    if (M == 0) return LSTM_OK;
    if (!x || !y8 != !y8_scale) return bad(entry, kNull);
    if (!matrix_ok(x, x_ld, M, N, dtype) || !matrix_ok(residual, residual_ld, M, N, dtype) || !matrix_ok(sum, sum_ld, M, N, dtype) ||
        !matrix_ok(y, y_ld, M, N, dtype) || !floats({weight, y8_scale, rstd}))
        return bad(entry, "rows overlap, or a pointer is not aligned to its element type");
    if (y8 && !eight_bits_ok(y8, y8_ld, N)) return bad(entry, "y8 must be 16-byte aligned, with y8_ld a multiple of 16 and at least N");
    if (y8 && !stride_ok(y8_scale_ld, blocks_of(N))) return bad(entry, "rows of y8_scale overlap");
    const NormArgs a = {M, N, dtype == LSTM_BF16, x, x_ld, residual, residual_ld, weight, eps, sum, sum_ld, y, y_ld, y8, y8_ld, y8_scale, y8_scale_ld, rstd};
    return launched(entry, launch_rmsnorm_forward, a, stream);
}

size_t lstm_rmsnorm_workspace_bytes(int M, int N)
{
    return M < 0 || M >= (1 << 24) || N < 1 || N > kNormMaxCols ? 0 : std::max(kLeastWorkspace, rmsnorm_workspace_bytes(M, N));
}

int lstm_rmsnorm_backward(int M, int N, int dtype, const void* sum, int64_t sum_ld, const float* weight, const float* rstd,
                          const void* dy, int64_t dy_ld, const void* dsum, int64_t dsum_ld, void* dx, int64_t dx_ld,
                          float* dweight, void* workspace, size_t workspace_bytes, void* stream)
{
    static const char entry[] = "lstm_rmsnorm_backward";
    if (M < 0 || M >= (1 << 24) || N < 1) return bad(entry, kSize);
    if (N > kNormMaxCols) return bad(entry, "rows of more than 16384 columns");
    if (!is_type(dtype)) return bad(entry, kType);
    if (M > 0 && (!sum || !rstd || !dy || !dx)) return bad(entry, kNull);
    if (!matrix_ok(sum, sum_ld, M, N, dtype) || !matrix_ok(dy, dy_ld, M, N, dtype) || !matrix_ok(dsum, dsum_ld, M, N, dtype) ||
        !matrix_ok(dx, dx_ld, M, N, dtype) || !floats({weight, rstd, dweight}))
        return bad(entry, "rows overlap, or a pointer is not aligned to its element type");
    const size_t need = lstm_rmsnorm_workspace_bytes(M, N);
    if (workspace_bytes < need) return small(entry, workspace_bytes, need);
    if (!workspace) return bad(entry, kNull);
    if (!aligned(workspace, 16)) return bad(entry, "the workspace is not 16-byte aligned");
    if (M == 0 && !dweight) return LSTM_OK;
    const NormGradArgs a = {M, N, dtype == LSTM_BF16, sum, sum_ld, weight, rstd, dy, dy_ld, dsum, dsum_ld, dx, dx_ld, dweight, (float*)workspace};
    return launched(entry, launch_rmsnorm_backward, a, stream);
}

int lstm_quantize_fp8(int M, int N, int dtype, int block_rows, const void* x, int64_t x_ld, uint8_t* q, int64_t q_ld,
                      float* scale, int64_t scale_ld, void* stream)
{
    static const char entry[] = "lstm_quantize_fp8";
    // four waves of 512 columns to a workgroup, whose threads have to stay under 2^32
    if (M < 0 || N < 0 || N > (1 << 30) || (int64_t)M * ((N + 511) / 512) >= ((int64_t)1 << 26)) return bad(entry, kSize);
    if (!is_type(dtype)) return bad(entry, kType);
    if (block_rows != 1 && block_rows != 128) return bad(entry, "block_rows must be 1 or 128");
    if (M == 0 || N == 0) return LSTM_OK;
    if (!x || !q || !scale) return bad(entry, kNull);
    if (!matrix_ok(x, x_ld, M, N, dtype) || !floats({scale})) return bad(entry, "rows overlap, or a pointer is not aligned to its element type");
    if (!eight_bits_ok(q, q_ld, N)) return bad(entry, "q must be 16-byte aligned, with q_ld a multiple of 16 and at least N");
    if (!stride_ok(scale_ld, blocks_of(N))) return bad(entry, "rows of scale overlap");
    const QuantizeArgs a = {M, N, dtype == LSTM_BF16, block_rows, x, x_ld, q, q_ld, scale, scale_ld};
    return launched(entry, launch_quantize_fp8, a, stream);
}

static bool product_fits(int M, int N, int K)
{
    // tiles of 16 by 64 to a workgroup, whose threads have to stay under 2^32
    return M >= 0 && N >= 0 && K >= 0 && M <= (1 << 24) && N <= (1 << 24) && K <= (1 << 30) &&
           (int64_t)((M + 63) / 64) * ((N + 15) / 16) < (1 << 24);
}

size_t lstm_matmul_fp8_workspace_bytes(int M, int N, int K)
{
    return product_fits(M, N, K) ? kLeastWorkspace : 0;
}

int lstm_matmul_fp8(int M, int N, int K, const uint8_t* A, int64_t a_ld, const float* a_scale, int64_t a_scale_ld,
                    const uint8_t* W, int64_t w_ld, const float* w_scale, int64_t w_scale_ld, int w_block_rows,
                    const float* bias, int out_dtype, void* C, int64_t c_ld, void* workspace, size_t workspace_bytes,
                    void* stream)
{
    static const char entry[] = "lstm_matmul_fp8";
    if (!product_fits(M, N, K)) return bad(entry, kSize);
    if (!is_type(out_dtype)) return bad(entry, kType);
    if (w_block_rows != 1 && w_block_rows != 128) return bad(entry, "w_block_rows must be 1 or 128");
    if (M == 0 || N == 0) return LSTM_OK;
    if (!C || (K > 0 && (!A || !a_scale || !W || !w_scale))) return bad(entry, kNull);
    if (K > 0 && (!eight_bits_ok(A, a_ld, K) || !eight_bits_ok(W, w_ld, K)))
        return bad(entry, "A and W must be 16-byte aligned, with a_ld and w_ld multiples of 16 and at least K");
    if (K > 0 && (!stride_ok(a_scale_ld, blocks_of(K)) || !stride_ok(w_scale_ld, blocks_of(K)))) return bad(entry, "rows of scales overlap");
    if (!matrix_ok(C, c_ld, M, N, out_dtype) || !floats({a_scale, w_scale, bias}))
        return bad(entry, "rows overlap, or a pointer is not aligned to its element type");
    const size_t need = lstm_matmul_fp8_workspace_bytes(M, N, K);
    if (workspace_bytes < need) return small(entry, workspace_bytes, need);
    if (!workspace) return bad(entry, kNull);
    if (!aligned(workspace, 16)) return bad(entry, "the workspace is not 16-byte aligned");
    const MatmulFp8Args a = {M, N, K, w_block_rows, out_dtype == LSTM_BF16, A, a_ld, a_scale, a_scale_ld, W, w_ld, w_scale, w_scale_ld, bias, C, c_ld};
    return launched(entry, launch_matmul_fp8, a, stream);
}

static bool sample_fits(int M, int V) { return M >= 0 && M < (1 << 22) && V >= 1 && V <= kSampleMaxVocabulary; }

size_t lstm_sample_workspace_bytes(int M, int V) { return sample_fits(M, V) ? kLeastWorkspace : 0; }

int lstm_sample(int M, int V, int dtype, const void* logits, int64_t ld, const uint8_t* allowed, int64_t allowed_ld,
                const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                int32_t* token, float* prob, int32_t* kept, void* workspace, size_t workspace_bytes, void* stream)
{
    static const char entry[] = "lstm_sample";
    if (!sample_fits(M, V)) return bad(entry, "M outside 0 .. 2^22 - 1, or V outside 1 .. 2^20");
    if (!is_type(dtype)) return bad(entry, kType);
    if (M == 0) return LSTM_OK;
    if (!logits || !u || !token) return bad(entry, kNull);
    if (!matrix_ok(logits, ld, M, V, dtype) || !floats({temperature, top_k, top_p, min_p, u, token, prob, kept}))
        return bad(entry, "rows overlap, or a pointer is not aligned to its element type");
    if (allowed && allowed_ld != 0 && !stride_ok(allowed_ld, V)) return bad(entry, "allowed_ld must be 0 or at least V");
    const size_t need = lstm_sample_workspace_bytes(M, V);
    if (workspace_bytes < need) return small(entry, workspace_bytes, need);
    if (!workspace) return bad(entry, kNull);
    if (!aligned(workspace, 16)) return bad(entry, "the workspace is not 16-byte aligned");
    const SampleArgs a = {M, V, dtype == LSTM_BF16, logits, ld, allowed, allowed_ld, temperature, top_k, top_p, min_p, u, token, prob, kept};
    return launched(entry, launch_sample, a, stream);
}

}  // extern "C"
