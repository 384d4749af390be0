// Element types of the operators around the cells: fp32, and bf16 held as 16-bit patterns; conversions and moves of a few
// neighbouring elements.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace l355 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2v __attribute__((ext_vector_type(2)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
// the same moved at the alignment of their elements: one access all the same (the processor's unaligned mode, which the
// compiler relies on for this target)
typedef f32x4v f32x4v_any __attribute__((aligned(4)));
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef u32x2v u32x2v_any __attribute__((aligned(2)));
typedef u32x4v u32x4v_any __attribute__((aligned(2)));

// nearest-even, NaN stays NaN (the instruction's own rounding)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v){lo, hi}, bf16x2));
}
__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

struct F32 {
    using T = float;
    static constexpr int kBytes = 4;
    static __device__ __forceinline__ float load(const T* p) { return *p; }
    static __device__ __forceinline__ void store(T* p, float v) { *p = v; }
    static __device__ __forceinline__ float round(float v) { return v; }
};
struct Bf16 {
    using T = uint16_t;
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ float load(const T* p) { return __uint_as_float((uint32_t)*p << 16); }
    static __device__ __forceinline__ void store(T* p, float v) { *p = to_bf16(v); }
    static __device__ __forceinline__ float round(float v) { return __uint_as_float((uint32_t)to_bf16(v) << 16); }
};

// N neighbouring elements; p is aligned to N elements (at most 16 bytes of them), ANY: to one
template <class E, int N, bool ANY = false>
__device__ __forceinline__ void load_n(const typename E::T* p, float* v)
{
    using std::conditional_t;
    if constexpr (N == 1) {
        v[0] = E::load(p);
    } else if constexpr (E::kBytes == 4) {
        static_assert(N % 4 == 0, "");
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const f32x4v w = *(const conditional_t<ANY, f32x4v_any, f32x4v>*)(p + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = w[j];
        }
    } else if constexpr (N == 2) {
        const uint32_t w = *(const conditional_t<ANY, u32_any, uint32_t>*)p;
        v[0] = bf16_lo(w);
        v[1] = bf16_hi(w);
    } else if constexpr (N == 4) {
        const u32x2v w = *(const conditional_t<ANY, u32x2v_any, u32x2v>*)p;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            v[2 * j] = bf16_lo(w[j]);
            v[2 * j + 1] = bf16_hi(w[j]);
        }
    } else {
        const u32x4v w = *(const conditional_t<ANY, u32x4v_any, u32x4v>*)p;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_lo(w[j]);
            v[2 * j + 1] = bf16_hi(w[j]);
        }
    }
}
template <class E, int N, bool ANY = false>
__device__ __forceinline__ void store_n(typename E::T* p, const float* v)
{
    using std::conditional_t;
    if constexpr (N == 1) {
        E::store(p, v[0]);
    } else if constexpr (E::kBytes == 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) *(conditional_t<ANY, f32x4v_any, f32x4v>*)(p + i) = (f32x4v){v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else if constexpr (N == 2) {
        *(conditional_t<ANY, u32_any, uint32_t>*)p = pack_bf16(v[0], v[1]);
    } else if constexpr (N == 4) {
        *(conditional_t<ANY, u32x2v_any, u32x2v>*)p = (u32x2v){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
        *(conditional_t<ANY, u32x4v_any, u32x4v>*)p = (u32x4v){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
}

// sum / maximum over the 16 lanes of a row of the wavefront, in every lane of it
template <int CTRL>
__device__ __forceinline__ float dpp_move(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float row16_max(float v)
{
    v = fmaxf(v, dpp_move<0xB1>(v));    // neighbour, other pair of the quad, half-row mirror, row mirror
    v = fmaxf(v, dpp_move<0x4E>(v));
    v = fmaxf(v, dpp_move<0x141>(v));
    return fmaxf(v, dpp_move<0x140>(v));
}

}  // namespace l355
