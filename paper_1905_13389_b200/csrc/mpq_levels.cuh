// Element types and level decoding shared by the operators of an encoded decoder block.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mpq_common.cuh"

namespace mpq {

inline bool dtype_ok(int d) { return d == MPQ_F32 || d == MPQ_F16 || d == MPQ_BF16; }
inline int dtype_size(int d) { return d == MPQ_F32 ? 4 : 2; }
inline bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

__host__ __device__ inline int64_t level_row_bytes(int64_t k) { return ceil_div(k, 16) * 16; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// N elements that start at an N * sizeof(T)-byte (at most 16-byte) aligned address.
template <typename T, int N>
__device__ __forceinline__ void load_vec(const T* p, float (&f)[N]) {
    constexpr int kBytes = N * (int)sizeof(T);
    if constexpr (N == 1) {
        f[0] = to_f32(*p);
    } else if constexpr (kBytes == 8) {
        const uint2 r = *reinterpret_cast<const uint2*>(p);
        const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = to_f32(e[i]);
    } else {
        static_assert(kBytes % 16 == 0, "vectors of 16 bytes");
        constexpr int kPer = 16 / (int)sizeof(T);
#pragma unroll
        for (int c = 0; c < kBytes / 16; ++c) {
            const uint4 r = reinterpret_cast<const uint4*>(p)[c];
            const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
            for (int i = 0; i < kPer; ++i) f[c * kPer + i] = to_f32(e[i]);
        }
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[N]) {
    constexpr int kBytes = N * (int)sizeof(T);
    if constexpr (N == 1) {
        *p = from_f32<T>(f[0]);
    } else if constexpr (kBytes == 8) {
        uint2 r;
        T* e = reinterpret_cast<T*>(&r);
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = from_f32<T>(f[i]);
        *reinterpret_cast<uint2*>(p) = r;
    } else {
        static_assert(kBytes % 16 == 0, "vectors of 16 bytes");
        constexpr int kPer = 16 / (int)sizeof(T);
#pragma unroll
        for (int c = 0; c < kBytes / 16; ++c) {
            uint4 r;
            T* e = reinterpret_cast<T*>(&r);
#pragma unroll
            for (int i = 0; i < kPer; ++i) e[i] = from_f32<T>(f[c * kPer + i]);
            reinterpret_cast<uint4*>(p)[c] = r;
        }
    }
}

// Quantizer constants of a width (see mpq_encode).
struct LevelRule {
    float half_L, lo, hi, magic;
    int H, L;
};
__host__ __device__ inline LevelRule level_rule(int bits) {
    LevelRule r;
    r.H = 1 << (bits - 1);
    r.L = (1 << bits) - 1;
    r.half_L = 0.5f * (float)r.L;
    r.lo = -(float)r.H;
    r.hi = (float)r.H - 0.5f;
    r.magic = 8388608.0f + (float)r.H;
    return r;
}

// level_index() without a conversion instruction (those run at an eighth of the rate): the quotient plus 2^23 + H,
// rounded down, holds floor(y) + H in its low mantissa bits, and float(u) is one subtraction away.
// Where the range is the row's own largest magnitude, finite with a finite reciprocal, and no element is a NaN, the
// quotient lies in [-L/2, L/2] up to two roundings, inside [-H, H): `plain` leaves the NaN test and both clamps out.
constexpr float kLevelMagic = 8388608.0f;                  // 2^23, bits 0x4b000000
template <int ACT, int N>
__device__ __forceinline__ void shifted_levels(const float (&x)[N], float inv_s, const LevelRule& r, bool plain, float (&shifted)[N]) {
    if (ACT == MPQ_ACT_HTANH && plain) {
#pragma unroll
        for (int i = 0; i < N; ++i) shifted[i] = __fadd_rd(__fmul_rn(__fmul_rn(x[i], inv_s), r.half_L), r.magic);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float y = __fmul_rn(__fmul_rn(x[i], inv_s), r.half_L);
            if (!(y == y)) y = 0.0f;                       // NaN -> level just above zero
            if (ACT == MPQ_ACT_HRELU) y = fmaxf(y, 0.0f);
            shifted[i] = __fadd_rd(fminf(fmaxf(y, r.lo), r.hi), r.magic);
        }
    }
}
// Zero, or NaN where an element is not finite: one multiply-add per element instead of a test.
template <int N>
__device__ __forceinline__ float finite_sum(const float (&x)[N]) {
    float z = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) z = fmaf(x[i], 0.0f, z);
    return z;
}
__device__ __forceinline__ bool ordinary(float v) { return fabsf(v) < __int_as_float(0x7f800000); }             // neither NaN nor infinite
constexpr float kNaN = __builtin_nanf("");
// max(a, b), NaN where either is one (fmaxf would give the other).
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Level bytes of four shifted levels (a level is below 2^8: the low byte of the float's bits).
__device__ __forceinline__ uint32_t level_word(float a, float b, float c, float d) {
    return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040),
                       __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}
__device__ __forceinline__ float level_number(float shifted, const LevelRule& r) {                              // 2u - L, exact
    return fmaf(2.0f, shifted - kLevelMagic, -(float)r.L);
}

}  // namespace mpq
