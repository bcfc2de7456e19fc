// Level bytes with one range per row: the root-mean-square norm with the residual's addition
// (mpq_rmsnorm_levels) and the plain row encoder (mpq_encode_levels).
#include "mpq_levels.cuh"

namespace mpq {

struct RowArgs {
    const void* x; int64_t ldx;
    const void* res; int64_t ldr;
    const float* gain;
    float eps;
    int64_t rows, k, row_bytes;
    LevelRule rule;
    void* res_out; int64_t ldo;
    uint8_t* levels; float* scale; int32_t* sums;
    void* values; int64_t ldv;
    int values_dtype;
};

// One row of partial results: sum of squares and the largest |h gain|.
// y = (h gain) r with one r > 0 per row, and a rounded product by r is monotone, so
// max |y| = r max |h gain| to the last bit: both statistics come out of ONE pass.
// The row's constants follow from them in the first warp alone: a root and four exact divisions in every thread were
// a third of the kernel's instructions, and it is bound by issuing them (0.74 of the issue slots).
// Under the norm the largest magnitude keeps NaNs: an infinite element gives r = 0, and its product with a gain of 0 or
// with r is the NaN that the row's range has to be.  Without the norm a NaN takes no part in the range.
// A finite row whose sum of squares overflows fp32 gives r = 0 as well.  Every thread sees that, the row is read again and
// its squares are summed 2^160 times smaller (large_row_scalars), so it keeps its range; residual_out, which may lie over
// the inputs, is therefore stored after the statistics.  (4096 x 4096: 28.2 us before, 28.9 so; with a sum of its own for large
// squares beside the ordinary one some 30.)
struct RowScalars { float r, s, inv, alpha; };
template <bool NORM> __device__ __forceinline__ float larger(float a, float b) { return NORM ? max_nan(a, b) : fmaxf(a, b); }
template <bool NORM>
__device__ __forceinline__ RowScalars row_scalars(float r, float mx, int L) {
    RowScalars c;
    c.r = r;
    c.s = NORM ? mx * r : mx;
    c.inv = inverse_scale(c.s);
    c.alpha = __fdiv_rn(c.s, (float)L);
    return c;
}
template <bool NORM>
__device__ __forceinline__ float row_factor(float ss, const RowArgs& g) {
    return NORM ? __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, (float)g.k), g.eps))) : 1.0f;
}
// The row's constants in every thread.  (sh keeps the warps' maxima, and the lanes of a single warp the row's in mx.)
template <bool NORM>
__device__ __forceinline__ RowScalars block_scalars(float ss, float& mx, const RowArgs& g, float2* sh, RowScalars* sh_scalars) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (NORM) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        mx = larger<NORM>(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    }
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (warps == 1) return row_scalars<NORM>(row_factor<NORM>(ss, g), mx, g.rule.L);
    if (lane == 0) sh[threadIdx.x >> 5] = make_float2(ss, mx);
    __syncthreads();
    if (threadIdx.x < 32) {
        const float2 v = lane < warps ? sh[lane] : make_float2(0.0f, 0.0f);
        ss = v.x; mx = v.y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            if (NORM) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            mx = larger<NORM>(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        }
        const RowScalars c = row_scalars<NORM>(row_factor<NORM>(ss, g), mx, g.rule.L);
        if (lane == 0) *sh_scalars = c;
    }
    __syncthreads();
    return *sh_scalars;
}
// The constants of a row whose squares overflow, in every thread; sh holds the warps' maxima of the first round.  Not inlined:
// hardly any call comes here.
template <typename T>
__device__ __noinline__ RowScalars large_row_scalars(const T* x, const T* res, int k, float eps, int L, float mx, float2* sh) {
    constexpr float kDown = 8.271806125530277e-25f;                      // 2^-80: 2^23 squares of 2^48 fit
    float ss = 0.0f;
#pragma unroll 1
    for (int i = threadIdx.x; i < k; i += blockDim.x) {
        const float v = (to_f32(x[i]) + (res ? to_f32(res[i]) : 0.0f)) * kDown;
        ss = fmaf(v, v, ss);
    }
#pragma unroll 1
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const int warps = blockDim.x >> 5;
    if (warps > 1) {
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5].x = ss;
        __syncthreads();
        ss = mx = 0.0f;
#pragma unroll 1
        for (int w = 0; w < warps; ++w) { ss += sh[w].x; mx = max_nan(mx, sh[w].y); }
    }
    const float r = __fdiv_rn(kDown, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, (float)k), eps * kDown * kDown)));
    return row_scalars<true>(ordinary(ss) ? r : kNaN, mx, L);            // an element is infinite: NaN
}
__device__ __forceinline__ void block_level_sum(int u, int32_t* dst, int* sh) {
    u = __reduce_add_sync(0xffffffffu, u);
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (warps > 1) {
        if (lane == 0) sh[threadIdx.x >> 5] = u;
        __syncthreads();
        if (threadIdx.x >= 32) return;
        u = __reduce_add_sync(0xffffffffu, lane < warps ? sh[lane] : 0);
    }
    if (lane == 0) *dst = u;
}

// N adjacent elements at once where addresses and strides allow it (VECTOR), one by one otherwise, `count` of
// them (the tail of a row).  Threads own the same N elements either way, so a row's sums do not depend on how
// it lies in memory.
template <typename T, int N, bool VECTOR>
__device__ __forceinline__ void load_part(const T* p, float (&f)[N], int count) {
    if constexpr (VECTOR) {
        load_vec<T, N>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = i < count ? to_f32(p[i]) : 0.0f;
    }
}
template <typename T, int N, bool VECTOR>
__device__ __forceinline__ void store_part(T* p, const float (&f)[N], int count) {
    if constexpr (VECTOR) {
        store_vec<T, N>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) if (i < count) p[i] = from_f32<T>(f[i]);
    }
}
// ... the same of values already rounded to T
template <typename T, int N> struct alignas(N * sizeof(T)) Rounded { T e[N]; };
template <typename T, int N, bool VECTOR>
__device__ __forceinline__ void store_rounded(T* p, const Rounded<T, N>& v, int count) {
    if constexpr (VECTOR) {
        static_assert(sizeof(v) == 16, "one vector");
        *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) if (i < count) p[i] = v.e[i];
    }
}
// Level bytes of N elements, `count` of them inside the row; returns the sum of the levels.  Level rows are 16-byte
// aligned and padded, so whole words always fit; bytes past the row's end are 0.
template <int N, bool VECTOR>
__device__ __forceinline__ uint32_t store_levels(uint8_t* p, const float (&shifted)[N], int count) {
    uint32_t total = 0;
#pragma unroll
    for (int c = 0; c < N / 4; ++c) {
        uint32_t w = level_word(shifted[4 * c], shifted[4 * c + 1], shifted[4 * c + 2], shifted[4 * c + 3]);
        if (!VECTOR) w &= count >= 4 * c + 4 ? 0xffffffffu : count <= 4 * c ? 0u : 0xffffffffu >> (8 * (4 * c + 4 - count));
        reinterpret_cast<uint32_t*>(p)[c] = w;
        total = __dp4a(w, 0x01010101u, total);
    }
    return total;
}
template <int N, bool VECTOR>
__device__ __forceinline__ void store_values(const RowArgs& g, int64_t row, int64_t at, const float (&shifted)[N], float alpha, int count) {
    float f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = level_number(shifted[i], g.rule) * alpha;
    const int64_t o = row * g.ldv + at;
    if (g.values_dtype == MPQ_BF16) store_part<__nv_bfloat16, N, VECTOR>(static_cast<__nv_bfloat16*>(g.values) + o, f, count);
    else if (g.values_dtype == MPQ_F16) store_part<__half, N, VECTOR>(static_cast<__half*>(g.values) + o, f, count);
    else store_part<float, N, VECTOR>(static_cast<float*>(g.values) + o, f, count);
}

// One CTA per row; the row stays in registers between the statistics and the quantizer (NV vectors of
// VEC elements per thread), so memory is read once and written once.
template <typename T, int VEC, int NV, bool VECTOR, bool NORM, int ACT>
__global__ void __launch_bounds__(1024, NV == 1 ? 2 : 1)           // 32 registers where a vector is all a thread has: every thread of the device
level_rows_kernel(const RowArgs g) {
    __shared__ float2 sh_stats[32];
    __shared__ RowScalars sh_scalars;
    __shared__ int sh_sum[32];
    chain_entry();
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(g.x) + row * g.ldx;
    const T* res = NORM && g.res ? static_cast<const T*>(g.res) + row * g.ldr : nullptr;
    const int k = (int)g.k, nvec = (k + VEC - 1) / VEC;
    float h[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = threadIdx.x + j * blockDim.x;
        if (i < nvec) load_part<T, VEC, VECTOR>(x + (int64_t)i * VEC, h[j], k - i * VEC);
    }
    if (NORM && res) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            if (i < nvec) {
                float f[VEC];
                load_part<T, VEC, VECTOR>(res + (int64_t)i * VEC, f, k - i * VEC);
#pragma unroll
                for (int e = 0; e < VEC; ++e) h[j][e] += f[e];
            }
        }
    }
    float ss = 0.0f, mx = 0.0f;
    Rounded<T, VEC> sum[NORM ? NV : 1];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = threadIdx.x + j * blockDim.x;
        if (i < nvec) {
            if (NORM) {
                if (g.res_out) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[j].e[e] = from_f32<T>(h[j][e]);
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) ss = fmaf(h[j][e], h[j][e], ss);
                if (g.gain) {
                    // read-only loads: the compiler may move them above the stores of residual_out
                    if constexpr (VECTOR) {
#pragma unroll
                        for (int c = 0; c < VEC / 4; ++c) {
                            const float4 gn = __ldg(reinterpret_cast<const float4*>(g.gain + (int64_t)i * VEC) + c);
                            h[j][4 * c] *= gn.x; h[j][4 * c + 1] *= gn.y; h[j][4 * c + 2] *= gn.z; h[j][4 * c + 3] *= gn.w;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) if (i * VEC + e < k) h[j][e] *= __ldg(g.gain + i * VEC + e);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) mx = larger<NORM>(mx, ACT == MPQ_ACT_HRELU ? h[j][e] : fabsf(h[j][e]));
        }
    }
    RowScalars c = block_scalars<NORM>(ss, mx, g, sh_stats, &sh_scalars);
    if (NORM && c.r == 0.0f) c = large_row_scalars(x, res, k, g.eps, g.rule.L, mx, sh_stats);
    const float r = c.r, s = c.s, inv = c.inv, alpha = c.alpha;
    // (a NaN range, after a NaN or an infinity under the norm, has the reciprocal 0 and is not ordinary)
    const bool plain = ordinary(s) && ordinary(inv);
    uint8_t* out = g.levels + row * g.row_bytes;
    int total = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = threadIdx.x + j * blockDim.x;
        if (i < nvec) {
            if (NORM && g.res_out) store_rounded<T, VEC, VECTOR>(static_cast<T*>(g.res_out) + row * g.ldo + (int64_t)i * VEC, sum[j], k - i * VEC);
            float y[VEC], shifted[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[e] = NORM ? h[j][e] * r : h[j][e];
            shifted_levels<ACT>(y, inv, g.rule, plain && finite_sum(y) == 0.0f, shifted);
            total += (int)store_levels<VEC, VECTOR>(out + (int64_t)i * VEC, shifted, k - i * VEC);
            if (g.values) store_values<VEC, VECTOR>(g, row, (int64_t)i * VEC, shifted, alpha, k - i * VEC);
        }
    }
    // padding words behind the last vector
    for (int i = nvec * VEC + threadIdx.x * 4; i < (int)g.row_bytes; i += blockDim.x * 4) *reinterpret_cast<uint32_t*>(out + i) = 0u;
    block_level_sum(total, g.sums + row, sh_sum);
    if (threadIdx.x == 0) g.scale[row] = s;
}

// Rows that do not fit the registers of one CTA: the row is read twice (statistics, quantizer), the
// residual sum formed both times.  residual_out is written in the second pass, element by element after
// the thread's own reads of the same element, so it may be x or the residual.
template <typename T, bool NORM, int ACT>
__global__ void __launch_bounds__(1024)
level_wide_rows_kernel(const RowArgs g) {
    __shared__ float2 sh_stats[32];
    __shared__ RowScalars sh_scalars;
    __shared__ int sh_sum[32];
    chain_entry();
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(g.x) + row * g.ldx;
    const T* res = NORM && g.res ? static_cast<const T*>(g.res) + row * g.ldr : nullptr;
    float ss = 0.0f, mx = 0.0f;
    for (int64_t i = threadIdx.x; i < g.k; i += blockDim.x) {
        float h = to_f32(x[i]);
        if (NORM) {
            if (res) h += to_f32(res[i]);
            ss = fmaf(h, h, ss);
            if (g.gain) h *= g.gain[i];
        }
        mx = larger<NORM>(mx, ACT == MPQ_ACT_HRELU ? h : fabsf(h));
    }
    RowScalars c = block_scalars<NORM>(ss, mx, g, sh_stats, &sh_scalars);
    if (NORM && c.r == 0.0f) c = large_row_scalars(x, res, (int)g.k, g.eps, g.rule.L, mx, sh_stats);
    const float r = c.r, s = c.s, inv = c.inv, alpha = c.alpha;
    uint8_t* out = g.levels + row * g.row_bytes;
    int total = 0;
    for (int64_t i = threadIdx.x; i < g.row_bytes; i += blockDim.x) {
        if (i >= g.k) { out[i] = 0; continue; }
        float h = to_f32(x[i]);
        if (NORM) {
            if (res) h += to_f32(res[i]);
            if (g.res_out) static_cast<T*>(g.res_out)[row * g.ldo + i] = from_f32<T>(h);
            if (g.gain) h *= g.gain[i];
            h *= r;
        }
        const float y[1] = {h};
        float shifted[1];
        shifted_levels<ACT>(y, inv, g.rule, false, shifted);
        const uint8_t u = (uint8_t)__float_as_uint(shifted[0]);
        total += u;
        out[i] = u;
        if (g.values) store_values<1, false>(g, row, i, shifted, alpha, 1);
    }
    block_level_sum(total, g.sums + row, sh_sum);
    if (threadIdx.x == 0) g.scale[row] = s;
}

// Threads and vectors per thread: one vector each up to 1024 threads (a single row of 4096: 2.7 us, with two 3.6, with
// four 6.2; 4096 rows 33, 33 and 39 us), then more.
template <typename T, int VEC, bool VECTOR, bool NORM, int ACT>
int launch_level_rows(const RowArgs& g, cudaStream_t st) {
    const int64_t nvec = ceil_div(g.k, VEC);
    auto threads_for = [&](int nv) { return (unsigned)(ceil_div(ceil_div(nvec, nv), 32) * 32); };
    if (threads_for(1) <= 1024) return launch_chained(level_rows_kernel<T, VEC, 1, VECTOR, NORM, ACT>, (unsigned)g.rows, threads_for(1), 0, st, g);
    if (threads_for(2) <= 1024) return launch_chained(level_rows_kernel<T, VEC, 2, VECTOR, NORM, ACT>, (unsigned)g.rows, threads_for(2), 0, st, g);
    if (threads_for(4) <= 1024) return launch_chained(level_rows_kernel<T, VEC, 4, VECTOR, NORM, ACT>, (unsigned)g.rows, threads_for(4), 0, st, g);
    return launch_chained(level_wide_rows_kernel<T, NORM, ACT>, (unsigned)g.rows, 1024u, 0, st, g);
}

template <typename T, bool NORM, int ACT>
int launch_level_rows_of(const RowArgs& g, cudaStream_t st) {
    constexpr int VEC = 16 / (int)sizeof(T);
    auto fits = [&](const void* p, int64_t ld, int size) { return !p || (aligned_to(p, VEC * size > 16 ? 16 : VEC * size) && (ld % VEC == 0 || g.rows == 1)); };
    const bool vec = g.k % VEC == 0 && fits(g.x, g.ldx, sizeof(T)) && fits(g.res, g.ldr, sizeof(T)) && fits(g.res_out, g.ldo, sizeof(T)) &&
                     fits(g.gain, 0, 4) && (!g.values || fits(g.values, g.ldv, dtype_size(g.values_dtype)));
    return vec ? launch_level_rows<T, VEC, true, NORM, ACT>(g, st) : launch_level_rows<T, VEC, false, NORM, ACT>(g, st);
}
template <bool NORM, int ACT>
int launch_level_rows_dtype(int dtype, const RowArgs& g, cudaStream_t st) {
    if (dtype == MPQ_F32) return launch_level_rows_of<float, NORM, ACT>(g, st);
    if (dtype == MPQ_F16) return launch_level_rows_of<__half, NORM, ACT>(g, st);
    return launch_level_rows_of<__nv_bfloat16, NORM, ACT>(g, st);
}

int check_level_rows(const RowArgs& g, int dtype, int bits) {
    if (!dtype_ok(dtype) || (g.values && !dtype_ok(g.values_dtype)) || !bits_ok(bits)) return MPQ_ERR_UNSUPPORTED;
    if (g.rows < 0 || g.rows > 0x7fffffff || g.k <= 0 || g.k >= (1 << 23)) return MPQ_ERR_BAD_SHAPE;
    if (g.rows > 1 && (g.ldx < g.k || (g.res && g.ldr < g.k) || (g.res_out && g.ldo < g.k) || (g.values && g.ldv < g.k)))
        return MPQ_ERR_BAD_SHAPE;
    const int e = dtype_size(dtype);
    if (!aligned16(g.levels) || !aligned_to(g.x, e) || !aligned_to(g.res, e) || !aligned_to(g.res_out, e) || !aligned_to(g.gain, 4) ||
        !aligned_to(g.scale, 4) || !aligned_to(g.sums, 4) || (g.values && !aligned_to(g.values, dtype_size(g.values_dtype))))
        return MPQ_ERR_ALIGN;
    return MPQ_OK;
}

}  // namespace mpq

using namespace mpq;

extern "C" int64_t mpq_level_row_bytes(int64_t k) { return k > 0 ? level_row_bytes(k) : 0; }

extern "C" int mpq_rmsnorm_levels(const void* x, int64_t ldx, const void* residual, int64_t ldr, int dtype,
                                  const float* gain, float eps, int64_t rows, int64_t k, int bits,
                                  void* residual_out, int64_t ldo,
                                  uint8_t* levels, float* scale, int32_t* sums,
                                  void* values, int values_dtype, int64_t ldv, void* stream) {
    if (rows != 0 && (!x || !levels || !scale || !sums)) return MPQ_ERR_NULL;
    RowArgs g = {x, ldx, residual, ldr, gain, eps, rows, k, level_row_bytes(k), {}, residual_out, ldo, levels, scale, sums,
                 values, ldv, values_dtype};
    const int rc = check_level_rows(g, dtype, bits);
    if (rc != MPQ_OK || rows == 0) return rc;
    if (!(eps >= 0.0f)) return MPQ_ERR_UNSUPPORTED;
    g.rule = level_rule(bits);
    return launch_level_rows_dtype<true, MPQ_ACT_HTANH>(dtype, g, (cudaStream_t)stream);
}

extern "C" int mpq_encode_levels(const void* x, int64_t ldx, int dtype, int64_t rows, int64_t k, int act, int bits,
                                 uint8_t* levels, float* scale, int32_t* sums,
                                 void* values, int values_dtype, int64_t ldv, void* stream) {
    if (rows != 0 && (!x || !levels || !scale || !sums)) return MPQ_ERR_NULL;
    if (act != MPQ_ACT_HTANH && act != MPQ_ACT_HRELU) return MPQ_ERR_UNSUPPORTED;
    RowArgs g = {x, ldx, nullptr, 0, nullptr, 0.0f, rows, k, level_row_bytes(k), {}, nullptr, 0, levels, scale, sums,
                 values, ldv, values_dtype};
    const int rc = check_level_rows(g, dtype, bits);
    if (rc != MPQ_OK || rows == 0) return rc;
    g.rule = level_rule(bits);
    return act == MPQ_ACT_HTANH ? launch_level_rows_dtype<false, MPQ_ACT_HTANH>(dtype, g, (cudaStream_t)stream)
                                : launch_level_rows_dtype<false, MPQ_ACT_HRELU>(dtype, g, (cudaStream_t)stream);
}
