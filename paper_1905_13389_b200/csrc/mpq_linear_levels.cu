// Product of level bytes with bias, activation and residual in its epilogue (mpq_linear_levels).
//
// With q = 2u - L (Eq. 16) the layer's integer product is
//   sum q_a q_w = 4 sum u_a u_w - 2 L_w sum u_a - 2 L_a sum u_w + k L_a L_w,
// so the inner loop multiplies unsigned bytes and the level sums that lie beside the operands do the rest.
// The result fits int32 (checked on the host), hence the terms may be combined modulo 2^32.
#include "mpq_levels.cuh"

namespace mpq {

struct LinearArgs {
    const uint8_t* a; const float* a_scale; const int32_t* a_sums;
    const uint8_t* w; const float* w_scale; const int32_t* w_sums;
    int64_t m, n, k, row_bytes;
    int La, Lw;
    const float* bias;
    int glue;
    const void* res; int64_t ldr;
    void* out; int64_t ldo;
};

// Epilogue constants of one row and one column, and the order of its fp32 operations (see the header).
__device__ __forceinline__ float glue_value(float f, int glue) {
    switch (glue) {
        case MPQ_GLUE_RELU: return fmaxf(f, 0.0f);
        case MPQ_GLUE_GELU: return 0.5f * f * (1.0f + erff(f * 0.70710678118654752f));
        case MPQ_GLUE_GELU_TANH: {
            // 0.5 f (1 + tanh z) = f / (1 + e^(-2z)); the exponential saturates to 0 or infinity, the quotient to f or 0
            const float z2 = 1.5957691216057308f * (f + 0.044715f * f * f * f);
            return __fdividef(f, 1.0f + __expf(-z2));
        }
        case MPQ_GLUE_SILU: return __fdividef(f, 1.0f + __expf(-f));
        default: return f;
    }
}

constexpr int kTile = 64, kStep = 64;      // 64 x 64 outputs, 64 bytes of k at a time

template <typename T>
__global__ void __launch_bounds__(256) linear_levels_kernel(const LinearArgs g) {
    __shared__ uint32_t sa[kTile][kStep / 4 + 1], sw[kTile][kStep / 4 + 1];
    chain_entry();
    const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    uint32_t acc[4][4] = {};
    for (int64_t k0 = 0; k0 < g.row_bytes; k0 += kStep) {
        for (int i = threadIdx.x; i < kTile * (kStep / 16); i += 256) {
            const int r = i / (kStep / 16), c = i % (kStep / 16);
            const int64_t at = k0 + c * 16;
            uint4 va = make_uint4(0, 0, 0, 0), vw = va;
            if (at < g.row_bytes) {
                if (m0 + r < g.m) va = *reinterpret_cast<const uint4*>(g.a + (m0 + r) * g.row_bytes + at);
                if (n0 + r < g.n) vw = *reinterpret_cast<const uint4*>(g.w + (n0 + r) * g.row_bytes + at);
            }
            sa[r][4 * c] = va.x; sa[r][4 * c + 1] = va.y; sa[r][4 * c + 2] = va.z; sa[r][4 * c + 3] = va.w;
            sw[r][4 * c] = vw.x; sw[r][4 * c + 1] = vw.y; sw[r][4 * c + 2] = vw.z; sw[r][4 * c + 3] = vw.w;
        }
        __syncthreads();
#pragma unroll 4
        for (int t = 0; t < kStep / 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(sa[ty * 4 + i][t], sw[tx + 16 * j][t], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int64_t r = m0 + ty * 4 + i;
        if (r >= g.m) break;
        const float ra = __fdiv_rn(g.a_scale[r], (float)g.La);
        const uint32_t row_term = (uint32_t)g.k * (uint32_t)g.La * (uint32_t)g.Lw - 2u * (uint32_t)g.Lw * (uint32_t)g.a_sums[r];
        for (int j = 0; j < 4; ++j) {
            const int64_t c = n0 + tx + 16 * j;
            if (c >= g.n) continue;
            const int32_t q = (int32_t)(4u * acc[i][j] + row_term - 2u * (uint32_t)g.La * (uint32_t)g.w_sums[c]);
            float f = (float)q * (ra * __fdiv_rn(g.w_scale[c], (float)g.Lw));
            if (g.bias) f += g.bias[c];
            f = glue_value(f, g.glue);
            if (g.res) f += to_f32(static_cast<const T*>(g.res)[r * g.ldr + c]);
            static_cast<T*>(g.out)[r * g.ldo + c] = from_f32<T>(f);
        }
    }
}

template <typename T>
int launch_linear_levels(const LinearArgs& g, cudaStream_t st) {
    const int64_t tiles_m = ceil_div(g.m, kTile);
    if (tiles_m > 65535) return MPQ_ERR_BAD_SHAPE;
    linear_levels_kernel<T><<<dim3((unsigned)ceil_div(g.n, kTile), (unsigned)tiles_m), 256, 0, st>>>(g);
    return launch_status();
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_linear_levels(const uint8_t* a, const float* a_scale, const int32_t* a_sums, int a_bits,
                                 const uint8_t* w, const float* w_scale, const int32_t* w_sums, int w_bits,
                                 int64_t m, int64_t n, int64_t k,
                                 const float* bias, int glue, const void* residual, int64_t ldr,
                                 void* out, int dtype, int64_t ldo, void* stream) {
    if (m != 0 && (!a || !a_scale || !a_sums || !w || !w_scale || !w_sums || !out)) return MPQ_ERR_NULL;
    if (m < 0 || n <= 0 || k <= 0 || m > 0x7fffffff || n > 0x7fffffff || (m > 1 && (ldo < n || (residual && ldr < n)))) return MPQ_ERR_BAD_SHAPE;
    if (!bits_ok(a_bits) || !bits_ok(w_bits) || !dtype_ok(dtype) || glue < MPQ_GLUE_NONE || glue > MPQ_GLUE_SILU) return MPQ_ERR_UNSUPPORTED;
    const int64_t La = (1 << a_bits) - 1, Lw = (1 << w_bits) - 1;
    if (k > 0x7fffffff / (La * Lw)) return MPQ_ERR_OVERFLOW;
    const int e = dtype_size(dtype);
    if (!aligned16(a) || !aligned16(w) || !aligned_to(a_scale, 4) || !aligned_to(a_sums, 4) || !aligned_to(w_scale, 4) || !aligned_to(w_sums, 4) ||
        !aligned_to(bias, 4) || !aligned_to(residual, e) || !aligned_to(out, e)) return MPQ_ERR_ALIGN;
    if (m == 0) return MPQ_OK;
    const LinearArgs g = {a, a_scale, a_sums, w, w_scale, w_sums, m, n, k, level_row_bytes(k), (int)La, (int)Lw, bias, glue, residual, ldr, out, ldo};
    if (dtype == MPQ_F32) return launch_linear_levels<float>(g, (cudaStream_t)stream);
    if (dtype == MPQ_F16) return launch_linear_levels<__half>(g, (cudaStream_t)stream);
    return launch_linear_levels<__nv_bfloat16>(g, (cudaStream_t)stream);
}
