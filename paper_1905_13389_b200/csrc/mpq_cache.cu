// Paged cache of keys and values on levels of 8 or 4 bits: quantised as it is written, and read back.
//
// A group of dim / 16 lanes (rounded up to a power of two) owns one (token, head), sixteen elements of the
// key and of the value per lane, the range by shuffles inside the group.  Nothing is staged or read twice.
// Large calls are bound by issuing instructions as much as by memory (with eight elements per lane 0.78 of the
// issue slots and 18 us for 8192 tokens x 8 heads x 128, 4 bits), hence the share per lane and a quantizer without
// tests or conversions where no element is out of the ordinary; small ones by the latency of the one round trip.
#include "mpq_levels.cuh"

namespace mpq {

struct CacheArgs {
    const void* k; int64_t k_ts, k_hs;
    const void* v; int64_t v_ts, v_hs;
    const int64_t* slots;
    int64_t tokens;
    int heads, dim;
    uint8_t *k_levels, *v_levels;
    float *k_scale, *v_scale;
    int64_t pages;
    int page_size, page_shift;                                // shift: log2 of a page size that is a power of two, else -1
};

constexpr int kCacheThreads = 256;
constexpr int kLaneElems = 16;

// Row of the cache (in tokens) that slot and head name, or -1.
__device__ __forceinline__ int64_t cache_row(const CacheArgs& g, int64_t slot, int head) {
    const uint64_t total = (uint64_t)g.pages * (uint32_t)g.page_size;
    if ((uint64_t)slot >= total) return -1;                    // negative slots are huge unsigned numbers
    int64_t page;
    if (g.page_shift >= 0) page = slot >> g.page_shift;
    else if (total <= 0xffffffffull) page = (uint32_t)slot / (uint32_t)g.page_size;       // a 32-bit division where it is enough
    else page = slot / g.page_size;
    return (page * g.heads + head) * g.page_size + (slot - page * g.page_size);
}

template <typename T, bool VEC>
__device__ __forceinline__ void load_lane(const T* p, float (&f)[kLaneElems]) {
    if constexpr (VEC) {
        load_vec<T, kLaneElems>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < kLaneElems; ++i) f[i] = to_f32(p[i]);
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_lane(T* p, const float (&f)[kLaneElems]) {
    if constexpr (VEC) {
        store_vec<T, kLaneElems>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < kLaneElems; ++i) p[i] = from_f32<T>(f[i]);
    }
}

template <int BITS>
__device__ __forceinline__ void encode_lane(const float (&f)[kLaneElems], float s, uint8_t* dst) {
    const LevelRule r = level_rule(BITS);
    const float inv = s > 0.0f && s < __int_as_float(0x7f800000) ? __frcp_rn(s) : 0.0f;      // = inverse_scale(s)
    float t[kLaneElems];
    shifted_levels<MPQ_ACT_HTANH>(f, inv, r, ordinary(inv) && finite_sum(f) == 0.0f, t);
    if (BITS == 4) {
        // two levels a byte, joined as numbers: (2^23 + u) + 16 u' is exact and keeps both in its low byte
#pragma unroll
        for (int i = 0; i < kLaneElems; i += 2) t[i / 2] = fmaf(16.0f, t[i + 1] - kLevelMagic, t[i]);
    }
    constexpr int kWords = kLaneElems * BITS / 32;
    uint32_t w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = level_word(t[4 * i], t[4 * i + 1], t[4 * i + 2], t[4 * i + 3]);
    if constexpr (kWords == 4) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
}
template <int BITS>
__device__ __forceinline__ void decode_lane(const uint8_t* src, float s, float (&f)[kLaneElems]) {
    constexpr int L = (1 << BITS) - 1;
    const float alpha = __fdiv_rn(s, (float)L);
    constexpr int kWords = kLaneElems * BITS / 32;
    uint32_t w[kWords];
    if constexpr (kWords == 4) { const uint4 v = *reinterpret_cast<const uint4*>(src); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    else { const uint2 v = *reinterpret_cast<const uint2*>(src); w[0] = v.x; w[1] = v.y; }
#pragma unroll
    for (int i = 0; i < kLaneElems; ++i) {                 // u into the mantissa of 2^23: no conversion instruction
        const float shifted = __uint_as_float(((w[i * BITS / 32] >> (i * BITS % 32)) & L) | 0x4b000000u);
        f[i] = fmaf(2.0f, shifted - kLevelMagic, -(float)L) * alpha;
    }
}

// max(m, |a|, |b|), NaNs ignored
__device__ __forceinline__ float max_abs(float m, float a, float b) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}

template <typename T, int BITS, bool VEC>
__global__ void __launch_bounds__(kCacheThreads) cache_write_kernel(const CacheArgs g, int group, int group_log2) {
    chain_entry();
    const int64_t token = ((int64_t)blockIdx.x * kCacheThreads + threadIdx.x) >> group_log2;
    const int lane = threadIdx.x & (group - 1), head = blockIdx.y;
    const bool live = token < g.tokens && lane * kLaneElems < g.dim;
    float kf[kLaneElems], vf[kLaneElems], km = 0.0f, vm = 0.0f;
    int64_t row = -1;
    if (live) {
        load_lane<T, VEC>(static_cast<const T*>(g.k) + token * g.k_ts + head * g.k_hs + lane * kLaneElems, kf);
        load_lane<T, VEC>(static_cast<const T*>(g.v) + token * g.v_ts + head * g.v_hs + lane * kLaneElems, vf);
        row = cache_row(g, g.slots[token], head);
#pragma unroll
        for (int i = 0; i < kLaneElems; i += 2) { km = max_abs(km, kf[i], kf[i + 1]); vm = max_abs(vm, vf[i], vf[i + 1]); }
    }
    for (int o = group >> 1; o > 0; o >>= 1) {
        km = fmaxf(km, __shfl_xor_sync(0xffffffffu, km, o));
        vm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, o));
    }
    if (!live || row < 0) return;
    const int64_t at = row * (g.dim * BITS / 8) + lane * (kLaneElems * BITS / 8);
    encode_lane<BITS>(kf, km, g.k_levels + at);
    encode_lane<BITS>(vf, vm, g.v_levels + at);
    if (lane == 0) { g.k_scale[row] = km; g.v_scale[row] = vm; }
}

template <typename T, int BITS, bool VEC>
__global__ void __launch_bounds__(kCacheThreads) cache_read_kernel(const CacheArgs g, int group, int group_log2) {
    chain_entry();
    const int64_t token = ((int64_t)blockIdx.x * kCacheThreads + threadIdx.x) >> group_log2;
    const int lane = threadIdx.x & (group - 1), head = blockIdx.y;
    if (token >= g.tokens || lane * kLaneElems >= g.dim) return;
    const int64_t row = cache_row(g, g.slots[token], head);
    float kf[kLaneElems] = {}, vf[kLaneElems] = {};
    if (row >= 0) {
        const int64_t at = row * (g.dim * BITS / 8) + lane * (kLaneElems * BITS / 8);
        decode_lane<BITS>(g.k_levels + at, g.k_scale[row], kf);
        decode_lane<BITS>(g.v_levels + at, g.v_scale[row], vf);
    }
    store_lane<T, VEC>(static_cast<T*>(const_cast<void*>(g.k)) + token * g.k_ts + head * g.k_hs + lane * kLaneElems, kf);
    store_lane<T, VEC>(static_cast<T*>(const_cast<void*>(g.v)) + token * g.v_ts + head * g.v_hs + lane * kLaneElems, vf);
}

template <typename T, int BITS>
int launch_cache(bool write, bool vec, const CacheArgs& g, cudaStream_t st) {
    int group = 1, log2 = 0;
    while (group * kLaneElems < g.dim) { group *= 2; ++log2; }
    const int64_t blocks = ceil_div(g.tokens * group, kCacheThreads);
    if (blocks > 0x7fffffff || g.heads > 65535) return MPQ_ERR_BAD_SHAPE;
    auto* kernel = write ? (vec ? cache_write_kernel<T, BITS, true> : cache_write_kernel<T, BITS, false>)
                         : (vec ? cache_read_kernel<T, BITS, true> : cache_read_kernel<T, BITS, false>);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)g.heads, 1);
    cfg.blockDim = dim3(kCacheThreads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, g, group, log2) != cudaSuccess) { cudaGetLastError(); return MPQ_ERR_CUDA; }
    return launch_status();
}

inline int page_shift(int page_size) {
    if (page_size <= 0 || (page_size & (page_size - 1))) return -1;
    int s = 0;
    while ((1 << s) < page_size) ++s;
    return s;
}

int cache_call(bool write, int dtype, int bits, const CacheArgs& g, cudaStream_t st) {
    if (g.tokens != 0 && (!g.k || !g.v || !g.slots || !g.k_levels || !g.v_levels || !g.k_scale || !g.v_scale)) return MPQ_ERR_NULL;
    if (!dtype_ok(dtype) || (bits != 8 && bits != 4) || g.dim < 32 || g.dim > 256 || g.dim % 32) return MPQ_ERR_UNSUPPORTED;
    if (g.tokens < 0 || g.heads <= 0 || g.pages <= 0 || g.page_size <= 0) return MPQ_ERR_BAD_SHAPE;
    // what is read may overlap (a broadcast head); what is written may not
    if (!write && ((g.heads > 1 && (g.k_hs < g.dim || g.v_hs < g.dim)) || (g.tokens > 1 && (g.k_ts < g.dim || g.v_ts < g.dim))))
        return MPQ_ERR_BAD_SHAPE;
    const int e = dtype_size(dtype);
    if (!aligned16(g.k_levels) || !aligned16(g.v_levels) || !aligned_to(g.k_scale, 4) || !aligned_to(g.v_scale, 4) ||
        !aligned_to(g.k, e) || !aligned_to(g.v, e) || !aligned_to(g.slots, 8)) return MPQ_ERR_ALIGN;
    if (g.tokens == 0) return MPQ_OK;
    const int step = 16 / e;
    const bool vec = aligned16(g.k) && aligned16(g.v) && g.k_ts % step == 0 && g.v_ts % step == 0 && g.k_hs % step == 0 && g.v_hs % step == 0;
    if (dtype == MPQ_F32) return bits == 8 ? launch_cache<float, 8>(write, vec, g, st) : launch_cache<float, 4>(write, vec, g, st);
    if (dtype == MPQ_F16) return bits == 8 ? launch_cache<__half, 8>(write, vec, g, st) : launch_cache<__half, 4>(write, vec, g, st);
    return bits == 8 ? launch_cache<__nv_bfloat16, 8>(write, vec, g, st) : launch_cache<__nv_bfloat16, 4>(write, vec, g, st);
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_cache_write(const void* k, int64_t k_token_stride, int64_t k_head_stride,
                               const void* v, int64_t v_token_stride, int64_t v_head_stride, int dtype,
                               const int64_t* slots, int64_t tokens, int heads, int dim, int bits,
                               uint8_t* k_levels, float* k_scale, uint8_t* v_levels, float* v_scale,
                               int64_t pages, int page_size, void* stream) {
    const CacheArgs g = {k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, slots, tokens, heads, dim,
                         k_levels, v_levels, k_scale, v_scale, pages, page_size, page_shift(page_size)};
    return cache_call(true, dtype, bits, g, (cudaStream_t)stream);
}

extern "C" int mpq_cache_read(const uint8_t* k_levels, const float* k_scale, const uint8_t* v_levels, const float* v_scale,
                              int64_t pages, int page_size, const int64_t* slots, int64_t tokens, int heads, int dim, int bits,
                              void* k, int64_t k_token_stride, int64_t k_head_stride,
                              void* v, int64_t v_token_stride, int64_t v_head_stride, int dtype, void* stream) {
    const CacheArgs g = {k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, slots, tokens, heads, dim,
                         const_cast<uint8_t*>(k_levels), const_cast<uint8_t*>(v_levels), const_cast<float*>(k_scale),
                         const_cast<float*>(v_scale), pages, page_size, page_shift(page_size)};
    return cache_call(false, dtype, bits, g, (cudaStream_t)stream);
}
