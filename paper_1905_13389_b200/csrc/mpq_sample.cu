// Drawing one token a row from logits: temperature, top-k, top-p, min-p, given random numbers (mpq_sample).
//
// Which token is drawn hangs on where a running sum passes a border, so weights are 64-bit fixed-point numbers
// (whole multiples of 2^-shift of the largest weight, made from 64-bit exponentials): their sums are exact whatever the
// order, and a border lies within 2^-44 or so of where real numbers would have it.
#include "mpq_levels.cuh"

namespace mpq {

struct SampleArgs {
    const void* logits; int64_t ld;
    int64_t rows; int vocab;
    const float *temperature; const int32_t* top_k; const float *top_p, *min_p, *uniform;
    int64_t* tokens; float* logprob;
    int shift;                                            // weights are multiples of 2^-shift: vocab 2^shift <= 2^62
};

constexpr int kSampleThreads = 1024;

// Whole numbers in the order of the logits; -0 and 0 are the same number.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

template <typename V, typename Op>
__device__ V block_reduce(V v, Op op, V* sh) {
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = sh[threadIdx.x & 31];
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(const SampleArgs g) {
    typedef unsigned long long u64;
    __shared__ u64 sh[32];
    __shared__ double shd[32];
    chain_entry();
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(g.logits) + row * g.ld;
    const float warm = g.temperature ? g.temperature[row] : 1.0f;
    const bool greedy = warm <= 0.0f;
    auto sum = [&](auto f) {
        u64 s = 0;
        for (int i = threadIdx.x; i < g.vocab; i += kSampleThreads) s += f(i, to_f32(x[i]) + 0.0f);
        return block_reduce(s, [](u64 a, u64 b) { return a + b; }, sh);
    };
    // the first of the order: largest value, lowest index
    u64 best = 0;
    bool bad = false;
    for (int i = threadIdx.x; i < g.vocab; i += kSampleThreads) {
        const float v = to_f32(x[i]);
        bad |= v != v;
        best = max(best, (u64)order_key(v) << 32 | (uint32_t)~i);
    }
    best = block_reduce(best, [](u64 a, u64 b) { return a > b ? a : b; }, sh);
    bad = __syncthreads_or(bad);
    const float top = key_value((uint32_t)(best >> 32));
    const int first = (int)~(uint32_t)best;
    const float p = g.top_p ? g.top_p[row] : 1.0f, least = g.min_p ? g.min_p[row] : 0.0f, u = greedy ? 0.0f : g.uniform[row];
    bad |= top == -INFINITY || warm != warm || (!greedy && (top == INFINITY || p != p || least != least || u != u));
    int token = first;
    if (!bad && !greedy) {
        const double cool = 1.0 / (double)warm, unit = (double)(1ull << g.shift);
        auto exact = [&](float v) { return exp(((double)v - (double)top) * cool); };
        auto weight = [&](float v) { return v == -INFINITY ? 0ull : max(1ull, (u64)__double2ll_rn(exact(v) * unit)); };
        // kept: keys over `edge`, and those equal to it up to index `cut`
        uint32_t edge = 0;
        int cut = 0x7fffffff;
        auto kept = [&](int i, float v) { const uint32_t k = order_key(v); return k > edge || (k == edge && i <= cut); };
        // the largest edge whose keys and those over it have f's sum at `goal` or more, then the place among its equals
        auto narrow = [&](u64 goal, auto f) {
            uint32_t e = 0;
            for (int bit = 31; bit >= 0; --bit) {
                const uint32_t next = e | 1u << bit;
                if (sum([&](int i, float v) { return kept(i, v) && order_key(v) >= next ? f(v) : 0ull; }) >= goal) e = next;
            }
            const u64 over = sum([&](int i, float v) { return kept(i, v) && order_key(v) > e ? f(v) : 0ull; });
            const u64 each = f(key_value(e));
            const u64 equals = goal > over && each ? (goal - over + each - 1) / each : 0;
            int c = -1;                                    // the largest cut with fewer than `equals` equals before it, plus one
            for (int bit = 30; bit >= 0; --bit) {
                const int next = c + (1 << bit);
                if (next < g.vocab && sum([&](int i, float v) { return (u64)(kept(i, v) && order_key(v) == e && i <= next); }) < equals) c = next;
            }
            edge = e;
            cut = c + 1;
        };
        const int k = g.top_k ? g.top_k[row] : 0;
        if (k > 0 && k < g.vocab) narrow(k, [](float) { return 1ull; });
        if (p < 1.0f) {
            const u64 all = sum([&](int i, float v) { return kept(i, v) ? weight(v) : 0ull; });
            narrow(max(1ull, (u64)ceil((double)fmaxf(p, 0.0f) * (double)all)), weight);
        }
        auto stays = [&](int i, float v) { return kept(i, v) && (i == first || exact(v) >= (double)least); };
        const u64 all = sum([&](int i, float v) { return stays(i, v) ? weight(v) : 0ull; });
        const u64 goal = min((u64)((double)fminf(fmaxf(u, 0.0f), 1.0f) * (double)all), all - 1);
        int c = -1;                                        // the largest index up to which no more than `goal` has come together
        for (int bit = 30; bit >= 0; --bit) {
            const int next = c + (1 << bit);
            if (next < g.vocab && sum([&](int i, float v) { return i <= next && stays(i, v) ? weight(v) : 0ull; }) <= goal) c = next;
        }
        token = c + 1;
    }
    if (threadIdx.x == 0) g.tokens[row] = bad ? -1 : token;
    if (g.logprob) {
        // The first of the order is left out of the sum: where it has nearly all of the probability, its logarithm is that of 1 + the rest.
        double rest = 0.0;
        for (int i = threadIdx.x; !bad && i < g.vocab; i += kSampleThreads)
            if (i != first) rest += exp((double)to_f32(x[i]) - (double)top);
        rest = block_reduce(rest, [](double a, double b) { return a + b; }, shd);
        if (threadIdx.x == 0) g.logprob[row] = bad ? kNaN : (float)(((double)to_f32(x[token]) - (double)top) - log1p(rest));
    }
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_sample(const void* logits, int64_t ld, int dtype, int64_t rows, int64_t vocab,
                          const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* uniform,
                          int64_t* tokens, float* logprob, void* stream) {
    if (rows != 0 && (!logits || !uniform || !tokens)) return MPQ_ERR_NULL;
    if (rows < 0 || rows > 0x7fffffff || vocab <= 0 || (rows > 1 && ld < vocab)) return MPQ_ERR_BAD_SHAPE;
    if (!dtype_ok(dtype) || vocab > 8 * (196608 / dtype_size(dtype))) return MPQ_ERR_UNSUPPORTED;
    if (!aligned_to(logits, dtype_size(dtype)) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) || !aligned_to(top_p, 4) || !aligned_to(min_p, 4) ||
        !aligned_to(uniform, 4) || !aligned_to(tokens, 8) || !aligned_to(logprob, 4)) return MPQ_ERR_ALIGN;
    if (rows == 0) return MPQ_OK;
    int bits = 0;
    while ((int64_t)1 << bits < vocab) ++bits;
    const SampleArgs g = {logits, ld, rows, (int)vocab, temperature, top_k, top_p, min_p, uniform, tokens, logprob, 62 - bits > 50 ? 50 : 62 - bits};
    auto* kernel = dtype == MPQ_F32 ? sample_kernel<float> : dtype == MPQ_F16 ? sample_kernel<__half> : sample_kernel<__nv_bfloat16>;
    return launch_chained_as(true, kernel, (unsigned)rows, kSampleThreads, 0, (cudaStream_t)stream, g);
}
