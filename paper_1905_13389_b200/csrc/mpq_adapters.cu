// Low-rank adapters beside a product of level bytes: what a request's adapter makes of its tokens before the product's
// epilogue (mpq_linear_adapted).
//
//   z[t][r] = c_id (s_t / L) sum_k (2 u[t][k] - L) D_id[r][k]
#include "mpq_adapters.cuh"

namespace mpq {

// Sequence of token t, -1 for a token of none: the last one that starts at t or before.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int batch, int64_t t) {
    if (batch <= 0 || t < starts[0] || t >= starts[batch]) return -1;
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename W>
__global__ void __launch_bounds__(256) adapter_down_kernel(const AdapterArgs g) {
    chain_entry();
    const int64_t t = blockIdx.x;
    const int b = sequence_of(g.starts, g.batch, t);
    int id = b < 0 ? -1 : g.ids[b];
    if (id >= g.adapters) id = -1;
    if (threadIdx.x == 0) g.chosen[t] = id;
    if (id < 0) return;
    const uint8_t* u = g.a + t * g.row_bytes;
    const float s = __fdiv_rn(g.a_scale[t], (float)g.La) * (g.factor ? g.factor[id] : 1.0f);
    for (int r = threadIdx.x >> 5; r < g.rank; r += 8) {
        const W* d = static_cast<const W*>(g.down) + ((int64_t)id * g.rank + r) * g.row_bytes;
        float sum = 0.0f;
        for (int64_t i = threadIdx.x & 31; i < g.k; i += 32) sum = fmaf((float)(2 * (int)u[i] - g.La), to_f32(d[i]), sum);
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if ((threadIdx.x & 31) == 0) g.z[t * g.rank + r] = s * sum;
    }
}

int adapter_down(const AdapterArgs& g, int dtype, cudaStream_t st) {
    auto* kernel = dtype == MPQ_F16 ? adapter_down_kernel<__half> : adapter_down_kernel<__nv_bfloat16>;
    return launch_chained_as(true, kernel, (unsigned)g.m, 256, 0, st, g);
}

}  // namespace mpq
