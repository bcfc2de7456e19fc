// Low-rank adapters beside a product of level bytes: what a request's adapter makes of its tokens before the product's
// epilogue (mpq_linear_adapted).
//
//   z[t][r] = c_id (s_t / L) sum_k (2 u[t][k] - L) D_id[r][k]
//
// A CTA takes a tile of tokens and one sequence at a time of those that lie in it; ranks are the rows and tokens the
// columns of 16 x 8 x 16 matrix instructions, whose operands are exact (odd numbers below 2^8, and D itself), with sums in
// 32 bits.  Lanes own eight adjacent k of 32, in both operands alike, so that loads are 16 and 8 bytes and nothing is staged.
// The k range is split over the CTA's warps and a cluster of CTAs; the parts meet in shared memory in a fixed order.
// Single tokens and other short pieces: tiles of 8 tokens and a CTA for each piece in them, bound by the latency of the
// loads (a token with rank 16 reads 32 k bytes).  Long pieces: tiles of 32.
#include "mpq_adapters.cuh"
#include "mpq_tensor.cuh"

namespace mpq {

constexpr int kDownThreads = 256, kDownWarps = kDownThreads / 32;

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
__device__ __forceinline__ int adapter_of(const AdapterArgs& g, int b) {
    const int id = b < 0 ? -1 : g.ids[b];
    return id >= g.adapters ? -1 : id;
}

// Two levels (bytes at `at` and above of a word) as the odd numbers 2u - L, in a pair of W.
template <typename W>
__device__ __forceinline__ uint32_t odd_pair(uint32_t word, int at, float L) {
    const float a = __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7650u + (uint32_t)at)) - 8388608.0f;
    const float b = __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7651u + (uint32_t)at)) - 8388608.0f;
    const float x = fmaf(2.0f, a, -L), y = fmaf(2.0f, b, -L);
    uint32_t r;
    if constexpr (sizeof(W) == 2 && std::is_same_v<W, __half>) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
}
template <typename W>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same_v<W, __half>)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NT: n-tiles of eight tokens.  MT: m-tiles of 16 ranks that a warp takes; rank / (16 MT) groups of warps take all of them.
template <typename W, int NT, int MT>
__global__ void __launch_bounds__(kDownThreads) adapter_down_kernel(const AdapterArgs g, int splits, int groups) {
    constexpr int kTokens = 8 * NT, kRow = kTokens + 1;   // (a row more than its tokens: ranks are read side by side)
    extern __shared__ float sums[];                       // [k part][rank][kRow]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3;
    const int split = splits > 1 ? (int)cluster_rank() : 0;
    const int64_t t0 = (int64_t)(blockIdx.x / (unsigned)splits) * kTokens;
    const int parts = kDownWarps / groups, part = warp / groups, r0 = warp % groups * 16 * MT;
    chain_entry();
    if (split == 0 && blockIdx.y == 0 && threadIdx.x < kTokens && t0 + threadIdx.x < g.m)
        g.chosen[t0 + threadIdx.x] = adapter_of(g, sequence_of(g.starts, g.batch, t0 + threadIdx.x));
    // the first sequence that has something in this tile
    const int64_t begin = g.batch > 0 ? max((int64_t)g.starts[0], t0) : t0 + kTokens, end = min(t0 + kTokens, g.m);
    int b = begin < end ? sequence_of(g.starts, g.batch, begin) : -1;
    if (b < 0) return;                                    // (in all CTAs of the cluster)
    b += blockIdx.y;
    const int64_t blocks = ceil_div(g.row_bytes, 32);
    const int64_t kb0 = blocks * split / splits, kb1 = blocks * (split + 1) / splits;
    for (; b < g.batch && g.starts[b] < end; b += gridDim.y) {
        const int64_t from = max(t0, (int64_t)g.starts[b]), to = min(end, (int64_t)g.starts[b + 1]);
        const int id = adapter_of(g, b);
        if (id < 0 || from >= to) continue;
        const W* down = static_cast<const W*>(g.down) + (int64_t)id * g.rank * g.row_bytes;
        float acc[MT][NT][4] = {};
        for (int64_t kb = kb0 + part; kb < kb1; kb += parts) {
            const int64_t at = kb * 32 + quad * 8;
            const bool in = at < g.row_bytes;
            uint4 a[MT][2];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = r0 + i * 16 + h * 8 + row;
                    a[i][h] = in && r < g.rank ? __ldg(reinterpret_cast<const uint4*>(down + (int64_t)r * g.row_bytes + at)) : make_uint4(0, 0, 0, 0);
                }
            uint2 u[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j)
                u[j] = in ? __ldg(reinterpret_cast<const uint2*>(g.a + min(t0 + j * 8 + row, g.m - 1) * g.row_bytes + at)) : make_uint2(0, 0);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint32_t x0 = odd_pair<W>(u[j].x, 0, (float)g.La), x1 = odd_pair<W>(u[j].x, 2, (float)g.La);
                const uint32_t x2 = odd_pair<W>(u[j].y, 0, (float)g.La), x3 = odd_pair<W>(u[j].y, 2, (float)g.La);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    mma_16x8x16<W>(acc[i][j], a[i][0].x, a[i][1].x, a[i][0].y, a[i][1].y, x0, x1);
                    mma_16x8x16<W>(acc[i][j], a[i][0].z, a[i][1].z, a[i][0].w, a[i][1].w, x2, x3);
                }
            }
        }
        __syncthreads();                                  // the sums of the sequence before have been read
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = r0 + i * 16 + (e >> 1) * 8 + row;
                    if (r < g.rank) sums[(part * g.rank + r) * kRow + j * 8 + quad * 2 + (e & 1)] = acc[i][j][e];
                }
        if (splits > 1) cluster_sync_all();
        else __syncthreads();
        // each CTA of the cluster finishes a share of the numbers
        const int all = g.rank * kTokens;
        for (int i = split * kDownThreads + threadIdx.x; i < all; i += splits * kDownThreads) {
            // neighbours in z are ranks of a token
            const int t = i / g.rank, r = i % g.rank;
            if (t0 + t < from || t0 + t >= to) continue;
            float s = 0.0f;
            for (int c = 0; c < splits; ++c)
                for (int p = 0; p < parts; ++p) {
                    const float* from_part = sums + (p * g.rank + r) * kRow + t;
                    float v;
                    if (splits > 1) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(map_to_cta(smem_addr(from_part), (uint32_t)c)) : "memory");
                    else v = *from_part;
                    s += v;
                }
            g.z[(t0 + t) * g.rank + r] = s * (__fdiv_rn(g.a_scale[t0 + t], (float)g.La) * (g.factor ? g.factor[id] : 1.0f));
        }
        if (splits > 1) cluster_sync_all();               // nobody overwrites or gives up what others still read
    }
}

template <typename W, int NT, int MT>
int launch_down(const AdapterArgs& g, int slots, int groups, cudaStream_t st) {
    const int parts = kDownWarps / groups;
    const size_t smem = (size_t)parts * g.rank * (8 * NT + 1) * sizeof(float);        // 33 KB at most
    const int sms = sm_count();
    if (sms == 0) return MPQ_ERR_CUDA;
    const int64_t tiles = ceil_div(g.m, 8 * NT), blocks = ceil_div(g.row_bytes, 32);
    // more splits of k while they fit the device together and a warp has two blocks of 32
    int splits = 1;
    if (tiles > 0x7fffffff / 8) return MPQ_ERR_BAD_SHAPE;
    while (splits < 8 && tiles * slots * splits * 2 <= 2 * sms && blocks >= (int64_t)parts * splits * 4) splits *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(splits * tiles), (unsigned)slots, 1);
    cfg.blockDim = dim3(kDownThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, adapter_down_kernel<W, NT, MT>, g, splits, groups) != cudaSuccess) { cudaGetLastError(); return MPQ_ERR_CUDA; }
    return launch_status();
}

template <typename W>
int adapter_down_typed(const AdapterArgs& g, cudaStream_t st) {
    const int tiles = g.rank / 16, groups = tiles <= 2 ? 1 : tiles <= 4 ? 2 : 4;         // two m-tiles to a warp
    // pieces of up to 8 tokens on average: a CTA for each of a tile's eight possible pieces
    if (g.m <= 8 * (int64_t)(g.batch > 0 ? g.batch : 1) || g.m <= 8) {
        const int slots = g.m < 8 ? (int)g.m : 8;
        return tiles == 1 ? launch_down<W, 1, 1>(g, slots, 1, st) : launch_down<W, 1, 2>(g, slots, groups, st);
    }
    return tiles == 1 ? launch_down<W, 4, 1>(g, 1, 1, st) : launch_down<W, 4, 2>(g, 1, groups, st);
}

int adapter_down(const AdapterArgs& g, int dtype, cudaStream_t st) {
    return dtype == MPQ_F16 ? adapter_down_typed<__half>(g, st) : adapter_down_typed<__nv_bfloat16>(g, st);
}

}  // namespace mpq
