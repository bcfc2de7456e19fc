// Low-rank adapters beside a product of level bytes: what a request's adapter makes of its tokens before the product's
// epilogue (mpq_linear_adapted).
//
//   z[t][r] = c_id (s_t / L) sum_k (2 u[t][k] - L) D_id[r][k]
//
// The tokens are cut at every sequence's start and at every multiple of a tile's size; a CTA (or a cluster that splits k)
// takes one piece.  Ranks are the rows and tokens the columns of 16 x 8 x 16 matrix instructions, whose operands are exact (odd
// numbers below 2^8, and D itself), with sums in 32 bits.  A lane owns sixteen adjacent k of 64, in both operands alike, so
// that loads are 16 bytes and nothing is staged.  The k range is split over the CTA's warps too; the parts meet in shared
// memory in a fixed order.  Pieces of single tokens: tiles of 8, bound by the latency of the loads (a token with rank 16
// reads 32 k bytes): 64 tokens over 9216 with 48 adapters of rank 16 take 10 us in a graph.  Longer pieces: tiles of 32; 4096
// tokens over 4096 with rank 64 take 28 us, bound by L1 lookups (eight lines a load) and by making the odd numbers, five
// instructions a pair in bfloat16 and three in float16.  (One m-tile a warp, with the next block under way: 31 us; a CTA that
// takes all sequences of its tile in turn: 72.  Tiles of 64 staged by cp.async, one CTA a multiprocessor: 11.5 us for k = 1024, as
// long as two CTAs here take for 32 tokens and k = 2048 each.)
#include "mpq_adapters.cuh"
#include "mpq_tensor.cuh"

namespace mpq {

constexpr int kDownThreads = 256, kDownWarps = kDownThreads / 32;

// Two levels (bytes `at` and `at` + 1 of a word) as the odd numbers 2u - L, in a pair of W.
template <typename W>
__device__ __forceinline__ uint32_t odd_pair(uint32_t word, int at, float L) {
    if constexpr (std::is_same_v<W, __half>) {            // 2^10 + u, twice, in the low bits of a pair
        const uint32_t raised = __byte_perm(word, 0x64646464u, at == 0 ? 0x4140 : 0x4342);
        const __half2 u = __hsub2(*reinterpret_cast<const __half2*>(&raised), __float2half2_rn(1024.0f));
        const __half2 x = __hfma2(u, __float2half2_rn(2.0f), __float2half2_rn(-L));
        return *reinterpret_cast<const uint32_t*>(&x);
    }
    // 1 + 2^-15 u, so that one multiply-add makes the number
    const float a = __uint_as_float(__byte_perm(word, 0x3f800000u, 0x7604u | (uint32_t)at << 4));
    const float b = __uint_as_float(__byte_perm(word, 0x3f800000u, 0x7604u | (uint32_t)(at + 1) << 4));
    const float x = fmaf(65536.0f, a, -65536.0f - L), y = fmaf(65536.0f, b, -65536.0f - L);
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// The piece with number `item`: tokens [from, to) and their sequence (-1: none).  The cuts are the starts of all sequences, the
// end of the last one, and every `tile` tokens, in ascending order (a tile's before a sequence's); cut b of the sequences is
// number b + starts[b] / tile + 1 of all, so that the last one that is not behind the item is found by a search, 32 at a time.
struct Piece { int64_t from, to; int sequence; };
__device__ __forceinline__ Piece piece_of(const AdapterArgs& g, int tile, int64_t item, int lane) {
    auto start = [&](int b) { return min(max((int64_t)g.starts[b], (int64_t)0), g.m); };
    int lo = -1, hi = g.batch + 1;                        // the cut that is looked for is lo or later, and before hi
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 33, b = lo + (lane + 1) * step;
        const bool before = b < hi && b + start(b) / tile + 1 <= item;
        const int n = __popc(__ballot_sync(0xffffffffu, before));
        lo += n * step;
        if (n < 32) hi = min(hi, lo + step);
    }
    Piece p;
    const bool own = lo >= 0 && lo + start(lo) / tile + 1 == item;
    p.from = own ? start(lo) : (item - (lo + 1)) * tile;
    p.to = min((p.from / tile + 1) * tile, g.m);
    if (lo < g.batch) p.to = min(p.to, start(lo + 1));
    p.sequence = lo >= 0 && lo < g.batch ? lo : -1;
    return p;
}

// NT: n-tiles of eight tokens.  MT: m-tiles of 16 ranks that a warp takes; `groups` of warps take all ranks.
template <typename W, int NT, int MT>
__global__ void __launch_bounds__(kDownThreads) adapter_down_kernel(const AdapterArgs g, int splits, int groups) {
    constexpr int kTokens = 8 * NT, kRow = kTokens + 1;   // (a row more than its tokens: ranks are read side by side)
    extern __shared__ float sums[];                       // [k part][rank][kRow]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3;
    const int split = splits > 1 ? (int)cluster_rank() : 0;
    const int parts = kDownWarps / groups, part = warp / groups, r0 = warp % groups * 16 * MT;
    // The product is let in only now: what it reads before it waits for this kernel belongs to those before.
    chain_wait();
    chain_next();
    const Piece piece = piece_of(g, kTokens, blockIdx.x / (unsigned)splits, lane);
    if (piece.from < 0 || piece.from >= piece.to) return; // (in all CTAs of the cluster)
    int id = piece.sequence < 0 ? -1 : g.ids[piece.sequence];
    if (id < 0 || id >= g.adapters) id = -1;
    const int count = (int)(piece.to - piece.from);
    if (split == 0 && threadIdx.x < count) g.low.chosen[piece.from + threadIdx.x] = id;
    if (id < 0) return;
    const W* down = static_cast<const W*>(g.down) + (int64_t)id * g.rank * g.row_bytes;
    const uint8_t* levels = g.a + piece.from * g.row_bytes;
    const int64_t blocks = ceil_div(g.row_bytes, 64);
    const int64_t kb0 = blocks * split / splits, kb1 = blocks * (split + 1) / splits;
    const float L = (float)g.La;
    float acc[MT][NT][4] = {};
    struct Block { uint4 a[MT][2][2], u[NT]; };
    auto ask = [&](int64_t kb, Block& x) {
        const int64_t at = kb * 64 + quad * 16;
        const bool in = kb < kb1 && at < g.row_bytes;
#pragma unroll
        for (int j = 0; j < NT; ++j)
            x.u[j] = in ? load16(levels + min(j * 8 + row, count - 1) * g.row_bytes + at) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = r0 + i * 16 + h * 8 + row;
                const uint4* from = reinterpret_cast<const uint4*>(down + (int64_t)r * g.row_bytes + at);
#pragma unroll
                for (int q = 0; q < 2; ++q) x.a[i][h][q] = in && r < g.rank ? load16(from + q) : make_uint4(0, 0, 0, 0);
            }
    };
    auto multiply = [&](const Block& x) {
#pragma unroll
        for (int s = 0; s < 4; ++s)                       // four of the sixteen k at a time
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint32_t x0 = odd_pair<W>(word_of(x.u[j], s), 0, L), x1 = odd_pair<W>(word_of(x.u[j], s), 2, L);
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    mma_16x8x16<W>(acc[i][j], word_of(x.a[i][0][s >> 1], 2 * (s & 1)), word_of(x.a[i][1][s >> 1], 2 * (s & 1)),
                                   word_of(x.a[i][0][s >> 1], 2 * (s & 1) + 1), word_of(x.a[i][1][s >> 1], 2 * (s & 1) + 1), x0, x1);
            }
    };
    if constexpr (NT == 1) {                              // several blocks on their way: these pieces are bound by latency
        constexpr int kAhead = MT == 1 ? 4 : 2;
        for (int64_t kb = kb0 + part; kb < kb1; kb += kAhead * parts) {
            Block x[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) ask(kb + q * parts, x[q]);
#pragma unroll
            for (int q = 0; q < kAhead; ++q) multiply(x[q]);
        }
    } else if constexpr (MT == 2) {                       // (a second block would not fit beside the first)
        for (int64_t kb = kb0 + part; kb < kb1; kb += parts) {
            Block x;
            ask(kb, x);
            multiply(x);
        }
    } else {
        Block next;
        ask(kb0 + part, next);
        for (int64_t kb = kb0 + part; kb < kb1; kb += parts) {
            const Block x = next;
            ask(kb + parts, next);
            multiply(x);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = r0 + i * 16 + (e >> 1) * 8 + row;
                if (r < g.rank) sums[(part * g.rank + r) * kRow + j * 8 + quad * 2 + (e & 1)] = acc[i][j][e];
            }
    __syncthreads();
    for (int i = threadIdx.x; i < g.rank * kRow; i += kDownThreads) {
        float s = sums[i];
        for (int p = 1; p < parts; ++p) s += sums[p * g.rank * kRow + i];
        sums[i] = s;
    }
    if (splits > 1) cluster_sync_all();
    else __syncthreads();
    // A warp a token: its share of the tokens, the ranks side by side.
    for (int t = split * kDownWarps + warp; t < count; t += splits * kDownWarps) {
        const int64_t token = piece.from + t;
        const float c = __fdiv_rn(g.a_scale[token], L) * (g.factor ? g.factor[id] : 1.0f);
        constexpr int kMost = 4;                          // 128 ranks
        float z[kMost], top = 0.0f;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const int r = i * 32 + lane;
            z[i] = 0.0f;
            if (r >= g.rank) continue;
            float s = 0.0f;
            for (int q = 0; q < splits; ++q) {
                float v;
                if (splits > 1) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(map_to_cta(smem_addr(sums + r * kRow + t), (uint32_t)q)) : "memory");
                else v = sums[r * kRow + t];
                s += v;
            }
            z[i] = s * c;
            top = max_nan(top, fabsf(z[i]));
            g.low.z[token * g.rank + r] = z[i];
        }
        for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
        int e = 0;
        if (std::is_same_v<W, __half> && ordinary(top) && top > 0.0f) e = max(ilogbf(top) - 14, -126);
        if (lane == 0) g.low.scale[token] = ldexpf(1.0f, e);
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const int r = i * 32 + lane;
            if (r >= g.rank) continue;
            float left = ldexpf(z[i], -e);
#pragma unroll
            for (int q = 0; q < (std::is_same_v<W, __half> ? 2 : kLowParts); ++q) {
                const W w = from_f32<W>(left);
                reinterpret_cast<W*>(g.low.parts)[((int64_t)q * g.m + token) * g.rank + r] = w;
                left -= to_f32(w);
                if (!ordinary(left)) left = 0.0f;         // of an infinity nothing is left
            }
        }
    }
    if (splits > 1) cluster_sync_all();                   // nobody leaves while others read its sums
}

template <typename W, int NT, int MT>
int launch_down(const AdapterArgs& g, int groups, cudaStream_t st) {
    const int parts = kDownWarps / groups;
    const size_t smem = (size_t)parts * g.rank * (8 * NT + 1) * sizeof(float);        // 33 KB at most
    const int sms = sm_count();
    if (sms == 0) return MPQ_ERR_CUDA;
    const int64_t items = ceil_div(g.m, 8 * NT) + g.batch + 1, blocks = ceil_div(g.row_bytes, 64);
    if (items > 0x7fffffff / 8) return MPQ_ERR_BAD_SHAPE;
    // more splits of k while they fit the device together and a warp has two blocks of 64
    int splits = 1;
    while (splits < 8 && items * splits <= sms && blocks >= (int64_t)parts * splits * 2) splits *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(splits * items), 1, 1);
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
    const int tiles = g.rank / 16;
    if (g.m <= 8 * (int64_t)(g.batch > 0 ? g.batch : 1))  // pieces of up to 8 tokens on average
        return tiles == 1 ? launch_down<W, 1, 1>(g, 1, st) : launch_down<W, 1, 2>(g, tiles / 2, st);
    return tiles == 1 ? launch_down<W, 4, 1>(g, 1, st) : launch_down<W, 4, 2>(g, tiles / 2, st);
}

int adapter_down(const AdapterArgs& g, int dtype, cudaStream_t st) {
    return dtype == MPQ_F16 ? adapter_down_typed<__half>(g, st) : adapter_down_typed<__nv_bfloat16>(g, st);
}

}  // namespace mpq
