// Product of level bytes with bias, activation and residual in its epilogue (mpq_linear_levels).
//
// With q = 2u - L (Eq. 16) the layer's integer product is
//   sum q_a q_w = 4 sum u_a u_w - 2 L_w sum u_a - 2 L_a sum u_w + k L_a L_w,
// so the inner loop multiplies unsigned bytes and the level sums that lie beside the operands do the rest.
// The result fits int32 (checked on the host), hence the terms may be combined modulo 2^32.
#include "mpq_attention.cuh"
#include "mpq_tensor.cuh"

#include <atomic>
#include <type_traits>

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
    uint32_t polls;                                       // limit of a wait
};

// acc (levels u, unsigned) -> one output, in the header's order of operations
struct RowTerm { float scale; uint32_t term; };          // a_scale / L_a;  k L_a L_w - 2 L_w sums_a
struct ColTerm { float scale; uint32_t term; float bias; };   // w_scale / L_w;  2 L_a sums_w;  bias
__device__ __forceinline__ RowTerm row_term(const LinearArgs& g, int64_t r) {
    RowTerm t;
    t.scale = __fdiv_rn(__ldg(g.a_scale + r), (float)g.La);
    t.term = (uint32_t)g.k * (uint32_t)g.La * (uint32_t)g.Lw - 2u * (uint32_t)g.Lw * (uint32_t)__ldg(g.a_sums + r);
    return t;
}
__device__ __forceinline__ ColTerm col_term(const LinearArgs& g, int64_t c) {
    ColTerm t;
    t.scale = __fdiv_rn(__ldg(g.w_scale + c), (float)g.Lw);
    t.term = 2u * (uint32_t)g.La * (uint32_t)__ldg(g.w_sums + c);
    t.bias = g.bias ? __ldg(g.bias + c) : 0.0f;
    return t;
}
__device__ __forceinline__ float linear_value(const LinearArgs& g, uint32_t acc, const RowTerm& r, const ColTerm& c) {
    const float f = (float)(int32_t)(4u * acc + r.term - c.term) * (r.scale * c.scale);
    return g.bias ? f + c.bias : f;
}
// f Phi(f), with Phi(-|f|) = erfc(|f| / sqrt 2) / 2 made as a product, so that negative f keep their relative precision
// (0.5 f (1 + erf) cancels: it lost several percent of the result at -5 and all of it below -5.6).  erfc(z) e^(z^2) / 2 is
// a polynomial in t = 1 / (1 + 0.43 z), fitted here to the least largest relative error over z in [0, 10], 1.0e-7; with fp32
// roundings the relative error is 2.6e-6 for f down to -8, most of it from the rounded exponent.
// (erfcf: 73.9 us at 4096^3, 61.0 with this; 0.5 f (1 + erff) took 63.3.)
__device__ __forceinline__ float gelu(float f) {
    const float t = __fdividef(1.0f, fmaf(fabsf(f), 0.43f * 0.70710678f, 1.0f));
    float q = 0.036572885f;
    q = fmaf(q, t, -0.15404773f);
    q = fmaf(q, t, 0.18994352f);
    q = fmaf(q, t, -0.041152050f);
    q = fmaf(q, t, 0.12254029f);
    q = fmaf(q, t, 0.10273626f);
    q = fmaf(q, t, 0.12214691f);
    q = fmaf(q, t, 0.12125991f);
    const float below = q * t * fast_exp2(f * f * -0.72134752f);         // Phi(-|f|); log2(e) / 2
    return f * (f >= 0.0f ? 1.0f - below : below);
}
// The activation of N values at once: one (uniform) branch for all of them, so their chains overlap.  SiLU and the tanh form
// use the fast exponential and quotient also for fp32 results: between -8 and -3 they are off by 0.4e-6 and 3.3e-6 of the
// result (measured).
template <int N>
__device__ __forceinline__ void glue_values(float (&f)[N], int glue) {
    if (glue == MPQ_GLUE_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = max_nan(f[i], 0.0f);       // a NaN range stays visible, as under the other activations
    } else if (glue == MPQ_GLUE_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = gelu(f[i]);
    } else if (glue == MPQ_GLUE_GELU_TANH) {
        // 0.5 f (1 + tanh z) = f / (1 + e^(-2z)); the exponential saturates to 0 or infinity, the quotient to f or 0
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float z2 = 1.5957691216057308f * (f[i] + 0.044715f * f[i] * f[i] * f[i]);
            f[i] = __fdividef(f[i], 1.0f + __expf(-z2));
        }
    } else if (glue == MPQ_GLUE_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = __fdividef(f[i], 1.0f + __expf(-f[i]));
    }
}

constexpr int kBlock = 128;                               // bytes of k per stage: one swizzled row
constexpr int kThreads = 192;                             // warp 0 loads, warp 1 issues the products, warps 2-5 store

__device__ unsigned int g_wait_failures;                  // waits that ran out, over the life of the process

// ---- few rows: C^T = W A^T.  The 128 rows of a tile are weight rows (output columns), its BN columns are
// activation rows, so a handful of tokens wastes nothing of the 128 TMEM lanes and the weights are read once.
// These products are bound by reading the weights; with one CTA per multiprocessor and a ring of 130-180 KB
// the loads of a whole multiprocessor stay in flight.  Too few tiles for all multiprocessors: the k range of a
// tile is split over a cluster of S CTAs, which exchange their integer partial sums through distributed
// shared memory (exact, so any order gives the same result) -- CTA i finishes rows i BN/S .. of the tile.
template <int BN> struct SmallShape {
    static constexpr int stages = BN == 16 ? 10 : BN == 32 ? 8 : 6;
    static constexpr int stage_bytes = (128 + BN) * kBlock;
    static constexpr int exchange_bytes = BN * 128 * 4;   // [S source CTAs][BN / S rows][128 columns] int32
    static constexpr int smem = stages * stage_bytes + exchange_bytes + 1024;
};

// `count` of N results of one column, rows r .. : the residuals are all read before the first result is written
// (they may be the same tensor, so the compiler cannot move a load over a store).
template <typename T, int N>
__device__ __forceinline__ void store_column(const LinearArgs& g, float (&f)[N], int64_t r, int64_t c, int count) {
    if (c >= g.n) return;
    if (g.res) {
        const T* res = static_cast<const T*>(g.res) + r * g.ldr + c;
        T v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) if (j < count) v[j] = res[j * g.ldr];
#pragma unroll
        for (int j = 0; j < N; ++j) if (j < count) f[j] += to_f32(v[j]);
    }
    T* out = static_cast<T*>(g.out) + r * g.ldo + c;
#pragma unroll
    for (int j = 0; j < N; ++j) if (j < count) out[j * g.ldo] = from_f32<T>(f[j]);
}

template <typename T, int BN>
__global__ void __launch_bounds__(kThreads, 1)
linear_small_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a, const LinearArgs g,
                    int tiles_w, int splits) {
    using Shape = SmallShape<BN>;
    constexpr int kStages = Shape::stages;
    constexpr uint32_t kCols = BN < 32 ? 32 : BN;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 1];
    __shared__ uint32_t tmem_holder;
    __shared__ int failed, peer_failed;                   // a wait of this CTA, or a store of its cluster, gave up
    __shared__ float row_scale[BN];
    __shared__ uint32_t row_terms[BN];
    const uint32_t ring = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t exchange = ring + kStages * Shape::stage_bytes;
    uint32_t* exchange_ptr = reinterpret_cast<uint32_t*>(smem_raw + (exchange - smem_addr(smem_raw)));
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    auto full = [&](int s) { return smem_addr(&bars[s]); };
    auto empty = [&](int s) { return smem_addr(&bars[kStages + s]); };
    const uint32_t done = smem_addr(&bars[2 * kStages]);
    auto has_failed = [&]() { return *(volatile int*)&failed != 0; };

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2 * kStages + 1; ++i) mbar_init(smem_addr(&bars[i]), 1);
        failed = peer_failed = 0;
        mbar_init_fence();
        tma_prefetch(&map_w);
        tma_prefetch(&map_a);
    }
    if (warp == 0) tmem_alloc<1>(&tmem_holder, kCols);
    tmem_fence_before();
    if (splits > 1) cluster_sync_all();                   // the other CTAs' shared memory is there
    else __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_holder;
    chain_entry();

    const int split = splits > 1 ? (int)cluster_rank() : 0;
    const int tile = (int)blockIdx.x / splits;
    const int n0 = tile % tiles_w * 128, m0 = tile / tiles_w * BN;
    const int blocks = (int)((g.row_bytes + kBlock - 1) / kBlock);
    const int kb0 = (int)((int64_t)blocks * split / splits), kb1 = (int)((int64_t)blocks * (split + 1) / splits);

    if (warp == 0) {
        const bool leader = elect_one();
        int i = 0;
        for (int kb = kb0; kb < kb1; ++kb, ++i) {
            const int s = i % kStages;
            if (i >= kStages && !mbar_wait_warp(empty(s), (i / kStages - 1) & 1, &failed, g.polls)) break;
            if (leader) {
                const uint32_t dst = ring + s * Shape::stage_bytes;
                mbar_expect_tx(full(s), Shape::stage_bytes);
                tma_load_2d(dst, &map_w, kb * kBlock, n0, full(s));
                tma_load_2d(dst + 128 * kBlock, &map_a, kb * kBlock, m0, full(s));
            }
        }
        // Every copy has landed before the CTA ends, also where the products have given up on them.
        for (int q = i > kStages ? i - kStages : 0; q < i; ++q) mbar_wait(full(q % kStages), (q / kStages) & 1);
    } else if (warp == 1) {
        constexpr uint32_t idesc = umma_idesc_u8(128, BN);
        const bool leader = elect_one();
        const uint32_t d = __shfl_sync(0xffffffffu, tmem, 0);
        int i = 0;
        for (int kb = kb0; kb < kb1; ++kb, ++i) {
            const int s = i % kStages;
            if (!mbar_wait_warp(full(s), (i / kStages) & 1, &failed, g.polls)) break;
            tmem_fence_after();
            const uint32_t at = ring + s * Shape::stage_bytes;
            if (leader) {
                const uint64_t da = umma_desc(at), db = umma_desc(at + 128 * kBlock);
#pragma unroll
                for (int j = 0; j < kBlock / 32; ++j) umma_u8<1>(d, da + 2 * j, db + 2 * j, idesc, i > 0 || j > 0);
                umma_commit<1>(empty(s));
            }
        }
        if (leader) umma_commit<1>(done);
    } else if (warp >= 2) {
        // constants of the tile's rows while the products run
        const int t = threadIdx.x - 64;
        for (int r = t; r < BN; r += 128) {
            RowTerm rt = {0.0f, 0u};
            if (m0 + r < g.m) rt = row_term(g, m0 + r);
            row_scale[r] = rt.scale;
            row_terms[r] = rt.term;
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        const int quarter = warp & 3;
        const int col = quarter * 32 + lane;              // TMEM lane = weight row = output column
        const int64_t c = (int64_t)n0 + col;
        ColTerm ct = {0.0f, 0u, 0.0f};
        if (c < g.n) ct = col_term(g, c);
        bool ok = mbar_wait_warp(done, 0, &failed, g.polls);
        if (!ok) mbar_wait(done, 0);                      // what has been issued must end before TMEM is freed
        ok = ok && !__any_sync(0xffffffffu, has_failed());
        if (!ok) {                                        // results are NaN from here on, in all CTAs of the tile
            ct.scale = kNaN;
            if (splits > 1 && lane < splits) st_cluster(map_to_cta(smem_addr(&peer_failed), (uint32_t)lane), 1u);
        }
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        const int own = BN / splits;
        {
            tmem_fence_after();
#pragma unroll 1
            for (int r0 = 0; r0 < BN; r0 += 16) {
                uint32_t v[16];
                tmem_load16(lanes + r0, v);
                tmem_wait_ld();
                if (splits == 1) {
                    float f[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) f[j] = linear_value(g, v[j], RowTerm{row_scale[r0 + j], row_terms[r0 + j]}, ct);
                    glue_values(f, g.glue);
                    store_column<T, 16>(g, f, (int64_t)m0 + r0, c, (int)min((int64_t)16, g.m - m0 - r0));
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int r = r0 + j, owner = r / own;
                        st_cluster(map_to_cta(exchange + (uint32_t)(((split * own + r % own) * 128 + col) * 4), (uint32_t)owner), v[j]);
                    }
                }
            }
        }
        tmem_fence_before();
    }
    __syncwarp();
    if (splits > 1) {
        cluster_sync_all();                                // every CTA's partial sums have arrived
        if (warp >= 2) {
            const int col = (warp & 3) * 32 + lane, own = BN / splits;
            const int64_t c = (int64_t)n0 + col;
            if (c < g.n) {
                ColTerm ct = col_term(g, c);
                if (*(volatile int*)&peer_failed) ct.scale = kNaN;
                auto finish = [&](auto count, int j0) {    // `count` rows of this CTA's share at once
                    constexpr int N = decltype(count)::value;
                    const int rr = split * own + j0;
                    if (m0 + rr >= g.m) return;
                    float f[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        uint32_t acc = 0;
                        for (int s = 0; s < splits; ++s) acc += exchange_ptr[(s * own + j0 + j) * 128 + col];
                        f[j] = linear_value(g, acc, RowTerm{row_scale[rr + j], row_terms[rr + j]}, ct);
                    }
                    glue_values(f, g.glue);
                    store_column<T, N>(g, f, (int64_t)m0 + rr, c, (int)min((int64_t)N, g.m - m0 - rr));
                };
                // own is a power of two, 2 or more: every batch lies inside this CTA's share
                if (own >= 16) for (int j0 = 0; j0 < own; j0 += 16) finish(std::integral_constant<int, 16>(), j0);
                else if (own >= 4) for (int j0 = 0; j0 < own; j0 += 4) finish(std::integral_constant<int, 4>(), j0);
                else finish(std::integral_constant<int, 2>(), 0);
            }
        }
    }
    __syncthreads();
    tmem_fence_after();
    if (warp == 0) tmem_free<1>(tmem, kCols);
    if (threadIdx.x == 0 && failed) atomicAdd(&g_wait_failures, 1u);
}

// ---- many rows: 256 x 128 tiles on CTA pairs (cta_group::2).  The pair shares the 128 operand rows of the weights,
// each CTA holds half of them and 128 of the 256 activation rows.  Persistent: pair p takes tiles p, p + pairs, ...;
// two accumulators in TMEM, so a tile is stored while the next one is multiplied.  The store goes through a
// shared-memory transpose, after which a lane owns two columns (their constants in registers) and a warp writes whole
// row pieces whatever the row stride is.  Sixteen warps store (eight: 60.2 us for 57.7 at 4096^3, 45.9 for 41.5 at
// 777 x 5001 x 4100 with an unaligned residual and output).
// What bounds it: the operands' way from L2, 24 KB per CTA and 128 bytes of k, some 45 bytes a cycle and multiprocessor;
// 4096^3 with bias and GELU (tanh form) takes 57.3 us, 2.40 POP/s.  256 x 256 tiles read a quarter less but leave the last of their
// 3.5 rounds half empty (62 us for 61 with eight storing warps; 1024 x 4096 x 4096 23.5 for 22.0).
constexpr int kPairStoreWarps = 16;                       // four per quarter of the TMEM lanes: two for each half of the columns
constexpr int kPairThreads = 64 + 32 * kPairStoreWarps;
constexpr int kPairCols = 128;
struct PairShape {
    static constexpr int stage_bytes = (128 + kPairCols / 2) * kBlock;   // per CTA
    static constexpr int stages = 6;
    static constexpr int row_words = 64;                            // column pair p of row r lies at pair p ^ r: no bank conflicts either way
    static constexpr int transpose_bytes = kPairStoreWarps / 2 * 32 * row_words * 4;
    static constexpr int smem = stages * stage_bytes + transpose_bytes + 1024;
};

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w, const LinearArgs g,
                   int tiles_m, int tiles) {
    using Shape = PairShape;
    constexpr int BN = kPairCols, kStages = Shape::stages, kAccs = 2;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 2 * kAccs + 1];
    __shared__ uint32_t tmem_holder;
    __shared__ int failed, peer_failed;                    // a wait of this CTA, or of the other one, gave up
    const uint32_t ring = (smem_addr(smem_raw) + 1023u) & ~1023u;
    uint32_t* transpose = reinterpret_cast<uint32_t*>(smem_raw + (ring - smem_addr(smem_raw)) + kStages * Shape::stage_bytes);
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    auto full = [&](int s) { return smem_addr(&bars[s]); };                        // used in the leader (rank 0)
    auto empty = [&](int s) { return smem_addr(&bars[kStages + s]); };             // one in each CTA
    auto acc_full = [&](int a) { return smem_addr(&bars[2 * kStages + a]); };      // one in each CTA
    auto acc_empty = [&](int a) { return smem_addr(&bars[2 * kStages + kAccs + a]); };   // leader: the storing warps of both
    const uint32_t drained = smem_addr(&bars[2 * kStages + 2 * kAccs]);            // one in each CTA; used after a failure
    auto has_failed = [&]() { return *(volatile int*)&failed != 0; };

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2 * kStages + kAccs; ++i) mbar_init(smem_addr(&bars[i]), 1);
        for (int a = 0; a < kAccs; ++a) mbar_init(acc_empty(a), 2 * kPairStoreWarps);
        mbar_init(drained, 1);
        failed = peer_failed = 0;
        mbar_init_fence();
        tma_prefetch(&map_a);
        tma_prefetch(&map_w);
    }
    if (warp == 0) tmem_alloc<2>(&tmem_holder, kAccs * BN);
    tmem_fence_before();
    cluster_sync_all();                                    // both CTAs' barriers exist
    tmem_fence_after();
    const uint32_t tmem = tmem_holder;
    chain_entry();

    const int pair = (int)blockIdx.x / 2, pairs = (int)gridDim.x / 2;
    const int my_tiles = tiles > pair ? (tiles - pair + pairs - 1) / pairs : 0;
    const int blocks = (int)((g.row_bytes + kBlock - 1) / kBlock);
    // consecutive tiles share their weight rows: what a round of pairs reads of them stays in L2
    auto origin = [&](int i, int& m0, int& n0) {
        const int t = pair + i * pairs;
        m0 = t % tiles_m * 256;
        n0 = t / tiles_m * BN;
    };

    if (warp == 0) {
        const bool leader = elect_one();
        int issued = 0;
        bool ok = true;
        for (int i = 0; i < my_tiles && ok; ++i) {
            int m0, n0;
            origin(i, m0, n0);
            for (int kb = 0; kb < blocks; ++kb, ++issued) {
                const int s = issued % kStages;
                if (issued >= kStages && !mbar_wait_warp(empty(s), (issued / kStages - 1) & 1, &failed, g.polls)) { ok = false; break; }
                if (leader) {
                    const uint32_t dst = ring + s * Shape::stage_bytes, bar = map_to_cta(full(s), 0);
                    if (rank == 0) mbar_expect_tx(full(s), 2 * Shape::stage_bytes);
                    tma_load_2d_pair(dst, &map_a, kb * kBlock, m0 + (int)rank * 128, bar);
                    tma_load_2d_pair(dst + 128 * kBlock, &map_w, kb * kBlock, n0 + (int)rank * (BN / 2), bar);
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc = umma_idesc_u8(256, BN);
            const bool leader = elect_one();
            const uint32_t acc_base = __shfl_sync(0xffffffffu, tmem, 0);
            int consumed = 0;
            bool ok = true;
            for (int i = 0; i < my_tiles && ok; ++i) {
                const int acc = i & 1;
                if (i >= kAccs && !mbar_wait_warp(acc_empty(acc), ((i >> 1) - 1) & 1, &failed, g.polls)) break;
                tmem_fence_after();
                const uint32_t d = acc_base + (uint32_t)(acc * BN);
                for (int kb = 0; kb < blocks; ++kb, ++consumed) {
                    const int s = consumed % kStages;
                    if (!mbar_wait_warp(full(s), (consumed / kStages) & 1, &failed, g.polls)) { ok = false; break; }
                    tmem_fence_after();
                    const uint32_t at = ring + s * Shape::stage_bytes;
                    if (leader) {
                        const uint64_t da = umma_desc(at), db = umma_desc(at + 128 * kBlock);
#pragma unroll
                        for (int j = 0; j < kBlock / 32; ++j) umma_u8<2>(d, da + 2 * j, db + 2 * j, idesc, kb > 0 || j > 0);
                        umma_commit<2>(empty(s));
                    }
                }
                if (leader && ok) umma_commit<2>(acc_full(acc));        // a sum that is not complete is never handed over
            }
        }
    } else if (warp >= 2) {
        // two warps share 32 rows of 64 columns: each brings half of the columns into the transpose and stores half of the rows
        const int quarter = warp & 3, half = (warp - 2) >> 3, part = ((warp - 2) >> 2) & 1;
        const int block = half * 4 + quarter, c0 = half * (BN / 2);
        uint32_t* sh = transpose + block * 32 * Shape::row_words;
        auto block_sync = [&] { asm volatile("bar.sync %0, 64;" ::"r"(1 + block) : "memory"); };
        auto block_all = [&](bool mine) {                  // ... and whether it holds in both warps
            uint32_t all;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.and.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                         : "=r"(all) : "r"(1 + block), "r"((uint32_t)mine) : "memory");
            return all != 0;
        };
        bool ok = true;
        const T* res = static_cast<const T*>(g.res);
        T* out = static_cast<T*>(g.out);
        // Where rows start on a multiple of two elements a lane owns two adjacent columns, elsewhere columns 32 apart
        // (its accesses are then single elements, side by side across the warp).
        const bool twos = (reinterpret_cast<uintptr_t>(out) % (2 * sizeof(T))) == 0 && g.ldo % 2 == 0 &&
                          (!res || ((reinterpret_cast<uintptr_t>(res) % (2 * sizeof(T))) == 0 && g.ldr % 2 == 0));
        const int ca = twos ? 2 * lane : lane, cb = twos ? 2 * lane + 1 : lane + 32;
        struct alignas(2 * sizeof(T)) Two { T x, y; };
        for (int i = 0; i < my_tiles; ++i) {
            const int acc = i & 1;
            int m0, n0;
            origin(i, m0, n0);
            const int64_t row0 = (int64_t)m0 + (int)rank * 128 + quarter * 32;     // this warp's 32 rows
            const int rows = (int)min((int64_t)32, g.m - row0);                    // 0 or less: none of them exists
            RowTerm mine = {0.0f, 0u};                                             // lane's row; handed round by shuffles
            if (lane < rows) mine = row_term(g, row0 + lane);
            ok = ok && mbar_wait_warp(acc_full(acc), (i >> 1) & 1, &failed, g.polls) && !__any_sync(0xffffffffu, has_failed());
            const int64_t cx = (int64_t)n0 + c0 + ca, cy = (int64_t)n0 + c0 + cb;
            const bool in_x = cx < g.n, in_y = cy < g.n;
            ColTerm ct[2] = {{0.0f, 0u, 0.0f}, {0.0f, 0u, 0.0f}};
            if (in_x) ct[0] = col_term(g, cx);
            if (in_y) ct[1] = col_term(g, cy);
            const bool fast = twos && n0 + c0 + 64 <= g.n;
            if (ok) {
                tmem_fence_after();
                uint32_t v[32];
                tmem_load32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * BN + c0 + part * 32), v);
                tmem_wait_ld();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_cta(acc_empty(acc), 0));       // this warp's part of the accumulator is read
#pragma unroll
                for (int j = 0; j < 32; j += 2)
                    *reinterpret_cast<uint2*>(sh + lane * Shape::row_words + 2 * ((part * 16 + j / 2) ^ lane)) = make_uint2(v[j], v[j + 1]);
            }
            // (the other warp of the block may have given up: half of the columns are missing then)
            if (!block_all(ok)) ct[0].scale = ct[1].scale = kNaN;
            {
                // kRowsAtOnce rows at a time.  All residuals of a group are requested before any is used or any result is
                // written: they may lie in the result's own tensor, so the compiler could not move a load up by itself, and
                // one load after the other took 45 us of a tile's 51.  (All 32 rows at once spill: 61 -> 78 us at 4096^3.)
                constexpr int kRowsAtOnce = 8;
#pragma unroll 1
                for (int r0 = part * 16; r0 < min(rows, part * 16 + 16); r0 += kRowsAtOnce) {
                    const bool all_rows = r0 + kRowsAtOnce <= rows;
                    T* o = out + (row0 + r0) * g.ldo;
                    const T* q = res + (row0 + r0) * g.ldr;
                    Two w[kRowsAtOnce];
                    if (res && fast && all_rows) {
#pragma unroll
                        for (int j = 0; j < kRowsAtOnce; ++j) w[j] = *reinterpret_cast<const Two*>(q + j * g.ldr + cx);
                    } else if (res) {
#pragma unroll
                        for (int j = 0; j < kRowsAtOnce; ++j) {
                            const int64_t at = min(j, rows - 1 - r0) * g.ldr;      // a row that exists: no branch between the loads
                            w[j].x = q[at + min(cx, g.n - 1)];
                            w[j].y = q[at + min(cy, g.n - 1)];
                        }
                    }
                    float f[2 * kRowsAtOnce];
#pragma unroll
                    for (int j = 0; j < kRowsAtOnce; ++j) {
                        const int r = r0 + j;
                        uint2 v;
                        if (twos) {
                            v = *reinterpret_cast<const uint2*>(sh + r * Shape::row_words + 2 * (lane ^ r));
                        } else {
                            v.x = sh[r * Shape::row_words + 2 * ((ca >> 1) ^ r) + (ca & 1)];
                            v.y = sh[r * Shape::row_words + 2 * ((cb >> 1) ^ r) + (cb & 1)];
                        }
                        const RowTerm rt = {__shfl_sync(0xffffffffu, mine.scale, r), __shfl_sync(0xffffffffu, mine.term, r)};
                        f[2 * j] = linear_value(g, v.x, rt, ct[0]);
                        f[2 * j + 1] = linear_value(g, v.y, rt, ct[1]);
                    }
                    glue_values(f, g.glue);
                    if (res) {
#pragma unroll
                        for (int j = 0; j < kRowsAtOnce; ++j) { f[2 * j] += to_f32(w[j].x); f[2 * j + 1] += to_f32(w[j].y); }
                    }
                    if (fast && all_rows) {
#pragma unroll
                        for (int j = 0; j < kRowsAtOnce; ++j) *reinterpret_cast<Two*>(o + j * g.ldo + cx) = Two{from_f32<T>(f[2 * j]), from_f32<T>(f[2 * j + 1])};
                    } else {
#pragma unroll
                        for (int j = 0; j < kRowsAtOnce; ++j) {
                            if (r0 + j < rows && in_x) o[j * g.ldo + cx] = from_f32<T>(f[2 * j]);
                            if (r0 + j < rows && in_y) o[j * g.ldo + cy] = from_f32<T>(f[2 * j + 1]);
                        }
                    }
                }
            }
            block_sync();
        }
    }
    __syncwarp();
    if (has_failed() && lane == 0) st_cluster(map_to_cta(smem_addr(&peer_failed), rank ^ 1u), 1u);
    tmem_fence_before();
    cluster_sync_all();
    tmem_fence_after();
    if (has_failed() || *(volatile int*)&peer_failed) {
        // The same in both CTAs, none of which issues anything any more: the products under way end, and the copies that
        // nobody waited for have 10 ms to land before either CTA gives its memory back.
        if (warp == 1) {
            if (rank == 0 && elect_one()) umma_commit<2>(drained);
            __syncwarp();
            mbar_wait(drained, 0);
            for (int q = 0; q < 100; ++q) __nanosleep(100000);
        }
        __syncwarp();
        cluster_sync_all();
        tmem_fence_after();
    }
    if (warp == 0) tmem_free<2>(tmem, kAccs * BN);
    if (threadIdx.x == 0 && failed) atomicAdd(&g_wait_failures, 1u);
}

// Splits of k: as many as still fit the device at once, with two blocks each and two rows of the tile each at least.
inline int small_splits(int64_t tiles, int64_t blocks, int bn, int64_t sms) {
    int splits = 1;
    while (splits < 8 && splits * 4 <= bn && tiles * splits * 2 <= sms && blocks >= splits * 4) splits *= 2;
    return splits;
}

template <typename T, int BN>
int launch_linear_small(const LinearArgs& g, cudaStream_t st) {
    using Shape = SmallShape<BN>;
    static PerDeviceOnce once;
    auto* kernel = linear_small_kernel<T, BN>;
    int rc = once.raise_smem_limit(kernel, Shape::smem);
    if (rc != MPQ_OK) return rc;
    CUtensorMap map_w, map_a;
    if (!byte_tensor_map(&map_w, g.w, g.n, g.row_bytes, 128) || !byte_tensor_map(&map_a, g.a, g.m, g.row_bytes, BN)) return MPQ_ERR_CUDA;
    const int sms = sm_count();
    if (sms == 0) return MPQ_ERR_CUDA;
    const int64_t tiles_w = ceil_div(g.n, 128), tiles = tiles_w * ceil_div(g.m, BN), blocks = ceil_div(g.row_bytes, kBlock);
    if (tiles > (1 << 28)) return MPQ_ERR_BAD_SHAPE;
    const int splits = small_splits(tiles, blocks, BN, sms);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * splits), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = Shape::smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // barriers and TMEM are set up before the wait
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kernel, map_w, map_a, g, (int)tiles_w, splits) != cudaSuccess) { cudaGetLastError(); return MPQ_ERR_CUDA; }
    return launch_status();
}

template <typename T>
int launch_linear_pair(const LinearArgs& g, cudaStream_t st) {
    using Shape = PairShape;
    constexpr int BN = kPairCols;
    static PerDeviceOnce once;
    auto* kernel = linear_pair_kernel<T>;
    int rc = once.raise_smem_limit(kernel, Shape::smem);
    if (rc != MPQ_OK) return rc;
    CUtensorMap map_w, map_a;
    if (!byte_tensor_map(&map_w, g.w, g.n, g.row_bytes, BN / 2) || !byte_tensor_map(&map_a, g.a, g.m, g.row_bytes, 128)) return MPQ_ERR_CUDA;
    const int pairs = sm_count() / 2;
    if (pairs == 0) return MPQ_ERR_CUDA;
    const int64_t tiles_m = ceil_div(g.m, 256), tiles = tiles_m * ceil_div(g.n, BN);
    if (tiles > (1 << 28)) return MPQ_ERR_BAD_SHAPE;
    const unsigned ctas = 2u * (unsigned)(tiles < pairs ? tiles : pairs);
    return launch_chained_as(true, kernel, ctas, (unsigned)kPairThreads, Shape::smem, st, map_a, map_w, g, (int)tiles_m, (int)tiles);
}

// Which form.  Up to 64 rows the weights' own traffic decides: the small form, its tile just wide enough.  Above, the
// small form too while its 128 x 64 tiles fit the device at once (it may split k then), else CTA pairs: us for
// m x n x k, small / pairs --
//   64 tiles: 128 x 4096 x 4096 11.8 / 15.2;  128: 200 x 4096 x 4096 12.5 / 15.2;  142: 100 x 9000 x 1000 9.4 / 11.9;
//   144: 128 x 9216 x 4096 14.3 / 17.1, 2300 x 512 x 9216 19.5 / 22.4;  150: 128 x 9600 x 4096 23.7 / 22.4;
//   213: 130 x 9000 x 1000 16.6 / 12.6;  256: 1000 x 2000 x 2000 19.8 / 13.1.
template <typename T>
int launch_linear_levels(const LinearArgs& g, cudaStream_t st) {
    if (g.m <= 16) return launch_linear_small<T, 16>(g, st);
    if (g.m <= 32) return launch_linear_small<T, 32>(g, st);
    if (g.m <= 64 || ceil_div(g.m, 64) * ceil_div(g.n, 128) <= sm_count()) return launch_linear_small<T, 64>(g, st);
    return launch_linear_pair<T>(g, st);
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
    const LinearArgs g = {a, a_scale, a_sums, w, w_scale, w_sums, m, n, k, level_row_bytes(k), (int)La, (int)Lw, bias, glue, residual, ldr, out, ldo,
                          wait_limit()};
    if (dtype == MPQ_F32) return launch_linear_levels<float>(g, (cudaStream_t)stream);
    if (dtype == MPQ_F16) return launch_linear_levels<__half>(g, (cudaStream_t)stream);
    return launch_linear_levels<__nv_bfloat16>(g, (cudaStream_t)stream);
}

namespace {
std::atomic<uint32_t> g_wait_limit{kSpinLimit};
}
uint32_t mpq::wait_limit() { return g_wait_limit.load(std::memory_order_relaxed); }

extern "C" void mpq_wait_limit(int polls) { g_wait_limit.store(polls < 0 ? kSpinLimit : (uint32_t)polls, std::memory_order_relaxed); }

extern "C" int mpq_wait_failures(unsigned int* count_host, void* stream) {
    if (!count_host) return MPQ_ERR_NULL;
    unsigned int attention = 0;
    cudaStream_t st = (cudaStream_t)stream;
    if (attention_wait_failures(&attention, st) != MPQ_OK ||
        cudaMemcpyFromSymbolAsync(count_host, g_wait_failures, sizeof(unsigned int), 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess) { cudaGetLastError(); return MPQ_ERR_CUDA; }
    *count_host += attention;
    return MPQ_OK;
}
