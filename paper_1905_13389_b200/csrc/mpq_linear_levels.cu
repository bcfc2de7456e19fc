// Product of level bytes with bias, activation and residual in its epilogue (mpq_linear_levels).
//
// With q = 2u - L (Eq. 16) the layer's integer product is
//   sum q_a q_w = 4 sum u_a u_w - 2 L_w sum u_a - 2 L_a sum u_w + k L_a L_w,
// so the inner loop multiplies unsigned bytes and the level sums that lie beside the operands do the rest.
// The result fits int32 (checked on the host), hence the terms may be combined modulo 2^32.
#include "mpq_adapters.cuh"
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
    const void* up = nullptr; int rank = 0;               // adapters: [..][n][rank]
    int adapters = 0, sequences = 0;
    LowWorkspace low = {};                                // what the adapters have made of the tokens
};

// acc (levels u, unsigned) -> one output, in the header's order of operations
struct RowTerm { float scale; uint32_t term; };          // a_scale / L_a;  k L_a L_w - 2 L_w sums_a
struct ColTerm { float scale; uint32_t term; float bias; };   // w_scale / L_w;  2 L_a sums_w;  bias
__device__ __forceinline__ RowTerm row_term(const LinearArgs& g, int64_t r) {
    RowTerm t;
    t.scale = __fdiv_rn(g.a_scale[r], (float)g.La);
    t.term = (uint32_t)g.k * (uint32_t)g.La * (uint32_t)g.Lw - 2u * (uint32_t)g.Lw * (uint32_t)g.a_sums[r];
    return t;
}
__device__ __forceinline__ ColTerm col_term(const LinearArgs& g, int64_t c) {
    ColTerm t;
    t.scale = __fdiv_rn(g.w_scale[c], (float)g.Lw);
    t.term = 2u * (uint32_t)g.La * (uint32_t)g.w_sums[c];
    t.bias = g.bias ? g.bias[c] : 0.0f;
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
    static constexpr int low_bytes = BN * 128 * 4;        // [BN rows][128 columns] fp32: what the adapters add
};

// What the adapters of rows row0 + first .. + count (64 at most) add to a warp's 32 columns c0 .., to low[row][..]: each row's z times
// the columns' rows of `up`, in fp32.  The 32 rows of `up` are 64 RANK adjacent bytes, read as whole lines: a lane owns
// the same eight ranks of RANK / 8 columns, and the sums of the lanes that share a column are exchanged so that each lane
// is left with one column.  It is the latency of these reads that bounds it: eight to sixteen are on their way while as many are summed.
template <typename W, int RANK>
__device__ __forceinline__ void low_rank_rows_of(const LinearArgs& g, int64_t row0, int first, int count, int64_t c0, float* low, int lane) {
    constexpr int kReads = RANK / 8, kRows = RANK <= 32 ? 4 : 128 / RANK;  // reads of a row, rows at once
    constexpr int kStep = 32 / kReads;                     // columns of a read
    const int sub = lane % kReads;
    auto adapter = [&](int r) {
        const int id = r < count && row0 + first + r < g.m ? g.low.chosen[row0 + first + r] : -1;
        return id < g.adapters ? id : -1;
    };
    const int ids[2] = {adapter(lane), adapter(lane + 32)};
    auto id_of = [&](int r) { return __shfl_sync(0xffffffffu, r < 32 ? ids[0] : ids[1], r & 31); };
    const bool any = __any_sync(0xffffffffu, ids[0] >= 0 || ids[1] >= 0);
    uint4 next[kRows][kReads];
    float4 next_z[kRows][2];
    auto ask = [&](int r0) {
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const int r = min(r0 + j, count - 1);
            const int64_t id = max(id_of(r), 0);
#pragma unroll
            for (int q = 0; q < kReads; ++q) {
                const int64_t c = min(c0 + q * kStep + lane / kReads, g.n - 1);
                next[j][q] = __ldg(reinterpret_cast<const uint4*>(static_cast<const W*>(g.up) + (id * g.n + c) * RANK + sub * 8));
            }
            const float4* z = reinterpret_cast<const float4*>(g.low.z + min(row0 + first + r, g.m - 1) * RANK + sub * 8);
            next_z[j][0] = z[0];
            next_z[j][1] = z[1];
        }
    };
    if (any) ask(0);
#pragma unroll 1
    for (int r0 = 0; r0 < count; r0 += kRows) {
        uint4 u[kRows][kReads];
        float4 z[kRows][2];
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
#pragma unroll
            for (int q = 0; q < kReads; ++q) u[j][q] = next[j][q];
            z[j][0] = next_z[j][0];
            z[j][1] = next_z[j][1];
        }
        if (any && r0 + kRows < count) ask(r0 + kRows);
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            if (r0 + j >= count) break;
            float sum[kReads] = {};
            if (id_of(r0 + j) >= 0) {                      // (the same for all lanes)
                const float v[8] = {z[j][0].x, z[j][0].y, z[j][0].z, z[j][0].w, z[j][1].x, z[j][1].y, z[j][1].z, z[j][1].w};
#pragma unroll
                for (int q = 0; q < kReads; ++q) {
                    const W* e = reinterpret_cast<const W*>(&u[j][q]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[q] = fmaf(to_f32(e[i]), v[i], sum[q]);
                }
#pragma unroll
                for (int o = kReads / 2; o > 0; o >>= 1)   // a lane keeps the half of the reads that its bit `o` names
#pragma unroll
                    for (int q = 0; q < o; ++q) {
                        const bool upper = (sub & o) != 0;
                        const float give = upper ? sum[q] : sum[q + o], keep = upper ? sum[q + o] : sum[q];
                        sum[q] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                    }
            }
            low[(first + r0 + j) * 128 + sub * kStep + lane / kReads] = sum[0];        // read number `sub` is this lane's
        }
    }
    __syncwarp();
}
template <typename W>
__device__ __forceinline__ void low_rank_rows(const LinearArgs& g, int64_t row0, int first, int count, int64_t c0, float* low, int lane) {
    if (g.rank == 16) low_rank_rows_of<W, 16>(g, row0, first, count, c0, low, lane);
    else if (g.rank == 32) low_rank_rows_of<W, 32>(g, row0, first, count, c0, low, lane);
    else if (g.rank == 64) low_rank_rows_of<W, 64>(g, row0, first, count, c0, low, lane);
    else low_rank_rows_of<W, 128>(g, row0, first, count, c0, low, lane);
}

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

template <typename T, typename W, int BN>
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
    [[maybe_unused]] float* low = reinterpret_cast<float*>(exchange_ptr) + Shape::exchange_bytes / 4;        // [BN][128]: what the adapters add
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
    // With adapters the kernel before has made z, and was let in only when those before it had ended: the operands are there, and
    // only the storing warps wait.
    if constexpr (std::is_void_v<W>) {
        chain_entry();
    } else {
        chain_next();
        if (warp >= 2) chain_wait();
    }

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
        const int own = BN / splits;
        if constexpr (!std::is_void_v<W>) low_rank_rows<W>(g, m0, split * own, own, (int64_t)n0 + quarter * 32, low + quarter * 32, lane);
        bool ok = mbar_wait_warp(done, 0, &failed, g.polls);
        if (!ok) mbar_wait(done, 0);                      // what has been issued must end before TMEM is freed
        ok = ok && !__any_sync(0xffffffffu, has_failed());
        if (!ok) {                                        // results are NaN from here on, in all CTAs of the tile
            ct.scale = kNaN;
            if (splits > 1 && lane < splits) st_cluster(map_to_cta(smem_addr(&peer_failed), (uint32_t)lane), 1u);
        }
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
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
                    if constexpr (!std::is_void_v<W>) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) f[j] += low[(r0 + j) * 128 + col];
                    }
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
                    if constexpr (!std::is_void_v<W>) {
#pragma unroll
                        for (int j = 0; j < N; ++j) f[j] += low[(rr + j) * 128 + col];
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
template <bool ADAPTED>
struct PairShape {
    static constexpr int stage_bytes = (128 + kPairCols / 2) * kBlock;   // per CTA
    static constexpr int stages = ADAPTED ? 5 : 6;        // with adapters L1 keeps what their reads share
    static constexpr int row_words = 64;                            // column pair p of row r lies at pair p ^ r: no bank conflicts either way
    static constexpr int transpose_bytes = kPairStoreWarps / 2 * 32 * row_words * 4;
    static constexpr int term_bytes = ADAPTED ? kPairStoreWarps / 2 * 64 * 16 : 0;      // the columns' constants
    static constexpr int smem = stages * stage_bytes + transpose_bytes + term_bytes + 1024;
};

__device__ __forceinline__ void umma_f16_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// What adapters add in the pair form.  Where one adapter has all 256 rows of a tile, the parts of z times its rows of `up` are more
// blocks of the tile's product, on the 5th-generation tensor cores, into accumulators of their own (kind::f16; 64 ranks
// of a part are a block, ranks that are not there are read as zeros).  Other tiles, with ends of sequences in them, have it
// from low_rank_tile: 16 rows and 64 columns by 16 x 8 x 16 matrix instructions of the storing warps, a lane owning four adjacent
// ranks of 16 in both operands alike, one adapter after the other of those that the rows have: a row takes its own one's
// sums alone, so that nothing of another's reaches it.  4096^3 with rank 64: 88 us where one sequence has all rows (28 of
// them the first kernel's), 110 with six; all tiles the second way 120 to 127, bound by L1 lookups.  PARTS: of z; 32-bit
// results have all of it, 16-bit ones two parts, which lose 2^-16 of it in bfloat16 and 2^-22 in float16, little beside
// their own last rounding unless the product and its adapter cancel (a third part: six sequences 110 -> 117 us, 4096 x 4096 x 512 with rank 128 103 -> 114).
template <typename W, int PARTS>
__device__ __forceinline__ void low_rank_tile(const LinearArgs& g, int64_t row0, int64_t c0, uint32_t at, int lane, int turn) {
    const int row = lane >> 2, quad = lane & 3;
    int id = lane < 16 && row0 + lane < g.m ? g.low.chosen[row0 + lane] : -1;
    if (id >= g.adapters) id = -1;
    uint32_t left = __ballot_sync(0xffffffffu, id >= 0);
    const int64_t z0 = min(row0 + row, g.m - 1), z1 = min(row0 + row + 8, g.m - 1);
    bool begun = false;
    do {
        float acc[32] = {};                                // as the instruction leaves them and TMEM takes them: 4 j + 2 h + e is row + 8 h, column 8 j + 2 quad + e
        uint32_t rows = 0xffffu;
        if (left) {
            const int which = __shfl_sync(0xffffffffu, id, __ffs(left) - 1);
            rows = __ballot_sync(0xffffffffu, id == which);
            left &= ~rows;
            const W* up = static_cast<const W*>(g.up) + (int64_t)which * g.n * g.rank + 4 * quad;
            const W* z = reinterpret_cast<const W*>(g.low.parts) + 4 * quad;
            int i = turn * 16 % g.rank;                    // warps begin with different ranks: each is fetched once and is in L1 for the others
#pragma unroll 1
            for (int n = 0; n < g.rank; n += 16, i = i + 16 < g.rank ? i + 16 : 0) {
                uint2 u[8], a[PARTS][2];
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = __ldg(reinterpret_cast<const uint2*>(up + min(c0 + 8 * j + row, g.n - 1) * g.rank + i));
#pragma unroll
                for (int q = 0; q < PARTS; ++q) {
                    a[q][0] = *reinterpret_cast<const uint2*>(z + (q * g.m + z0) * g.rank + i);
                    a[q][1] = *reinterpret_cast<const uint2*>(z + (q * g.m + z1) * g.rank + i);
                }
#pragma unroll
                for (int q = PARTS - 1; q >= 0; --q)
#pragma unroll
                    for (int j = 0; j < 8; ++j) mma_16x8x16<W>(acc + 4 * j, a[q][0].x, a[q][1].x, a[q][0].y, a[q][1].y, u[j].x, u[j].y);
            }
            const float s0 = g.low.scale[z0], s1 = g.low.scale[z1];
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[i] *= (i >> 1) & 1 ? s1 : s0;
        }
        uint32_t sums[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) sums[i] = __float_as_uint(acc[i]);
        if (rows != 0xffffu) {
            uint32_t before[32] = {};
            if (begun) {
                tmem_load_frag(at, before);
                tmem_wait_ld();
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) sums[i] = rows >> (row + 8 * ((i >> 1) & 1)) & 1 ? sums[i] : before[i];
        }
        tmem_store_frag(at, sums);
        tmem_wait_st();
        begun = true;
    } while (left);
}

// The adapter that all of a tile's rows have (those behind the last row have any), or -1; by a warp, after chain_wait().
__device__ __forceinline__ int tile_adapter(const LinearArgs& g, int64_t m0, int lane) {
    const int64_t last = g.m - 1;
    const int first = g.low.chosen[m0];
    bool same = first >= 0 && first < g.adapters;
#pragma unroll
    for (int i = 0; i < 8; ++i) same &= g.low.chosen[min(m0 + i * 32 + lane, last)] == first;
    return __all_sync(0xffffffffu, same) ? first : -1;
}
constexpr int kBlockRanks = 64;                            // of a block, which is 128 bytes wide

// The largest size of three, NaN if one is.
__device__ __forceinline__ float max_size(float a, float b, float c) {
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}

// What an adapter adds to one result, term by term in fp32.  An infinity in `up` meets every part of z in the matrix instructions, and
// parts may be zero or of the other sign (NaN, where z itself makes an infinity); sums that are not finite are made again from z.
template <typename W>
__device__ __noinline__ float low_rank_one(const W* up, const float* z, int rank) {
    float s = 0.0f;
    for (int i = 0; i < rank; ++i) s = fmaf(to_f32(up[i]), z[i], s);
    return s;
}

template <typename T, typename W>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w,
                   const __grid_constant__ CUtensorMap map_z, const __grid_constant__ CUtensorMap map_up, const LinearArgs g, int tiles_m, int tiles) {
    constexpr int kZParts = std::is_same_v<W, __nv_bfloat16> && std::is_same_v<T, float> ? kLowParts : 2;
    using Shape = PairShape<!std::is_void_v<W>>;
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
    constexpr uint32_t kTmemCols = kAccs * BN * (std::is_void_v<W> ? 1 : 2);       // what the adapters add lies behind the accumulators, as many
    if (warp == 0) tmem_alloc<2>(&tmem_holder, kTmemCols);
    tmem_fence_before();
    cluster_sync_all();                                    // both CTAs' barriers exist
    tmem_fence_after();
    const uint32_t tmem = tmem_holder;
    if constexpr (std::is_void_v<W>) {
        chain_entry();
    } else {                                               // (see linear_small_kernel)
        chain_next();
        if (warp >= 2) chain_wait();
    }
    [[maybe_unused]] bool waited = false;                  // of the other warps: once they need what the kernel before has made
    [[maybe_unused]] const int low_blocks = std::is_void_v<W> ? 0 : kZParts * ((g.rank + kBlockRanks - 1) / kBlockRanks);

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
            if constexpr (!std::is_void_v<W>) {
                if (!waited) chain_wait();
                waited = true;
                const int id = tile_adapter(g, m0, lane);
                for (int e = 0; ok && id >= 0 && e < low_blocks; ++e, ++issued) {
                    const int s = issued % kStages, part = e % kZParts, r0 = e / kZParts * kBlockRanks;
                    if (issued >= kStages && !mbar_wait_warp(empty(s), (issued / kStages - 1) & 1, &failed, g.polls)) { ok = false; break; }
                    if (leader) {
                        const uint32_t dst = ring + s * Shape::stage_bytes, bar = map_to_cta(full(s), 0);
                        if (rank == 0) mbar_expect_tx(full(s), 2 * Shape::stage_bytes);
                        tma_load_2d_pair(dst, &map_z, r0, (int)(part * g.m) + m0 + (int)rank * 128, bar);
                        tma_load_2d_pair(dst + 128 * kBlock, &map_up, r0, (int)(id * g.n) + n0 + (int)rank * (BN / 2), bar);
                    }
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
                if constexpr (!std::is_void_v<W>) {
                    if (!waited) chain_wait();
                    waited = true;
                    int m0, n0;
                    origin(i, m0, n0);
                    const int id = tile_adapter(g, m0, lane);
                    constexpr uint32_t idesc_low = umma_idesc_f16(256, BN) | (std::is_same_v<W, __nv_bfloat16> ? 1u << 7 | 1u << 10 : 0u);
                    for (int e = 0; ok && id >= 0 && e < low_blocks; ++e, ++consumed) {
                        const int s = consumed % kStages, r0 = e / kZParts * kBlockRanks;
                        if (!mbar_wait_warp(full(s), (consumed / kStages) & 1, &failed, g.polls)) { ok = false; break; }
                        tmem_fence_after();
                        const uint32_t at = ring + s * Shape::stage_bytes;
                        if (leader) {
                            const uint64_t da = umma_desc(at), db = umma_desc(at + 128 * kBlock);
                            for (int j = 0; j < kBlockRanks / 16 && r0 + 16 * j < g.rank; ++j)
                                umma_f16_pair(d + kAccs * BN, da + 2 * j, db + 2 * j, idesc_low, e > 0 || j > 0);
                            umma_commit<2>(empty(s));
                        }
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
            const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
            [[maybe_unused]] bool whole_tile = false;
            [[maybe_unused]] float4* terms = reinterpret_cast<float4*>(transpose + kPairStoreWarps / 2 * 32 * Shape::row_words) + block * 64;
            if constexpr (!std::is_void_v<W>) {
                // Sums of what the adapters add lie by rows, so the columns' constants are needed by rows too: this warp's 32
                // columns of them.  Where the storing warps make those sums they do it while the tile is multiplied.
                const int64_t c = (int64_t)n0 + c0 + part * 32 + lane;
                const ColTerm t = c < g.n ? col_term(g, c) : ColTerm{0.0f, 0u, 0.0f};
                terms[part * 32 + lane] = make_float4(t.scale, __uint_as_float(t.term), t.bias, 0.0f);
                whole_tile = tile_adapter(g, m0, lane) >= 0;
                if (!whole_tile) {
                    tmem_fence_after();                    // (the block has read what an earlier tile had there)
                    low_rank_tile<W, kZParts>(g, row0 + part * 16, (int64_t)n0 + c0, lanes + ((uint32_t)(part * 16) << 16) + (uint32_t)((kAccs + acc) * BN + c0), lane, quarter * 2 + part);
                    tmem_fence_before();
                }
                block_sync();
                tmem_fence_after();
            }
            ok = ok && mbar_wait_warp(acc_full(acc), (i >> 1) & 1, &failed, g.polls) && !__any_sync(0xffffffffu, has_failed());
            const int64_t cx = (int64_t)n0 + c0 + ca, cy = (int64_t)n0 + c0 + cb;
            const bool in_x = cx < g.n, in_y = cy < g.n;
            ColTerm ct[2] = {{0.0f, 0u, 0.0f}, {0.0f, 0u, 0.0f}};
            if (std::is_void_v<W> && in_x) ct[0] = col_term(g, cx);
            if (std::is_void_v<W> && in_y) ct[1] = col_term(g, cy);
            const bool fast = twos && n0 + c0 + 64 <= g.n;
            if (ok) {
                tmem_fence_after();
                uint32_t v[32];
                tmem_load32(lanes + (uint32_t)(acc * BN + c0 + part * 32), v);
                [[maybe_unused]] uint32_t low[32];
                if constexpr (!std::is_void_v<W>) tmem_load32(lanes + (uint32_t)((kAccs + acc) * BN + c0 + part * 32), low);
                tmem_wait_ld();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_cta(acc_empty(acc), 0));       // this warp's part of the accumulator is read
                if constexpr (!std::is_void_v<W>) {
                    const float scale = whole_tile ? g.low.scale[min(row0 + lane, g.m - 1)] : 1.0f;
                    float most = 0.0f;                     // (32 multiply-adds instead: 120 us for 114)
#pragma unroll
                    for (int j = 0; j < 32; j += 2) most = max_size(most, __uint_as_float(low[j]), __uint_as_float(low[j + 1]));
                    if (__any_sync(0xffffffffu, lane < rows && !ordinary(most))) {
                        uint32_t* own = sh + lane * Shape::row_words;      // (this lane's and warp's part, in columns of pairs; see below)
                        auto at = [&](int j) { return 2 * ((part * 16 + j / 2) ^ lane) + j % 2; };
#pragma unroll
                        for (int j = 0; j < 32; ++j) own[at(j)] = __float_as_uint(scale * __uint_as_float(low[j]));
                        const int id = lane < rows ? g.low.chosen[row0 + lane] : -1;
#pragma unroll 1
                        for (int j = 0; j < 32; ++j) {
                            const int64_t c = (int64_t)n0 + c0 + part * 32 + j;
                            if (id >= 0 && id < g.adapters && c < g.n && !ordinary(__uint_as_float(own[at(j)])))
                                own[at(j)] = __float_as_uint(low_rank_one(static_cast<const W*>(g.up) + (id * g.n + c) * g.rank, g.low.z + (row0 + lane) * g.rank, g.rank));
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float4 t = terms[part * 32 + j];
                            v[j] = __float_as_uint(linear_value(g, v[j], mine, ColTerm{t.x, __float_as_uint(t.y), t.z}) + __uint_as_float(own[at(j)]));
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float4 t = terms[part * 32 + j];
                            v[j] = __float_as_uint(linear_value(g, v[j], mine, ColTerm{t.x, __float_as_uint(t.y), t.z}) + scale * __uint_as_float(low[j]));
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 32; j += 2)
                    *reinterpret_cast<uint2*>(sh + lane * Shape::row_words + 2 * ((part * 16 + j / 2) ^ lane)) = make_uint2(v[j], v[j + 1]);
            }
            // (the other warp of the block may have given up: half of the columns are missing then)
            const bool all_ok = block_all(ok);
            if (!all_ok) ct[0].scale = ct[1].scale = kNaN;
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
                        if constexpr (std::is_void_v<W>) {
                            const RowTerm rt = {__shfl_sync(0xffffffffu, mine.scale, r), __shfl_sync(0xffffffffu, mine.term, r)};
                            f[2 * j] = linear_value(g, v.x, rt, ct[0]);
                            f[2 * j + 1] = linear_value(g, v.y, rt, ct[1]);
                        } else {
                            f[2 * j] = all_ok ? __uint_as_float(v.x) : kNaN;
                            f[2 * j + 1] = all_ok ? __uint_as_float(v.y) : kNaN;
                        }
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
    if (warp == 0) tmem_free<2>(tmem, kTmemCols);
    if (threadIdx.x == 0 && failed) atomicAdd(&g_wait_failures, 1u);
}

// Splits of k: as many as still fit the device at once, with two blocks each and two rows of the tile each at least.
inline int small_splits(int64_t tiles, int64_t blocks, int bn, int64_t sms) {
    int splits = 1;
    while (splits < 8 && splits * 4 <= bn && tiles * splits * 2 <= sms && blocks >= splits * 4) splits *= 2;
    return splits;
}

template <typename T, typename W, int BN>
int launch_linear_small(const LinearArgs& g, cudaStream_t st) {
    using Shape = SmallShape<BN>;
    static PerDeviceOnce once;
    auto* kernel = linear_small_kernel<T, W, BN>;
    constexpr int smem = Shape::smem + (std::is_void_v<W> ? 0 : Shape::low_bytes);
    int rc = once.raise_smem_limit(kernel, smem);
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
    cfg.dynamicSmemBytes = smem;
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

// [rows][ranks] pairs of bytes; boxes of box_rows rows x 64 ranks, 128-byte swizzle; what lies outside reads as 0.
inline bool pair_tensor_map(CUtensorMap* map, const void* base, int64_t rows, int64_t ranks, int box_rows) {
    const TensorMapEncodeFn encode = tensor_map_encoder();
    const cuuint64_t dims[2] = {(cuuint64_t)ranks, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ranks * 2};
    const cuuint32_t box[2] = {(cuuint32_t)kBlockRanks, (cuuint32_t)box_rows};
    const cuuint32_t elem[2] = {1, 1};
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(base), dims, strides, box, elem,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, typename W>
int launch_linear_pair(const LinearArgs& g, cudaStream_t st) {
    using Shape = PairShape<!std::is_void_v<W>>;
    constexpr int BN = kPairCols;
    static PerDeviceOnce once;
    auto* kernel = linear_pair_kernel<T, W>;
    constexpr int smem = Shape::smem;
    int rc = once.raise_smem_limit(kernel, smem);
    if (rc != MPQ_OK) return rc;
    CUtensorMap map_w, map_a;
    if (!byte_tensor_map(&map_w, g.w, g.n, g.row_bytes, BN / 2) || !byte_tensor_map(&map_a, g.a, g.m, g.row_bytes, 128)) return MPQ_ERR_CUDA;
    CUtensorMap map_z = map_a, map_up = map_w;
    if constexpr (!std::is_void_v<W>) {
        if (!pair_tensor_map(&map_z, g.low.parts, (int64_t)kLowParts * g.m, g.rank, 128) ||
            !pair_tensor_map(&map_up, g.up, (int64_t)g.adapters * g.n, g.rank, BN / 2)) return MPQ_ERR_CUDA;
    }
    const int pairs = sm_count() / 2;
    if (pairs == 0) return MPQ_ERR_CUDA;
    const int64_t tiles_m = ceil_div(g.m, 256), tiles = tiles_m * ceil_div(g.n, BN);
    if (tiles > (1 << 28)) return MPQ_ERR_BAD_SHAPE;
    const unsigned ctas = 2u * (unsigned)(tiles < pairs ? tiles : pairs);
    return launch_chained_as(true, kernel, ctas, (unsigned)kPairThreads, smem, st, map_a, map_w, map_z, map_up, g, (int)tiles_m, (int)tiles);
}

// Which form.  Up to 64 rows the weights' own traffic decides: the small form, its tile just wide enough.  Above, the
// small form too while its 128 x 64 tiles fit the device at once (it may split k then), else CTA pairs: us for
// m x n x k, small / pairs --
//   64 tiles: 128 x 4096 x 4096 11.8 / 15.2;  128: 200 x 4096 x 4096 12.5 / 15.2;  142: 100 x 9000 x 1000 9.4 / 11.9;
//   144: 128 x 9216 x 4096 14.3 / 17.1, 2300 x 512 x 9216 19.5 / 22.4;  150: 128 x 9600 x 4096 23.7 / 22.4;
//   213: 130 x 9000 x 1000 16.6 / 12.6;  256: 1000 x 2000 x 2000 19.8 / 13.1.
// With adapters the small form's sums take longer the more rows and ranks there are, the pairs' the more sequences a tile
// has: pairs from sequences of 12 tokens on average.  us for m x n x k, rank, sequences, small / pairs --
//   33 x 4096 x 4096, 16, 1 16.4 / 14.1, 64, 1 25.8 / 18.0;  60 x 4096 x 4096, 64, 1 25.9 / 18.5, 5 26.7 / 30.1, 25 21.7 / 41.7;
//   140 x 4096 x 4096, 64, 9 41.2 / 33.7, 17 40.4 / 36.8, 35 36.2 / 46.6;  256 x 4096 x 1024, 16, 16 21.2 / 17.9, 64 21.6 / 21.8;
//   512 x 2048 x 2048, 64, 1 43.6 / 23.5, 25 40.6 / 32.2, 50 39.9 / 40.0, 200 39.2 / 48.7;  20 x 4096 x 4096, 64, 1 21.1 / 21.3.
// A long k is another matter, since the small form splits it: the more rows and ranks, the longer it may be.  One sequence --
//   64 x 128 x 30000, 16 19.3 / 57.7, 64 33.8 / 58.2;  64 x 1024 x 9216, 16 16.6 / 18.4, 64 24.8 / 20.9;  64 x 4096 x 16384, 16 21.8 / 28.4,
//   64 34.7 / 30.6;  100 x 2048 x 9216, 16 18.8 / 18.5, 64 33.6 / 21.4;  200 x 512 x 9216, 16 24.4 / 18.5;  256 x 4096 x 9216, 16 27.5 / 19.3.
template <typename T, typename W = void>
int launch_linear_levels(const LinearArgs& g, cudaStream_t st) {
    if constexpr (!std::is_void_v<W>)
        if (g.m > 32 && g.m > 12 * (int64_t)g.sequences && g.k <= 4096 + 4 * (g.m < 256 ? g.m : 256) * g.rank) return launch_linear_pair<T, W>(g, st);
    if (g.m <= 16) return launch_linear_small<T, W, 16>(g, st);
    if (g.m <= 32) return launch_linear_small<T, W, 32>(g, st);
    if (g.m <= 64 || ceil_div(g.m, 64) * ceil_div(g.n, 128) <= sm_count()) return launch_linear_small<T, W, 64>(g, st);
    return launch_linear_pair<T, W>(g, st);
}

}  // namespace mpq

using namespace mpq;

namespace {
// What both calls look at; `g` is filled in where they are right.
int linear_args(LinearArgs& g, const uint8_t* a, const float* a_scale, const int32_t* a_sums, int a_bits,
                const uint8_t* w, const float* w_scale, const int32_t* w_sums, int w_bits, int64_t m, int64_t n, int64_t k,
                const float* bias, int glue, const void* residual, int64_t ldr, void* out, int dtype, int64_t ldo) {
    if (m != 0 && (!a || !a_scale || !a_sums || !w || !w_scale || !w_sums || !out)) return MPQ_ERR_NULL;
    if (m < 0 || n <= 0 || k <= 0 || m > 0x7fffffff || n > 0x7fffffff || (m > 1 && (ldo < n || (residual && ldr < n)))) return MPQ_ERR_BAD_SHAPE;
    if (!bits_ok(a_bits) || !bits_ok(w_bits) || !dtype_ok(dtype) || glue < MPQ_GLUE_NONE || glue > MPQ_GLUE_SILU) return MPQ_ERR_UNSUPPORTED;
    const int64_t La = (1 << a_bits) - 1, Lw = (1 << w_bits) - 1;
    if (k > 0x7fffffff / (La * Lw)) return MPQ_ERR_OVERFLOW;
    const int e = dtype_size(dtype);
    if (!aligned16(a) || !aligned16(w) || !aligned_to(a_scale, 4) || !aligned_to(a_sums, 4) || !aligned_to(w_scale, 4) || !aligned_to(w_sums, 4) ||
        !aligned_to(bias, 4) || !aligned_to(residual, e) || !aligned_to(out, e)) return MPQ_ERR_ALIGN;
    g = LinearArgs{a, a_scale, a_sums, w, w_scale, w_sums, m, n, k, level_row_bytes(k), (int)La, (int)Lw, bias, glue, residual, ldr, out, ldo, wait_limit()};
    return MPQ_OK;
}
template <typename W>
int launch_linear_typed(const LinearArgs& g, int dtype, cudaStream_t st) {
    if (dtype == MPQ_F32) return launch_linear_levels<float, W>(g, st);
    if (dtype == MPQ_F16) return launch_linear_levels<__half, W>(g, st);
    return launch_linear_levels<__nv_bfloat16, W>(g, st);
}
}  // namespace

extern "C" int mpq_linear_levels(const uint8_t* a, const float* a_scale, const int32_t* a_sums, int a_bits,
                                 const uint8_t* w, const float* w_scale, const int32_t* w_sums, int w_bits,
                                 int64_t m, int64_t n, int64_t k,
                                 const float* bias, int glue, const void* residual, int64_t ldr,
                                 void* out, int dtype, int64_t ldo, void* stream) {
    LinearArgs g;
    const int rc = linear_args(g, a, a_scale, a_sums, a_bits, w, w_scale, w_sums, w_bits, m, n, k, bias, glue, residual, ldr, out, dtype, ldo);
    return rc != MPQ_OK || m == 0 ? rc : launch_linear_typed<void>(g, dtype, (cudaStream_t)stream);
}

extern "C" int64_t mpq_linear_adapted_workspace(int64_t m, int rank) {
    return m <= 0 || rank <= 0 ? 0 : LowWorkspace::bytes(m, rank);
}

extern "C" int mpq_linear_adapted(const uint8_t* a, const float* a_scale, const int32_t* a_sums, int a_bits,
                                  const uint8_t* w, const float* w_scale, const int32_t* w_sums, int w_bits,
                                  int64_t m, int64_t n, int64_t k,
                                  const void* down, const void* up, int adapter_dtype, const float* factor, int adapters, int rank,
                                  const int32_t* q_starts, const int32_t* ids, int batch,
                                  const float* bias, int glue, const void* residual, int64_t ldr,
                                  void* out, int dtype, int64_t ldo, void* workspace, int64_t workspace_bytes, void* stream) {
    LinearArgs g;
    int rc = linear_args(g, a, a_scale, a_sums, a_bits, w, w_scale, w_sums, w_bits, m, n, k, bias, glue, residual, ldr, out, dtype, ldo);
    if (rc != MPQ_OK) return rc;
    if (m != 0 && (!down || !up || !q_starts || (batch != 0 && !ids) || !workspace)) return MPQ_ERR_NULL;
    if (adapters <= 0 || rank <= 0 || batch < 0 || kLowParts * m > 0x7fffffff || adapters * n > 0x7fffffff) return MPQ_ERR_BAD_SHAPE;
    if ((adapter_dtype != MPQ_F16 && adapter_dtype != MPQ_BF16) || (rank != 16 && rank != 32 && rank != 64 && rank != 128)) return MPQ_ERR_UNSUPPORTED;
    if (!aligned16(down) || !aligned16(up) || !aligned16(workspace) || !aligned_to(factor, 4) || !aligned_to(q_starts, 4) || !aligned_to(ids, 4)) return MPQ_ERR_ALIGN;
    if (m == 0) return MPQ_OK;
    if (workspace_bytes < mpq_linear_adapted_workspace(m, rank)) return MPQ_ERR_WORKSPACE;
    g.up = up;
    g.rank = rank;
    g.adapters = adapters;
    g.sequences = batch;
    g.low = LowWorkspace(workspace, m, rank);
    const AdapterArgs d = {a, a_scale, g.La, m, g.row_bytes, down, factor, adapters, rank, q_starts, ids, batch, g.low};
    rc = adapter_down(d, adapter_dtype, (cudaStream_t)stream);
    if (rc != MPQ_OK) return rc;
    return adapter_dtype == MPQ_F16 ? launch_linear_typed<__half>(g, dtype, (cudaStream_t)stream) : launch_linear_typed<__nv_bfloat16>(g, dtype, (cudaStream_t)stream);
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
