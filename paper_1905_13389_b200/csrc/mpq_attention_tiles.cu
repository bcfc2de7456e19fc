// Attention over a paged cache of levels for many query rows (mpq_cache_attention): tiles of 256 rows on the
// 5th-generation tensor cores.
//
// A CTA takes 256 query rows (tokens x heads of one key head, two tiles of 128) and a stretch of the context
// in steps of 128 tokens.  Warps 16-19 turn level bytes into fp16 levels: keys as rows [token][dim], values
// transposed, [dim][token], both in the 128-byte swizzled K-major layout that tcgen05.mma reads; they load a
// step ahead into registers, so pages of any size cost nothing but the address arithmetic.  Warp 20 issues
//     S_h = Q_h K^T  (fp16, fp32 accumulator in TMEM),    O_h += W_h V  (W_h in TMEM, where S_h was)
// in half steps of 64 tokens, two of S_h at a time per tile, so that a tile's softmax (warps 0-7 and 8-15, 16 rows
// each) finds its next scores ready; all 512 TMEM columns are in use.  A row's reference moves only when its maximum
// has outgrown it by 2^3; the weights are then made again and its part of O_h is rescaled.
//
// What bounds it (dim 128, 8 bits; cycles per step of 128 tokens and both tiles, of 5800 measured): shared memory
// some 4900 at 128 bytes a cycle (the products' operands 2000 -- those 64 wide read Q again for every half step -- and 2900
// wavefronts of loads and stores as counted, a launch's beginning and end among them: the softmax's constants, which all
// 16 warps read, are 1500 of these, the levels' stores 500 without their conflicts), the issue slots 3200, the tensor cores
// 2000 at their full rate, the exponentials 2048 of the special-function units.  None is full, each phase waits for
// another one's.  2048 tokens over 10240, 32 heads on 8: 503 us, 615 TFLOP/s.  On the way: 1181 us with row-per-thread
// softmax and loads as they were needed, 715 with everything loaded a step ahead, 690 with constants shared by four
// rows a thread and half steps, 518 once the issuing warp ran its loop with all lanes (see mbar_wait_warp), 508 with
// sixteen softmax warps for eight.  Fetching S before the weights of the half step before are handed over was slower
// (574-635), as were more registers for eight softmax warps (543); a second issuing warp changed nothing (509).
#include "mpq_attention.cuh"

namespace mpq {

constexpr int kSoftmaxWarps = 16;                         // eight per tile
constexpr int kTileThreads = (kSoftmaxWarps + 4 + 4) * 32; // ... four that decode levels, one that issues (and three idle: register
                                                          // shares are handed out by fours): 512 x 80 + 128 x 120 + 128 x 40 = 768 x 80

__device__ unsigned int g_attention_wait_failures;

template <int D> struct TileSmem {
    static constexpr int q_half = 128 * 128;              // 128 rows x 64 elements
    static constexpr int q_tile = q_half * (D / 64);
    static constexpr int k_stage = 128 * 128 * (D / 64);  // [D / 64][128 tokens][64 dims]
    static constexpr int v_stage = D * 128 * 2;           // [2][D dims][64 tokens]
    static constexpr int q = 0, k = 2 * q_tile, v = k + 2 * k_stage, consts = v + 2 * v_stage;
    static constexpr int const_stage = 3 * kStepTokens * 4;   // [64 token pairs](key factors, value exponents), [128] value reciprocals
    static constexpr int rows = consts + 2 * const_stage;     // cache row numbers, two steps
    static constexpr int ranges = rows + 2 * kStepTokens * 4; // first and last visible token of each row
    static constexpr int scales = ranges + kTileRows * 8;     // scale of each row (and NaN if the row is not finite); at the end its (reference, denominator)
    static constexpr int total = scales + kTileRows * 8 + 1024;
};

template <int REGS> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS)); }
template <int REGS> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS)); }

__device__ __forceinline__ void st_shared16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// Two 16-bit lanes holding 2u + 1 + 1024 (as fp16 bits 0x6401 + 2u) -> fp16 level 2u - L
template <int BITS>
__device__ __forceinline__ uint32_t exact_level(uint32_t x) {
    constexpr float c = BITS == 8 ? -1280.0f : -1040.0f;
    const __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&x), __float2half2_rn(c));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Bytes sel and sel' of (a, b), zero-extended to 16 bits each by the caller's masks -> levels
__device__ __forceinline__ uint32_t level8(uint32_t spread) { return exact_level<8>(spread * 2u + 0x64016401u); }
// Nibble i (0..3) of each half word of x -> levels
__device__ __forceinline__ uint32_t level4(uint32_t x, int i) {
    return exact_level<4>(((i == 0 ? x << 1 : x >> (4 * i - 1)) & 0x001e001eu) | 0x64016401u);
}
// Eight key elements as one 16-byte chunk: in order for 8 bits; 0 4 1 5 2 6 3 7 for 4 bits (the queries are
// staged in the same order).
__device__ __forceinline__ void key_chunk8(uint32_t w0, uint32_t w1, uint32_t addr) {
    st_shared16(addr, level8(__byte_perm(w0, 0, 0x4140)), level8(__byte_perm(w0, 0, 0x4342)),
                level8(__byte_perm(w1, 0, 0x4140)), level8(__byte_perm(w1, 0, 0x4342)));
}
__device__ __forceinline__ void key_chunk4(uint32_t w, uint32_t addr) {
    st_shared16(addr, level4(w, 0), level4(w, 1), level4(w, 2), level4(w, 3));
}
// 16-byte chunk `c` of row r in a [rows][128 bytes] tile with the 128-byte swizzle
__device__ __forceinline__ uint32_t swizzled(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }

// Two fp32 operations in one instruction (sm_100's f32x2 forms).
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <typename T, int D, int BITS>
__global__ void __launch_bounds__(kTileThreads, 1)
attn_tiles_kernel(const AttnArgs g) {
    using Smem = TileSmem<D>;
    constexpr int kRowBytes = D * BITS / 8;
    constexpr uint32_t kTmemS = 0, kTmemO = 256;          // S_0, S_1: two half steps of 64 columns each; O_0, O_1: D columns each, 128 apart
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[22];
    __shared__ uint32_t tmem_holder;
    __shared__ int failed;
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    unsigned char* base_ptr = smem_raw + (base - smem_addr(smem_raw));
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t q_ready = smem_addr(&bars[0]), o_full = smem_addr(&bars[1]);
    auto k_full = [&](int s) { return smem_addr(&bars[2 + s]); };
    auto k_empty = [&](int s) { return smem_addr(&bars[4 + s]); };
    auto v_full = [&](int s) { return smem_addr(&bars[6 + s]); };
    auto v_empty = [&](int s) { return smem_addr(&bars[8 + s]); };
    auto c_empty = [&](int s) { return smem_addr(&bars[10 + s]); };      // constants of a step: read by the softmax warps
    auto s_full = [&](int h, int half) { return smem_addr(&bars[12 + 2 * h + half]); };
    auto p_ready = [&](int h, int half) { return smem_addr(&bars[16 + 2 * h + half]); };
    auto o_done = [&](int h) { return smem_addr(&bars[20 + h]); };       // W V of a half step is in O
    // element d of row r of the tile in the buffer that a cluster joins: all of the keys' and values' stages, 16-byte chunks
    // swizzled, since a thread writes along a row
    static_assert(2 * Smem::k_stage + 2 * Smem::v_stage >= kTileRows * D * 4, "no room for the rows that a cluster joins");
    auto joined_at = [](int r, int d) { return (uint32_t)(Smem::k + r * (D * 4) + (((d >> 2) ^ (r & 7)) << 4) + (d & 3) * 4); };
    auto has_failed = [&]() { return *(volatile int*)&failed != 0; };

    chain_entry();
    // ---- which rows, which part of the context (the same in every warp)
    AttnTile t;
    // later tiles see more: they go first -- but for the last one, which only tokens of no sequence can make use of
    const int last_tile = (int)gridDim.x - 1, tile_index = (int)blockIdx.x == last_tile ? last_tile : last_tile - 1 - (int)blockIdx.x;
    const int kv_head = blockIdx.y;
    if (!find_tile<kTileRows>(g, tile_index, t)) return;
    tile_range<kTileRows, kStepTokens>(g, t);
    const int used = tile_splits(g, t);
    if ((int)blockIdx.z >= used) return;
    int begin, end;
    split_range(g, t, blockIdx.z, used, begin, end);
    const int steps = (end - begin + kStepTokens - 1) / kStepTokens;
    const int tiles = t.rows - t.row0 > 128 ? 2 : 1;

    if (threadIdx.x == 0) {
        mbar_init(q_ready, 8 * tiles);
        mbar_init(o_full, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(k_full(s), 4); mbar_init(k_empty(s), 1);
            mbar_init(v_full(s), 4); mbar_init(v_empty(s), 1);
            mbar_init(c_empty(s), 8 * tiles);
            for (int half = 0; half < 2; ++half) { mbar_init(s_full(s, half), 1); mbar_init(p_ready(s, half), 8); }
            mbar_init(o_done(s), 1);
        }
        failed = 0;
        mbar_init_fence();
    }
    if (warp == kSoftmaxWarps + 4) tmem_alloc<1>(&tmem_holder, 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_holder;

    if (warp < kSoftmaxWarps) {
        // ================= softmax
        const int h = warp >> 3, sixteen = (warp >> 2) & 1, quarter = warp & 3;
        if (h < tiles) {
            int2* ranges = reinterpret_cast<int2*>(base_ptr + Smem::ranges) + h * 128;       // of the tile's rows
            float2* scales = reinterpret_cast<float2*>(base_ptr + Smem::scales) + h * 128;
            auto tile_sync = [&] { asm volatile("bar.sync %0, 256;" ::"r"(3 + h) : "memory"); };
            auto row_of_tile = [&](int in_tile, bool& live, int& token, int& head) {
                const int r = t.row0 + h * 128 + in_tile;
                live = r < t.rows;
                token = live ? r / g.group : t.n_q - 1;
                head = kv_head * g.group + (live ? r % g.group : 0);
            };
            {
                // A warp stages the 16 rows that it has in the loop as fp16, each scaled by a power of two: two threads a row,
                // every second 16 bytes each, all loads at once (a thread per row, in four rounds of loads, took 3 us more).
                const int in_tile = quarter * 32 + sixteen * 16 + (lane >> 1), odd = lane & 1;
                bool live;
                int token, head;
                row_of_tile(in_tile, live, token, head);
                const T* q = static_cast<const T*>(g.q) + (int64_t)(t.q0 + token) * g.q_ts + (int64_t)head * g.q_hs;
                uint4 raw[D / 16];
                if (!live) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) raw[c] = make_uint4(0, 0, 0, 0);
                } else if ((reinterpret_cast<uintptr_t>(q) & 15u) == 0) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) raw[c] = __ldg(reinterpret_cast<const uint4*>(q) + 2 * c + odd);
                } else {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        const unsigned short* e = reinterpret_cast<const unsigned short*>(q) + (2 * c + odd) * 8;
                        raw[c] = make_uint4(__ldg(e) | (uint32_t)__ldg(e + 1) << 16, __ldg(e + 2) | (uint32_t)__ldg(e + 3) << 16,
                                            __ldg(e + 4) | (uint32_t)__ldg(e + 5) << 16, __ldg(e + 6) | (uint32_t)__ldg(e + 7) << 16);
                    }
                }
                float amax = 0.0f;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const T* e = reinterpret_cast<const T*>(&raw[c]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) amax = max_nan(amax, fabsf(to_f32(e[i])));
                }
                amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
                const bool finite = ordinary(amax);                      // otherwise the row is computed with q = 0
                float down, up;
                row_power(finite ? amax : 0.0f, down, up);
                const uint32_t tile = base + Smem::q + h * Smem::q_tile;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const T* e = reinterpret_cast<const T*>(&raw[c]);
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int a = BITS == 8 ? 2 * i : i, b = BITS == 8 ? 2 * i + 1 : i + 4;
                        const float qa = to_f32(e[a]) * down, qb = to_f32(e[b]) * down;
                        const __half2 v = __floats2half2_rn(finite ? qa : 0.0f, finite ? qb : 0.0f);
                        w[i] = *reinterpret_cast<const uint32_t*>(&v);
                    }
                    const int at = 2 * c + odd;
                    st_shared16(tile + (at >> 3) * Smem::q_half + swizzled(in_tile, at & 7), w[0], w[1], w[2], w[3]);
                }
                if (!odd) {
                    int first, last;
                    row_range(g, t, token, first, last);
                    if (!live) { first = 0; last = 0x7fffffff; }         // computed with q = 0, never stored
                    ranges[in_tile] = make_int2(first, last);
                    scales[in_tile] = make_float2(row_factor(up, g.scale_log2), finite ? 0.0f : kNaN);
                }
                proxy_fence();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_ready);
            }
            // In the loop a warp has 16 rows, and a thread a quarter of the columns of two of them (the matrix-fragment
            // shape): row k of the thread is row (lane / 4) + 8 k of the warp's.
            const int row0 = quarter * 32 + sixteen * 16 + (lane >> 2);
            const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), mine = lanes + ((uint32_t)(sixteen * 16) << 16);
            const uint32_t ts = mine + kTmemS + h * 128, to = mine + kTmemO + h * 128;
            float set[2];                                 // the maximum that the weights' reference belongs to
            uint64_t rs[2], l[2];                         // the row's scale, twice; two partial sums
            int first_of_all = 0, last_of_all = 0x7fffffff;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float x = scales[row0 + 8 * k].x;
                rs[k] = pack2(x, x);
                set[k] = -INFINITY;
                l[k] = 0;
                const int2 seen = ranges[row0 + 8 * k];
                first_of_all = max(first_of_all, seen.x);
                last_of_all = min(last_of_all, seen.y);
            }
            first_of_all = __reduce_max_sync(0xffffffffu, first_of_all);
            last_of_all = __reduce_min_sync(0xffffffffu, last_of_all);
            bool ok = true;
#pragma unroll 1
            for (int i = 0; i < 2 * steps; ++i) {         // half steps of 64 tokens
                const int half = i & 1, st = (i >> 1) & 1, j0 = begin + i * 64;
                ok = mbar_wait_or(s_full(h, half), (i >> 1) & 1, &failed, g.polls);
                // the constants were written before the keys that S is made of
                if (half == 0) ok = ok && mbar_wait_or(k_full(st), (i >> 2) & 1, &failed, g.polls);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tmem_fence_after();
                const uint32_t from_s = ts + half * 64;
                const float4* consts = reinterpret_cast<const float4*>(base_ptr + Smem::consts + st * Smem::const_stage) + half * 32 + (lane & 3);
                const float2* inv = reinterpret_cast<const float2*>(base_ptr + Smem::consts + st * Smem::const_stage + 2 * kStepTokens * 4) + half * 32 + (lane & 3);
                uint32_t p[16];                           // weights
                uint64_t ls[2];
                // The weights are made with the reference of the half step before, in one pass over S; only when a row's
                // maximum has outgrown it (always in the first one, rarely later) is the pass repeated with a new one.
                while (true) {
                    uint64_t less[2];                     // minus the reference: set - kBoost, 0 while nothing was seen
                    float top[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float x = set[k] == -INFINITY ? 0.0f : kBoost - set[k];
                        less[k] = pack2(x, x);
                        top[k] = -INFINITY;
                        ls[k] = 0;
                    }
                    uint32_t v[32];
                    tmem_load_frag(from_s, v);
                    tmem_wait_ld();
                    uint64_t y[8][2];                     // [8-column group][row]: two neighbouring tokens each
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 kl = consts[e * 4];
                        const uint64_t kf = pack2(kl.x, kl.y), lg = pack2(kl.z, kl.w);
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            y[e][k] = fma2(mul2(pack2(__uint_as_float(v[e * 4 + k * 2]), __uint_as_float(v[e * 4 + k * 2 + 1])), kf), rs[k], lg);
                    }
                    if (j0 < first_of_all || j0 + 63 > last_of_all) {                 // some row of the warp sees only a part
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int2 seen = ranges[row0 + 8 * k];
                            const int at = j0 + 2 * (lane & 3), from = seen.x - at, upto = seen.y - at;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                float u, w;
                                unpack2(y[e][k], u, w);
                                y[e][k] = pack2(e * 8 < from || e * 8 > upto ? -INFINITY : u, e * 8 + 1 < from || e * 8 + 1 > upto ? -INFINITY : w);
                            }
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 i2 = inv[e * 4];
                        const uint64_t iv = pack2(i2.x, i2.y);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float w0, w1;
                            unpack2(y[e][k], w0, w1);
                            top[k] = max3(top[k], w0, w1);
                            unpack2(add2(y[e][k], less[k]), w0, w1);
                            w0 = fast_exp2(w0);
                            w1 = fast_exp2(w1);
                            ls[k] = fma2(pack2(w0, w1), iv, ls[k]);
                            const __half2 w = __floats2half2_rn(w0, w1);
                            p[e * 2 + k] = *reinterpret_cast<const uint32_t*>(&w);
                        }
                    }
                    // a thread's own quarter of the columns decides whether to look at the others': nearly always it does not
                    if (!__any_sync(0xffffffffu, top[0] > set[0] + kLag || top[1] > set[1] + kLag)) break;
                    float f[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
                        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
                        f[k] = 1.0f;
                        if (top[k] > set[k] + kLag) {
                            f[k] = fast_exp2(set[k] - top[k]);                        // set = -infinity: 0
                            set[k] = top[k];
                            l[k] = mul2(l[k], pack2(f[k], f[k]));
                        }
                    }
                    if (i > 0) {
                        ok = mbar_wait_or(o_done(h), (i - 1) & 1, &failed, g.polls);           // O is complete up to the half step before
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        tmem_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D / 64; ++c) {
                            uint32_t o[32];
                            tmem_load_frag(to + c * 64, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f[(e >> 1) & 1]);
                            tmem_store_frag(to + c * 64, o);
                        }
                    }
                }
                if (!ok) break;
                tmem_store_frag_half(from_s, p);
#pragma unroll
                for (int k = 0; k < 2; ++k) l[k] = add2(l[k], ls[k]);
                tmem_wait_st();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(p_ready(h, half));
                    if (half) mbar_arrive(c_empty(st));
                }
            }
            // ---- result: back to one row per thread, half of the dims for each of the two warps that share 32 rows
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float sum, odd;
                unpack2(l[k], sum, odd);
                sum += odd;
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                const float ref = part_reference(set[k], sum);
                if ((lane & 3) == 0) scales[row0 + 8 * k] = make_float2(ref, ref == -INFINITY ? sum : sum + scales[row0 + 8 * k].y);
            }
            tile_sync();
            ok = mbar_wait_or(o_full, 0, &failed, g.polls);
            ok = __all_sync(0xffffffffu, ok && !has_failed());
            {                                             // after a failure (!ok) the warp's part of the result is NaN
                tmem_fence_after();
                const int in_tile = quarter * 32 + lane;
                bool live;
                int token, head;
                row_of_tile(in_tile, live, token, head);
                if (!ok && live) scales[in_tile] = make_float2(INFINITY, kNaN);           // what a cluster joins
                const float set_row = ok ? scales[in_tile].x : INFINITY, l_row = ok ? scales[in_tile].y : kNaN;
                const bool empty = set_row == -INFINITY;
                constexpr float kInvL = 1.0f / (float)((1 << BITS) - 1);
                const int64_t at = (int64_t)(t.q0 + token) * g.heads + head;
                const float den = used > 1 && ok ? kInvL : __fdiv_rn(kInvL, l_row);
                T* out = static_cast<T*>(g.out) + (int64_t)(t.q0 + token) * g.o_ts + (int64_t)head * g.o_hs;
                const int64_t slot = at * g.splits + blockIdx.z;
                const bool aligned = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
#pragma unroll 1
                for (int c = sixteen * (D / 32); c < (sixteen + 1) * (D / 32); ++c) {        // 16 dims at a time
                    uint32_t o[16] = {};
                    if (ok && steps > 0) { tmem_load16(lanes + kTmemO + h * 128 + c * 16, o); tmem_wait_ld(); }
                    if (!live) continue;
                    float f[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) f[e] = empty ? 0.0f : __uint_as_float(o[e]) * den;
                    if (used > 1 && g.joined && !ok) continue;           // (products may still read what lies there)
                    if (used > 1 && g.joined) {                          // for the cluster, where the keys and values were
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            st_shared16(base + joined_at(h * 128 + in_tile, c * 16 + e * 4), __float_as_uint(f[e * 4]), __float_as_uint(f[e * 4 + 1]),
                                        __float_as_uint(f[e * 4 + 2]), __float_as_uint(f[e * 4 + 3]));
                    } else if (used > 1) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4)
                            *reinterpret_cast<float4*>(g.part_o + slot * D + c * 16 + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) f[e] = final_value(f[e]);
                        if (aligned) {
#pragma unroll
                            for (int e = 0; e < 16; e += 8) {
                                const float part[8] = {f[e], f[e + 1], f[e + 2], f[e + 3], f[e + 4], f[e + 5], f[e + 6], f[e + 7]};
                                store_vec<T, 8>(out + c * 16 + e, part);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 16; ++e) out[c * 16 + e] = from_f32<T>(f[e]);
                        }
                    }
                }
                if (live && sixteen == 0) {
                    if (used > 1 && !g.joined) g.part_ml[slot] = make_float2(empty ? -INFINITY : set_row, l_row);
                    else if (used == 1 && g.lse) g.lse[at] = empty ? -INFINITY : (set_row - kBoost + log2f(l_row)) * 0.6931471805599453f;
                }
                tmem_fence_before();
            }
        }
    } else if (warp < kSoftmaxWarps + 4) {
        // ================= levels: bytes of the cache -> fp16 operands
        regs_up<120>();
        const int th = threadIdx.x - kSoftmaxWarps * 32;
        const int32_t* pages_of = g.table + (int64_t)t.b * g.table_stride;
        uint32_t* row_of = reinterpret_cast<uint32_t*>(base_ptr + Smem::rows);
        // keys: kKeyLanes lanes share a row, 16 bytes each
        constexpr int kKeyLanes = kRowBytes / 16, kKeyLoads = kKeyLanes;
        const int key_row = th / kKeyLanes, key_part = th % kKeyLanes;
        // values: eight tokens and an eighth of the dims per thread; neighbouring lanes take neighbouring token groups
        constexpr int kValBytes = kRowBytes / 8, kDims = D / 8;
        const int group8 = th & 15, eighth = th >> 4;
        // Everything is loaded a step before it is needed: the page numbers two steps ahead, then the ranges, keys
        // and values of the next step while this one is converted.  row_of holds the rows of two steps; the barrier
        // at the end of step i publishes those of step i + 2 (over those of step i, whose loads are all issued).
        auto find_row = [&](int i) {                                     // this thread's token of step i
            const int j = begin + i * kStepTokens + th;
            return j < end ? context_row(g, pages_of, j, kv_head) : 0xffffffffu;
        };
        auto publish = [&](int i, uint32_t row, float& ks, float& vs) {
            row_of[(i & 1) * kStepTokens + th] = row == 0xffffffffu ? 0u : row;       // a row that can be read; weight 0
            ks = 0.0f;
            vs = -1.0f;                                                  // no token
            if (row != 0xffffffffu) { ks = __ldg(g.k_scale + row); vs = __ldg(g.v_scale + row); }
        };
        uint4 kw[kKeyLoads];
        uint32_t vw[8][kValBytes / 4];
        auto load_keys = [&](int i) {
#pragma unroll
            for (int x = 0; x < kKeyLoads; ++x) {
                const uint32_t row = row_of[(i & 1) * kStepTokens + key_row + x * (128 / kKeyLanes)];
                kw[x] = __ldg(reinterpret_cast<const uint4*>(g.k_levels + (uint64_t)row * kRowBytes + key_part * 16));
            }
        };
        auto load_values = [&](int i) {
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const uint32_t row = row_of[(i & 1) * kStepTokens + group8 * 8 + x];
                const uint8_t* p = g.v_levels + (uint64_t)row * kRowBytes + eighth * kValBytes;
                if constexpr (kValBytes == 16) { const uint4 r = __ldg(reinterpret_cast<const uint4*>(p)); vw[x][0] = r.x; vw[x][1] = r.y; vw[x][2] = r.z; vw[x][3] = r.w; }
                else if constexpr (kValBytes == 8) { const uint2 r = __ldg(reinterpret_cast<const uint2*>(p)); vw[x][0] = r.x; vw[x][1] = r.y; }
                else vw[x][0] = __ldg(reinterpret_cast<const uint32_t*>(p));
            }
        };
        float ks, vs, next_ks, next_vs;
        {
            const uint32_t r0 = find_row(0), r1 = find_row(1);
            publish(0, r0, ks, vs);
            publish(1, r1, next_ks, next_vs);
        }
        asm volatile("bar.sync 2, 128;" ::: "memory");
        load_keys(0);
        load_values(0);
        asm volatile("bar.sync 2, 128;" ::: "memory");
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
            const int st = i & 1;
            const uint32_t row2 = find_row(i + 2);
            bool ok = true;
            if (i >= 2) ok = mbar_wait_or(k_empty(st), ((i >> 1) - 1) & 1, &failed, g.polls) && mbar_wait_or(c_empty(st), ((i >> 1) - 1) & 1, &failed, g.polls);
            ok = __all_sync(0xffffffffu, ok && !has_failed());
            if (ok) {                                                    // after a failure only the barriers are kept up
                float* consts = reinterpret_cast<float*>(base_ptr + Smem::consts + st * Smem::const_stage);
                float lg, inv;
                range_exponent(vs, lg, inv);
                const bool here = vs != -1.0f;
                consts[(th >> 1) * 4 + (th & 1)] = key_factor<BITS>(ks);
                consts[(th >> 1) * 4 + 2 + (th & 1)] = here ? lg : -INFINITY;    // a token that is not there: weight 0
                consts[2 * kStepTokens + th] = here ? inv : 0.0f;
                {
                    const uint32_t tile = base + Smem::k + st * Smem::k_stage;
#pragma unroll
                    for (int x = 0; x < kKeyLoads; ++x) {
                        const int r = key_row + x * (128 / kKeyLanes);
                        const uint32_t w[4] = {kw[x].x, kw[x].y, kw[x].z, kw[x].w};
                        if constexpr (BITS == 8) {
                            // the two 8-element chunks; lanes of the two halves of a row start with different ones (banks)
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                const int z = (key_part * 2 >= 8) ^ y, c = key_part * 2 + z;
                                key_chunk8(z ? w[2] : w[0], z ? w[3] : w[1], tile + (c >> 3) * 16384 + swizzled(r, c & 7));
                            }
                        } else {
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const int c = key_part * 4 + y;
                                key_chunk4(w[y], tile + (c >> 3) * 16384 + swizzled(r, c & 7));
                            }
                        }
                    }
                }
                proxy_fence();
                __syncwarp();
                if (lane == 0) mbar_arrive(k_full(st));
                load_keys(i + 1);
            }
            if (i >= 2) ok = mbar_wait_or(v_empty(st), ((i >> 1) - 1) & 1, &failed, g.polls);
            ok = __all_sync(0xffffffffu, ok && !has_failed());
            if (ok) {
                const uint32_t tile = base + Smem::v + st * Smem::v_stage + (group8 >> 3) * (D * 128);
                constexpr int kPer = 32 / BITS;                          // dims per word
#pragma unroll
                for (int w = 0; w < kValBytes / 4; ++w)
#pragma unroll
                    for (int e = 0; e < kPer; ++e) {
                        uint32_t p[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const uint32_t a = vw[2 * x][w], b = vw[2 * x + 1][w];
                            if constexpr (BITS == 8) p[x] = level8(__byte_perm(a, b, 0x0400 + 0x0101 * e) & 0x00ff00ffu);
                            else p[x] = level4(__byte_perm(a, b, e < 4 ? 0x5410 : 0x7632), e & 3);
                        }
                        const int d = eighth * kDims + w * kPer + e;
                        st_shared16(tile + swizzled(d, group8 & 7), p[0], p[1], p[2], p[3]);
                    }
                proxy_fence();
                __syncwarp();
                if (lane == 0) mbar_arrive(v_full(st));
                load_values(i + 1);
            }
            ks = next_ks; vs = next_vs;
            // every warp has issued its loads of step i + 1 when it comes here, none still reads rows of step i
            publish(i + 2, row2, next_ks, next_vs);
            asm volatile("bar.sync 2, 128;" ::: "memory");
        }
    } else {
        // ================= tensor-core issue
        regs_down<40>();
        if (warp == kSoftmaxWarps + 4) {
            constexpr uint32_t idesc_s = umma_idesc_f16(128, 64), idesc_o = umma_idesc_f16(128, D);
            const uint32_t acc = __shfl_sync(0xffffffffu, tmem, 0);
            const bool leader = elect_one();
            bool ok = mbar_wait_warp(q_ready, 0, &failed, g.polls);
            // scores of half step i (64 tokens) of tile h; the keys of a step lie in one stage
            auto scores = [&](int h, int i) {
                const int half = i & 1, st = (i >> 1) & 1;
                const uint32_t a = umma_desc_low(base + Smem::q + h * Smem::q_tile);
                const uint32_t b = umma_desc_low(base + Smem::k + st * Smem::k_stage + half * (64 * 128));
                const uint32_t d = acc + kTmemS + h * 128 + half * 64;
                if (leader) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {                   // 16 elements = 32 bytes, 64 elements per part
                        const uint32_t at = (uint32_t)((k >> 2) * (16384 >> 4) + (k & 3) * 2);
                        umma_f16_ss(d, a + at, b + at, idesc_s, k > 0);
                    }
                    umma_commit<1>(s_full(h, half));
                }
            };
            const int halves = 2 * steps;
            if (ok && steps > 0) {
                ok = mbar_wait_warp(k_full(0), 0, &failed, g.polls);
                tmem_fence_after();
                if (ok) {
                    for (int half = 0; half < 2; ++half)
                        for (int h = 0; h < tiles; ++h) scores(h, half);
                    if (leader) umma_commit<1>(k_empty(0));
                }
            }
#pragma unroll 1
            for (int i = 0; i < halves && ok; ++i) {
                const int half = i & 1, st = (i >> 1) & 1;
                if (half == 0) {
                    ok = mbar_wait_warp(v_full(st), (i >> 2) & 1, &failed, g.polls);
                    if (ok && i + 2 < halves) ok = mbar_wait_warp(k_full(st ^ 1), ((i + 2) >> 2) & 1, &failed, g.polls);
                }
#pragma unroll 1
                for (int h = 0; h < tiles && ok; ++h) {
                    ok = mbar_wait_warp(p_ready(h, half), (i >> 1) & 1, &failed, g.polls);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t d = acc + kTmemO + h * 128, w = acc + kTmemS + h * 128 + half * 64;
                    const uint32_t b = umma_desc_low(base + Smem::v + st * Smem::v_stage + half * (D * 128));
                    if (leader) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_f16_ts(d, w + k * 8, b + k * 2, idesc_o, i > 0 || k > 0);
                        umma_commit<1>(o_done(h));
                        if (half && h == tiles - 1) umma_commit<1>(v_empty(st));
                    }
                    if (i + 2 < halves) {                                // S of this half step is free now
                        scores(h, i + 2);
                        if (half && h == tiles - 1 && leader) umma_commit<1>(k_empty(st ^ 1));
                    }
                }
            }
            if (leader) umma_commit<1>(o_full);
            mbar_wait(o_full, 0);                                        // also after a failure: TMEM is freed next
        }
    }
    __syncwarp();
    __syncthreads();
    tmem_fence_after();
    if (warp == kSoftmaxWarps + 4) tmem_free<1>(tmem, 512);
    if (used > 1 && g.joined) {
        cluster_sync_all();                                              // (CTAs past `used` have exited, which counts as arrived)
        if (warp < kSoftmaxWarps) {
            const int rows = min(kTileRows, t.rows - t.row0), index = blockIdx.z * kSoftmaxWarps + warp, warps = used * kSoftmaxWarps;
            auto ml_at = [&](int r) { return base + Smem::scales + r * 8; };
            auto o_at = [&](int r, int d) { return base + joined_at(r, d); };
            if (used == 2) join_rows<T, D, 2>(g, t, kv_head, rows, used, index, warps, ml_at, o_at);
            else join_rows<T, D, kJoined>(g, t, kv_head, rows, used, index, warps, ml_at, o_at);
        }
        cluster_sync_all();                                              // nobody leaves while its shared memory is read
    }
    if (threadIdx.x == 0 && failed) atomicAdd(&g_attention_wait_failures, 1u);
}

template <typename T, int D, int BITS>
int launch_tiles(const AttnArgs& g, int64_t tiles, cudaStream_t st) {
    static PerDeviceOnce once;
    auto* kernel = attn_tiles_kernel<T, D, BITS>;
    const int rc = once.raise_smem_limit(kernel, TileSmem<D>::total);
    if (rc != MPQ_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)tiles, (unsigned)g.kv_heads, (unsigned)g.splits);
    cfg.blockDim = dim3(kTileThreads, 1, 1);
    cfg.dynamicSmemBytes = TileSmem<D>::total;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = (unsigned)g.splits;
    cfg.attrs = attr;
    cfg.numAttrs = g.joined ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, g) != cudaSuccess) { cudaGetLastError(); return MPQ_ERR_CUDA; }
    return launch_status();
}

int attention_tiles(const AttnArgs& g, int dtype, int dim, int bits, int64_t tiles, cudaStream_t st) {
    const bool bf = dtype == MPQ_BF16;
    if (dim == 128) {
        if (bits == 8) return bf ? launch_tiles<__nv_bfloat16, 128, 8>(g, tiles, st) : launch_tiles<__half, 128, 8>(g, tiles, st);
        return bf ? launch_tiles<__nv_bfloat16, 128, 4>(g, tiles, st) : launch_tiles<__half, 128, 4>(g, tiles, st);
    }
    if (bits == 8) return bf ? launch_tiles<__nv_bfloat16, 64, 8>(g, tiles, st) : launch_tiles<__half, 64, 8>(g, tiles, st);
    return bf ? launch_tiles<__nv_bfloat16, 64, 4>(g, tiles, st) : launch_tiles<__half, 64, 4>(g, tiles, st);
}

int attention_wait_failures(unsigned int* count_host, cudaStream_t st) {
    return cudaMemcpyFromSymbolAsync(count_host, g_attention_wait_failures, sizeof(unsigned int), 0, cudaMemcpyDeviceToHost, st) == cudaSuccess &&
                   cudaStreamSynchronize(st) == cudaSuccess ? MPQ_OK : MPQ_ERR_CUDA;
}

}  // namespace mpq
