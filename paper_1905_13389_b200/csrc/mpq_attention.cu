// Attention over a paged cache of levels for few query rows (mpq_cache_attention): tiles of 8 or 16 rows.
//
// A CTA of four warps takes 8 NQ query rows (tokens x heads of one key head) and a stretch of the context;
// each warp runs an online softmax of its own over every fourth chunk of 32 tokens and the four are merged
// at the end; splits of a context are joined through distributed shared memory where they are a cluster, else by
// a second kernel.  A warp copies its chunks asynchronously into a ring of its own in shared memory, one to seven of
// them under way while it works on one: 12 warps a multiprocessor keep some 100 KB in flight.  The products are
// transposed, S^T = K Q^T and O^T = V^T W^T with mma.sync.m16n8k16: tokens and dims fill the 16-wide side, eight
// query rows the other one, so a single token of a few heads wastes little.  The element order inside a dot product is free, so the 16 level bytes that a lane reads ARE its operand
// fragment, for the keys (lane = token, bytes along dim) and for the values (lane = 16 dims of a token pair);
// only W^T changes hands, by one 8 x 8 register transpose per 8 tokens.  With so few rows the work is bound by
// reading the cache, not by the matrix pipe, which is why the 256-row tcgen05 tile, mostly empty here, is not used.
#include "mpq_attention.cuh"

namespace mpq {

constexpr int kChunk = 32, kWarps = 4;
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// Operands are the even neighbours below the levels, 2u - (L + 1), exact in fp16: the level index behind a power of
// two, 1024 + u (8 bits: u below 0x64) or 16 + u (4 bits: u in bits 6-9 of 0x4c00), is a byte permutation or one shift
// and mask, and one packed multiply-add takes the power away.  The missing 1 comes back as one term per row, the sum of
// q or of w.  (The multiply-add cannot be left to such a term as well: over a long context the sum of w (1024 + u) is
// some 400 times the result, and the tensor cores' truncated sums then cost half of its bits.)
template <int BITS>
__device__ __forceinline__ uint32_t even_level(uint32_t x) {
    constexpr float c = BITS == 8 ? -2304.0f : -48.0f;
    const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&x), __float2half2_rn(2.0f), __float2half2_rn(c));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t even_nibbles(uint32_t x, int i) {
    return even_level<4>(((i == 0 ? x << 6 : i == 1 ? x << 2 : i == 2 ? x >> 2 : x >> 6) & 0x03c003c0u) | 0x4c004c00u);
}
// Word of level bytes -> operand register `pair` (0, 1: BITS = 8; 0..3: BITS = 4): elements pair*2, pair*2+1
// of the word for 8 bits, pair and pair + 4 for 4 bits.
template <int BITS>
__device__ __forceinline__ uint32_t key_pair(uint32_t w, int pair) {
    if (BITS == 8) return even_level<8>(__byte_perm(w, 0x64646464u, pair ? 0x4342 : 0x4140));
    return even_nibbles(w, pair);
}
// The words of two tokens -> operand registers of their elements side by side, `count` = 32 / BITS of them.
template <int BITS>
__device__ __forceinline__ void value_pairs(uint32_t a, uint32_t b, uint32_t* v) {
    if (BITS == 8) {
        const uint32_t lo = __byte_perm(a, b, 0x5140), hi = __byte_perm(a, b, 0x7362);       // a0 b0 a1 b1, a2 b2 a3 b3
        v[0] = even_level<8>(__byte_perm(lo, 0x64646464u, 0x4140));
        v[1] = even_level<8>(__byte_perm(lo, 0x64646464u, 0x4342));
        v[2] = even_level<8>(__byte_perm(hi, 0x64646464u, 0x4140));
        v[3] = even_level<8>(__byte_perm(hi, 0x64646464u, 0x4342));
    } else {
        const uint32_t lo = __byte_perm(a, b, 0x5410), hi = __byte_perm(a, b, 0x7632);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = even_nibbles(lo, i); v[4 + i] = even_nibbles(hi, i); }
    }
}
// Position inside a row of the element that operand register `pair` of word `word` holds in its low half
// (the high half holds + 1 for 8 bits, + 4 for 4 bits), for lane column t.
template <int D, int BITS>
__device__ __forceinline__ int key_element(int word, int pair, int t) {
    constexpr int kPerLane = D / 4;                       // elements of a lane
    constexpr int kPerWord = 32 / BITS, kWords = kPerLane / kPerWord;
    if (BITS == 8) {
        if (kWords <= 4) return t * kPerLane + word * 4 + pair * 2;
        return (word >> 2) * (D / 2) + t * 16 + (word & 3) * 4 + pair * 2;      // two 16-byte loads, half a row apart
    }
    return t * kPerLane + word * 8 + pair;
}

// N words of level bytes of a lane, from shared memory.
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
    if constexpr (N == 4) { const uint4 v = *reinterpret_cast<const uint4*>(p); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    else if constexpr (N == 2) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
    else { w[0] = *reinterpret_cast<const uint32_t*>(p); }
}
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
// Where byte `at` of token `row`'s keys and values lies in a chunk's tile: 16-byte pieces are exchanged inside a row so
// that the 8 lanes of one shared-memory access meet different banks (keys: two rows x four pieces for rows of 128 bytes;
// values: rows 2 t of four token pairs).
template <int ROW_BYTES>
__device__ __forceinline__ int key_place(int row, int at) { return row * ROW_BYTES + (ROW_BYTES == 128 ? at ^ ((row & 1) << 6) : at); }
template <int ROW_BYTES>
__device__ __forceinline__ int value_place(int row, int at) {
    return row * ROW_BYTES + (ROW_BYTES == 128 ? at ^ ((row & 7) << 4) : ROW_BYTES == 64 ? at ^ (((row >> 1) & 3) << 4) : at);
}

// Stages of a warp's ring.  Eight rows: three CTAs share a multiprocessor and 16 KB of level bytes a warp are enough;
// sixteen rows need more registers, two CTAs with 24 KB (1 context of 16384, 4 tokens of 32 heads: 24 us, with the
// smaller ring 31; 32 contexts, 1 token each: 127 us with the larger ring and two CTAs, 110 with the smaller and three).
template <int ROW_BYTES, int NQ> struct Ring {
    static constexpr int stages = (ROW_BYTES == 128 ? 2 : ROW_BYTES == 64 ? 4 : 8) * (NQ == 1 || ROW_BYTES == 32 ? 2 : 3) / 2;
    static constexpr int tile = kChunk * ROW_BYTES;       // a chunk's keys (or values)
    static constexpr int stage = 2 * tile + 2 * kChunk * 4;
    static constexpr int warp = stages * stage;
};

template <typename T, int D, int BITS, int NQ>
__global__ void __launch_bounds__(kWarps * 32, NQ == 1 ? 3 : 2)
attn_rows_kernel(const AttnArgs g) {
    constexpr int kRows = 8 * NQ;
    constexpr int kRowBytes = D * BITS / 8;
    constexpr int kKeyWords = D / 4 * BITS / 32;          // words of a key row per lane (4 lanes share a row)
    constexpr int kKeyLoads = kKeyWords > 4 ? 2 : 1;      // ... in loads of at most 16 bytes
    constexpr int kKeyStep = kKeyWords / kKeyLoads;
    constexpr int kValWords = D / 8 * BITS / 32;          // words of a value row per lane (8 lanes share a row)
    constexpr int kPairs = 16 / BITS;                     // operand registers per word (keys)
    constexpr int kSteps = D / 16;                        // k-steps of the score product, 16-dim tiles of the value product
    using R = Ring<kRowBytes, NQ>;
    constexpr int kTile = R::tile, kStages = R::stages;
    extern __shared__ __align__(128) unsigned char ring_raw[];            // [warps][stages][keys, values, ranges]; the merge's rows afterwards
    __shared__ float sh_ml[kWarps][kRows][2], sh_bad[kRows];              // sh_bad: NaN for a query row that is not finite, else 0
    float (*sh_o)[kRows][D + 4] = reinterpret_cast<float (*)[kRows][D + 4]>(ring_raw);

    chain_entry();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int gr = lane >> 2, t4 = lane & 3;
    const int kv_head = blockIdx.y;
    AttnTile t;
    if (!find_tile<kRows>(g, blockIdx.x, t)) return;
    tile_range<kRows, kChunk>(g, t);
    const int used = tile_splits(g, t);
    if ((int)blockIdx.z >= used) return;
    int begin, end;
    split_range(g, t, blockIdx.z, used, begin, end);
    const int32_t* pages_of = g.table + (int64_t)t.b * g.table_stride;

    // ---- context: this warp's chunks
    // lane's token of a chunk: its row number in the cache (all ones: there is no token), looked up before it is needed
    auto find_row = [&](int c) { return c + lane < end ? context_row(g, pages_of, c + lane, kv_head) : 0xffffffffu; };
    unsigned char* ring = ring_raw + warp * R::warp;
    auto request = [&](int stage, uint32_t row) {         // bytes and ranges of a chunk into a stage
        unsigned char* at_stage = ring + stage * R::stage;
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(at_stage);
        const uint32_t ranges = dst + 2 * kTile + lane * 4;
        if (row != 0xffffffffu) {
            copy_async4(ranges, g.k_scale + row);
            copy_async4(ranges + kChunk * 4, g.v_scale + row);
        } else {                                          // no token (range -1): read a row that is there, give it weight 0
            float* r = reinterpret_cast<float*>(at_stage + 2 * kTile);
            r[lane] = 0.0f;
            r[kChunk + lane] = -1.0f;
            row = 0u;
        }
        constexpr int kPieces = kRowBytes / 16;
#pragma unroll
        for (int x = 0; x < kPieces; ++x) {
            const int r = (x * 32 + lane) / kPieces, at = (x * 32 + lane) % kPieces * 16;
            const int64_t from = (int64_t)__shfl_sync(0xffffffffu, row, r) * kRowBytes + at;
            copy_async16(dst + key_place<kRowBytes>(r, at), g.k_levels + from);
            copy_async16(dst + kTile + value_place<kRowBytes>(r, at), g.v_levels + from);
        }
    };
    auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
    constexpr int kStride = kWarps * kChunk;
    int c0 = begin + warp * kChunk;
    uint32_t pending;
    // the page numbers and the query rows are requested together, the copies as soon as the pages are known
    uint32_t rows[kStages - 1];
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) rows[s] = find_row(c0 + s * kStride);
    pending = find_row(c0 + (kStages - 1) * kStride);
    // elements of a lane's share of a query row: 32 / BITS adjacent ones per operand word
    constexpr int kPerWord = 32 / BITS;
    T raw[NQ][kKeyWords * kPerWord];
    int q_token[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int r = t.row0 + gr + 8 * n;
        const bool live = r < t.rows;
        const int head = kv_head * g.group + (live ? r % g.group : 0);
        q_token[n] = live ? r / g.group : -1;
        const T* q = static_cast<const T*>(g.q) + (int64_t)(t.q0 + max(q_token[n], 0)) * g.q_ts + (int64_t)head * g.q_hs;
        const bool aligned = (reinterpret_cast<uintptr_t>(q) & 15u) == 0;
#pragma unroll
        for (int c = 0; c < kKeyWords * kPerWord; c += 8) {              // 8 adjacent elements
            const T* p = q + key_element<D, BITS>(c / kPerWord, 0, t4) + c % kPerWord;
            if (live && aligned) {
                *reinterpret_cast<uint4*>(&raw[n][c]) = __ldg(reinterpret_cast<const uint4*>(p));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) raw[n][c + i] = live ? p[i] : from_f32<T>(0.0f);
            }
        }
    }
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
        if (c0 + s * kStride < end) request(s, rows[s]);
        commit();
    }

    // ---- queries: row gr (+ 8) of the tile as operand fragments
    uint32_t qf[NQ][kSteps][2];
    float row_scale[NQ][2], q_sum[NQ][2];                 // of rows 2 t4 + e (+ 8): the columns of this lane's scores
    int first[NQ][2], last[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < kKeyWords * kPerWord; ++i) amax = max_nan(amax, fabsf(to_f32(raw[n][i])));
        amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        const bool finite = ordinary(amax);               // otherwise the row is computed with q = 0
        if (warp == 0 && t4 == 0) sh_bad[gr + 8 * n] = finite ? 0.0f : kNaN;
        float down, up, sum = 0.0f;
        row_power(finite ? amax : 0.0f, down, up);
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int reg = s * 2 + i, low = reg / kPairs * kPerWord + (BITS == 8 ? 2 : 1) * (reg % kPairs);   // as key_pair pairs them
                const float a = to_f32(raw[n][low]) * down, b = to_f32(raw[n][low + (BITS == 8 ? 1 : 4)]) * down;
                const __half2 h = __floats2half2_rn(finite ? a : 0.0f, finite ? b : 0.0f);
                qf[n][s][i] = *reinterpret_cast<const uint32_t*>(&h);
                sum += __low2float(h) + __high2float(h);
            }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        int from, upto;
        row_range(g, t, q_token[n], from, upto);
        if (q_token[n] < 0) { from = 0; upto = 0x7fffffff; }   // computed with q = 0, never stored: no masks on its account
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int src = (t4 * 2 + e) * 4;
            row_scale[n][e] = row_factor(__shfl_sync(0xffffffffu, up, src), g.scale_log2);
            q_sum[n][e] = __shfl_sync(0xffffffffu, sum, src);
            first[n][e] = __shfl_sync(0xffffffffu, from, src);
            last[n][e] = __shfl_sync(0xffffffffu, upto, src);
        }
    }
    int first_of_all = first[0][0], last_of_all = last[0][0];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) { first_of_all = max(first_of_all, first[n][e]); last_of_all = min(last_of_all, last[n][e]); }
    first_of_all = __reduce_max_sync(0xffffffffu, first_of_all);
    last_of_all = __reduce_min_sync(0xffffffffu, last_of_all);

    float o[kSteps][NQ][4] = {}, m[NQ][2], l[NQ][2], wsum[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) { m[n][e] = -INFINITY; l[n][e] = 0.0f; wsum[n][e] = 0.0f; }

    for (int stage = 0; c0 < end; c0 += kStride, stage = stage + 1 == kStages ? 0 : stage + 1) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");      // this chunk's copies are done
        __syncwarp();                                     // ... every lane's, and every lane has read the stage before
        if (c0 + (kStages - 1) * kStride < end) request(stage == 0 ? kStages - 1 : stage - 1, pending);
        commit();
        pending = find_row(c0 + kStages * kStride);
        const unsigned char* keys = ring + stage * R::stage;
        const unsigned char* values = keys + kTile;
        const float* ranges = reinterpret_cast<const float*>(keys + 2 * kTile);
        // scores of tokens 16 k + gr + 8 h (h: register pair) against rows 2 t4 + e
        float s[2][NQ][4] = {}, s_odd[2][NQ][4] = {};   // two chains of products each
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t kw[2][kKeyWords];                    // tokens 16 k + gr, + 8
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kKeyLoads; ++i)
                    load_words<kKeyStep>(keys + key_place<kRowBytes>(k * 16 + h * 8 + gr, t4 * (kKeyStep * 4) + i * (kRowBytes / 2)), kw[h] + i * kKeyStep);
#pragma unroll
            for (int x = 0; x < kSteps; ++x) {
                const int reg = x * 2;
                const uint32_t a[4] = {key_pair<BITS>(kw[0][reg / kPairs], reg % kPairs), key_pair<BITS>(kw[1][reg / kPairs], reg % kPairs),
                                       key_pair<BITS>(kw[0][(reg + 1) / kPairs], (reg + 1) % kPairs),
                                       key_pair<BITS>(kw[1][(reg + 1) / kPairs], (reg + 1) % kPairs)};
#pragma unroll
                for (int n = 0; n < NQ; ++n) mma_f16(x & 1 ? s_odd[k][n] : s[k][n], a, qf[n][x]);
            }
        }
        // y = x + log2 of the value's range; masks only where the chunk needs them
        const float vs = ranges[kChunk + lane];
        float lg, inv;
        range_exponent(vs, lg, inv);
        const bool here = vs != -1.0f;
        const float kf = key_factor<BITS>(ranges[lane]);
        lg = here ? lg : -INFINITY;                       // a token that is not there: weight 0
        inv = here ? inv : 0.0f;
        const bool partial = c0 < first_of_all || c0 + kChunk - 1 > last_of_all;
        float iv[2][2], top[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) top[n][0] = top[n][1] = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int src = k * 16 + h * 8 + gr;
                const float kj = __shfl_sync(0xffffffffu, kf, src), lj = __shfl_sync(0xffffffffu, lg, src);
                iv[k][h] = __shfl_sync(0xffffffffu, inv, src);
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float y = fmaf((s[k][n][h * 2 + e] + s_odd[k][n][h * 2 + e] + q_sum[n][e]) * kj, row_scale[n][e], lj);
                        if (partial && (c0 + src < first[n][e] || c0 + src > last[n][e])) y = -INFINITY;
                        s[k][n][h * 2 + e] = y;
                        top[n][e] = fmaxf(top[n][e], y);
                    }
            }
        bool grow = false;                                // also the first finite maximum
#pragma unroll
        for (int n = 0; n < NQ; ++n) grow = grow || top[n][0] > m[n][0] + kLag || top[n][1] > m[n][1] + kLag;
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int d = 4; d <= 16; d <<= 1) top[n][e] = fmaxf(top[n][e], __shfl_xor_sync(0xffffffffu, top[n][e], d));
                    if (top[n][e] > m[n][e] + kLag) {
                        const float f = fast_exp2(m[n][e] - top[n][e]);               // m = -infinity: 0
                        m[n][e] = top[n][e];
                        l[n][e] *= f; wsum[n][e] *= f;
#pragma unroll
                        for (int i = 0; i < kSteps; ++i) { o[i][n][e] *= f; o[i][n][2 + e] *= f; }
                    }
                }
        }
        uint32_t wt[2][NQ][2];                            // weights as the second operand: [token half][row group][8 tokens]
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const float ref[2] = {m[n][0] == -INFINITY ? 0.0f : m[n][0] - kBoost, m[n][1] == -INFINITY ? 0.0f : m[n][1] - kBoost};
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float w[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        w[e] = fast_exp2(s[k][n][h * 2 + e] - ref[e]);
                        l[n][e] = fmaf(w[e], iv[k][h], l[n][e]);
                    }
                    const __half2 p = __floats2half2_rn(w[0], w[1]);
                    wsum[n][0] += __low2float(p);
                    wsum[n][1] += __high2float(p);
                    wt[k][n][h] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&p));
                }
        }
        // values: dims gr D/8 + 2 i (+ 1) of the 16-dim tile i
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t vw[4][kValWords];                    // tokens 16 k + 2 t4 + {0, 1, 8, 9}
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_words<kValWords>(values + value_place<kRowBytes>(k * 16 + t4 * 2 + (i & 1) + (i >> 1) * 8, gr * (kValWords * 4)), vw[i]);
            constexpr int kPer = 32 / BITS;
#pragma unroll
            for (int word = 0; word < kValWords; ++word) {
                uint32_t low[kPer], high[kPer];
                value_pairs<BITS>(vw[0][word], vw[1][word], low);
                value_pairs<BITS>(vw[2][word], vw[3][word], high);
#pragma unroll
                for (int e = 0; e < kPer; e += 2) {
                    const uint32_t a[4] = {low[e], low[e + 1], high[e], high[e + 1]};
#pragma unroll
                    for (int n = 0; n < NQ; ++n) mma_f16(o[(word * kPer + e) / 2][n], a, wt[k][n]);
                }
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();                                      // the ring becomes the merge's buffer

    // ---- merge: rows of the four warps, then the splits (by the cluster or attn_merge_kernel) or the result
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d <= 16; d <<= 1) {
                l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
                wsum[n][e] += __shfl_xor_sync(0xffffffffu, wsum[n][e], d);
            }
            const int r = n * 8 + t4 * 2 + e;
            if (gr == 0) { sh_ml[warp][r][0] = part_reference(m[n][e], l[n][e]); sh_ml[warp][r][1] = l[n][e]; }
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                *reinterpret_cast<float2*>(&sh_o[warp][r][gr * (D / 8) + 2 * i]) = make_float2(o[i][n][e] + wsum[n][e], o[i][n][2 + e] + wsum[n][e]);
        }
    __syncthreads();
    constexpr float kInvL = 1.0f / (float)((1 << BITS) - 1);
    // one warp per row: 32 lanes along the dims
    for (int r = warp; r < kRows; r += kWarps) {
        if (t.row0 + r >= t.rows) break;
        float top = -INFINITY, den = 0.0f, f[kWarps];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh_ml[w][r][0]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float mw = sh_ml[w][r][0];
            f[w] = mw == -INFINITY ? 0.0f : fast_exp2(mw - top);
            den = mw == -INFINITY ? den : fmaf(sh_ml[w][r][1], f[w], den);
        }
        if (top != -INFINITY) den += sh_bad[r];
        const int token = (t.row0 + r) / g.group, head = kv_head * g.group + (t.row0 + r) % g.group;
        const int64_t at = (int64_t)(t.q0 + token) * g.heads + head, slot = at * g.splits + blockIdx.z;
        T* out = static_cast<T*>(g.out) + (int64_t)(t.q0 + token) * g.o_ts + (int64_t)head * g.o_hs;
#pragma unroll
        for (int d = lane; d < D; d += 32) {
            float num = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) num = fmaf(sh_o[w][r][d], f[w], num);
            num *= kInvL;
            if (g.joined && used > 1) sh_o[0][r][d] = num;               // read by this thread alone so far
            else if (used > 1) g.part_o[slot * D + d] = num;
            else out[d] = from_f32<T>(top == -INFINITY ? 0.0f : final_value(num / den));
        }
        __syncwarp();
        if (lane == 0) {
            if (g.joined && used > 1) { sh_ml[0][r][0] = top; sh_ml[0][r][1] = den; }
            else if (used > 1) g.part_ml[slot] = make_float2(top, den);
            else if (g.lse) g.lse[at] = top == -INFINITY ? -INFINITY : (top - kBoost + log2f(den)) * 0.6931471805599453f;
        }
    }
    if (!g.joined || used <= 1) return;
    // The cluster's CTAs hold a split each (those past `used` have exited, which counts as arrived): a warp joins a row
    // of all of them, read from their shared memory.  The result does not depend on which CTA's warp it is.
    cluster_sync_all();
    join_rows<T, D, kJoined>(g, t, kv_head, min(kRows, t.rows - t.row0), used, blockIdx.z * kWarps + warp, used * kWarps,
                             [&](int r) { return smem_addr(&sh_ml[0][r][0]); }, [&](int r, int d) { return smem_addr(&sh_o[0][r][d]); });
    cluster_sync_all();                                   // nobody leaves while its shared memory is read
}

// Splits of a context -> result: WARPS warps per (token, head), each with every WARPS-th split, so that the rows of up
// to 32 splits are loaded at once (one warp looping over 43 splits took 10 us).
constexpr int kMergeThreads = 256;
template <typename T, int D, int R, int CHUNK, int WARPS>
__global__ void __launch_bounds__(kMergeThreads) attn_merge_kernel(const AttnArgs g) {
    __shared__ float sh_acc[kMergeThreads / 32][D], sh_den[kMergeThreads / 32];
    chain_entry();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % WARPS;
    const int64_t at = (int64_t)blockIdx.x * (kMergeThreads / 32 / WARPS) + warp / WARPS;
    const bool exists = at < g.tokens * g.heads;
    const int token = exists ? (int)(at / g.heads) : 0, head = exists ? (int)(at % g.heads) : 0;
    // What the splits left is asked for before it is known how many there are (slots past them are in the workspace, and
    // not used): one round of loads instead of four, 1 to 2 us.
    const float2* ml = g.part_ml + at * g.splits;
    const float2 first_ml = exists && lane < g.splits ? ml[lane] : make_float2(-INFINITY, 0.0f);
    constexpr int kEarly = WARPS == 1 ? 4 : 0;               // all the splits that this form is launched for
    float early[kEarly + 1][D / 32];
#pragma unroll
    for (int s = 0; s < kEarly; ++s)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) early[s][i] = exists && s < g.splits ? g.part_o[(at * g.splits + s) * D + i * 32 + lane] : 0.0f;
    // the sequence that holds the token: the last one that starts at or before it (none: the tile itself has stored it)
    int used = 0;
    for (int base = 0; exists && base < g.batch; base += 32) {
        const int i = base + lane;
        int start = 0x7fffffff, next = 0, kv = 0;
        if (i < g.batch) { start = g.q_starts[i]; next = g.q_starts[i + 1]; kv = g.kv_lens[i]; }
        const uint32_t before = __ballot_sync(0xffffffffu, start <= token);
        if (before == 0) break;
        const int src = 31 - __clz(before);
        AttnTile t;
        t.b = base + src;
        t.q0 = __shfl_sync(0xffffffffu, start, src);
        const int64_t stop = __shfl_sync(0xffffffffu, next, src);
        t.kv_len = __shfl_sync(0xffffffffu, kv, src);
        t.n_q = (int)min(stop, g.tokens) - t.q0;
        t.rows = t.n_q * g.group;
        t.row0 = ((token - t.q0) * g.group + head % g.group) / R * R;
        used = 0;
        if (stop > token) {
            tile_range<R, CHUNK>(g, t);
            used = tile_splits(g, t);
        }
        if (before != 0xffffffffu) break;
    }
    if (used <= 1) used = 0;                                 // stored by the split itself (or not a token of any sequence)
    float top = lane < used ? first_ml.x : -INFINITY, den = 0.0f;
    for (int s = 32 + lane; s < used; s += 32) top = fmaxf(top, ml[s].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float acc[D / 32] = {};
    auto weight = [&](float2 of) {
        const float f = of.x == -INFINITY ? 0.0f : fast_exp2(of.x - top);
        if (of.x != -INFINITY) den = fmaf(of.y, f, den);
        return f;
    };
    if constexpr (WARPS == 1) {
        const float f = weight(lane < used ? first_ml : make_float2(-INFINITY, 0.0f));
#pragma unroll
        for (int s = 0; s < kEarly; ++s) {
            const float fs = __shfl_sync(0xffffffffu, f, s);
            if (s >= used) break;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) acc[i] = fmaf(early[s][i], fs, acc[i]);
        }
    } else {
        // lane i weighs split part + WARPS i; the rows are summed with the loads of four splits in flight
        for (int s0 = part; s0 < used; s0 += 32 * WARPS) {
            const int my = s0 + lane * WARPS;
            const float f = weight(my < used ? ml[my] : make_float2(-INFINITY, 0.0f));
            const int n = min(32, (used - s0 + WARPS - 1) / WARPS);
            const float* row = g.part_o + (at * g.splits + s0) * D + lane;
#pragma unroll 4
            for (int s = 0; s < n; ++s) {
                const float fs = __shfl_sync(0xffffffffu, f, s);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) acc[i] = fmaf(__ldg(row + (int64_t)s * (WARPS * D) + i * 32), fs, acc[i]);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
    if constexpr (WARPS > 1) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) sh_acc[warp][i * 32 + lane] = acc[i];
        if (lane == 0) sh_den[warp] = den;
        __syncthreads();
        if (part != 0) return;
        for (int w = 1; w < WARPS; ++w) {
            den += sh_den[warp + w];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) acc[i] += sh_acc[warp + w][i * 32 + lane];
        }
    }
    if (used == 0) return;
    T* out = static_cast<T*>(g.out) + (int64_t)token * g.o_ts + (int64_t)head * g.o_hs;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) out[i * 32 + lane] = from_f32<T>(top == -INFINITY ? 0.0f : final_value(acc[i] / den));
    if (g.lse && lane == 0) g.lse[at] = top == -INFINITY ? -INFINITY : (top - kBoost + log2f(den)) * 0.6931471805599453f;
}

// Tiles of `rows` query rows that `tokens` new tokens in at most `sequences` sequences can fill.
inline int64_t tile_bound(int64_t tokens, int64_t sequences, int group, int rows) {
    return tokens * group / rows + (tokens < sequences ? tokens : sequences);
}

struct AttnPlan { int rows; int64_t tiles; int splits, split_tokens; bool joined; };   // rows of a tile: 8, 16 or kTileRows

// Which kernel, and how far a context is split.
//   More than 32 rows per sequence and key head: 256-row tiles on the tensor cores.  A context is split only
// while the tiles do not fill the multiprocessors, in stretches of 512 tokens at least (each split hands over a row of
// fp32 results).
//   Otherwise: tiles of 8 rows where a sequence has no more, else of 16; as many splits as leave every CTA a place at
// once, three (two) to a multiprocessor: rounded down, since a second round of CTAs costs more than a few empty places
// (32 contexts of 1024 tokens: 21.9 us in 256 CTAs, 28.5 in 512 for 444 places; 8 contexts of 4000: 25.0 in 384, 24.2
// in 448).  But of no more than kLongSplit tokens, so that contexts of different lengths even out (32 contexts of up
// to 16384: 117, 110 and 127 us with 1536, 3072 and 4096, 113 with 3072 since the operands are exact).
//   Up to eight splits of a tile are one cluster and need no second launch, if all CTAs fit at once: a cluster holds its
// places until its longest split is through (one token over 8 contexts of 4000: 23.7 us with the second launch, 20.6
// without; 32 contexts of up to 16384: 113 and 150.  64 and 512 tokens over 4000, 8 and 2 splits: 39.7 and 83.3, 33.1
// and 72.1).  A GPU processing cluster of 16 to 20 multiprocessors may be unable to place up to splits - 1 CTAs of the
// form that has a multiprocessor to itself; eight of them are allowed for.
//   Short contexts are split no further than that, up to 512 tokens of a split (batches of 4, 2 and 1 over 4000: 15.6,
// 13.7 and 11.5 us in 8 splits, 17.5, 14.1 and 10.6 in 13, 27 and 32; and a call of one launch is 4 us shorter on the
// host; over 8000 20.2 and 18.0 against 17.2 and 13.1; tiles of 16 rows lose from 4000 on, 16.9 against 15.1).
constexpr int kLongSplit = 3072;
AttnPlan attn_plan(int64_t tokens, int batch, int group, int kv_heads, int64_t max_q, int64_t max_kv) {
    AttnPlan p;
    if (max_q > tokens) max_q = tokens;
    p.rows = max_q * group > 32 ? kTileRows : max_q * group > 8 ? 16 : 8;
    const int64_t context = max_kv < 1 ? 1 : max_kv > 0x7fffffff ? 0x7fffffff : max_kv;
    int64_t per, unit;
    p.tiles = tile_bound(tokens, (int64_t)batch + 1, group, p.rows);      // tokens of no sequence are one more (find_tile)
    // tiles to expect: full ones, and half a tile more per sequence; never more than the caller's bound allows
    int64_t likely = batch * ceil_div(max_q < 1 ? group : max_q * group, p.rows);
    const int64_t filled = tokens * group / p.rows + (batch + 1) / 2;
    if (likely > filled && p.rows == kTileRows) likely = filled;
    const int64_t most = tile_bound(tokens, batch, group, p.rows);
    if (likely > most) likely = most;
    if (p.rows == kTileRows) {
        unit = kStepTokens;
        int64_t splits = 148 / (likely * kv_heads);
        if (splits > ceil_div(context, 512)) splits = ceil_div(context, 512);
        per = ceil_div(context, splits < 1 ? 1 : splits);
    } else {
        unit = kChunk * kWarps;
        int64_t splits = 148 * (p.rows == 8 ? 3 : 2) / (likely * kv_heads);
        if (p.rows == 8 && splits > kJoined && context <= kJoined * 512) splits = kJoined;
        per = ceil_div(context, splits < 1 ? 1 : splits);
        if (per > kLongSplit) per = kLongSplit;
    }
    per = ceil_div(per, unit) * unit;
    if (ceil_div(context, per) > 256) per = ceil_div(ceil_div(context, 256), unit) * unit;
    p.splits = (int)ceil_div(context, per);
    p.split_tokens = (int)(per > 0x40000000 ? 0x40000000 : per);
    p.joined = p.splits > 1 && p.splits <= kJoined &&
               (p.rows == kTileRows ? likely * kv_heads * p.splits + 8 * (p.splits - 1) <= 148
                                    : likely * kv_heads * p.splits <= 148 * (p.rows == 8 ? 3 : 2));
    return p;
}

inline int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }

template <typename T, int D, int R, int CHUNK>
int launch_merge_of(const AttnArgs& g, cudaStream_t st) {
    const int64_t rows = g.tokens * g.heads;
    return g.splits > 4 ? launch_chained_as(true, attn_merge_kernel<T, D, R, CHUNK, 8>, (unsigned)rows, kMergeThreads, 0, st, g)
                        : launch_chained_as(true, attn_merge_kernel<T, D, R, CHUNK, 1>, (unsigned)ceil_div(rows, kMergeThreads / 32), kMergeThreads, 0, st, g);
}
template <typename T, int D>
int launch_merge(const AttnArgs& g, int rows, cudaStream_t st) {
    return rows == kTileRows ? launch_merge_of<T, D, kTileRows, kStepTokens>(g, st)
           : rows == 16      ? launch_merge_of<T, D, 16, kChunk>(g, st) : launch_merge_of<T, D, 8, kChunk>(g, st);
}

template <typename T, int D, int BITS>
int launch_rows(const AttnArgs& g, const AttnPlan& p, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.tiles, (unsigned)g.kv_heads, (unsigned)p.splits);
    cfg.blockDim = dim3(kWarps * 32, 1, 1);
    cfg.stream = st;
    const size_t ring = (size_t)kWarps * (p.rows == 8 ? Ring<D * BITS / 8, 1>::warp : Ring<D * BITS / 8, 2>::warp), merge = (size_t)kWarps * p.rows * (D + 4) * 4;
    cfg.dynamicSmemBytes = ring > merge ? ring : merge;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = (unsigned)p.splits;
    cfg.attrs = attr;
    cfg.numAttrs = p.joined ? 2 : 1;
    static PerDeviceOnce once8, once16;
    auto* kernel = p.rows == 8 ? attn_rows_kernel<T, D, BITS, 1> : attn_rows_kernel<T, D, BITS, 2>;
    const int rc = (p.rows == 8 ? once8 : once16).raise_smem_limit(kernel, cfg.dynamicSmemBytes);
    if (rc != MPQ_OK) return rc;
    if (cudaLaunchKernelEx(&cfg, kernel, g) != cudaSuccess) { cudaGetLastError(); return MPQ_ERR_CUDA; }
    return launch_status();
}

template <typename T, int D>
int launch_attention(const AttnArgs& g, const AttnPlan& p, int dtype, int bits, cudaStream_t st) {
    const int rc = p.rows == kTileRows ? attention_tiles(g, dtype, D, bits, p.tiles, st)
                          : bits == 8 ? launch_rows<T, D, 8>(g, p, st) : launch_rows<T, D, 4>(g, p, st);
    return rc != MPQ_OK || p.splits == 1 || p.joined ? rc : launch_merge<T, D>(g, p.rows, st);
}

}  // namespace mpq

using namespace mpq;

extern "C" int64_t mpq_cache_attention_workspace(int64_t tokens, int batch, int heads, int kv_heads, int dim,
                                                 int64_t max_q, int64_t max_kv) {
    if (tokens <= 0 || batch <= 0 || heads <= 0 || heads > 65536 || tokens > 0x7fffffff / heads || kv_heads <= 0 || heads % kv_heads || dim <= 0 ||
        max_q < 0 || max_kv < 0) return 0;
    const AttnPlan p = attn_plan(tokens, batch, heads / kv_heads, kv_heads, max_q, max_kv);
    if (p.splits <= 1 || p.joined) return 0;
    return up16(tokens * heads * p.splits * dim * 4) + up16(tokens * heads * p.splits * 8);
}

extern "C" int mpq_cache_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride, int dtype,
                                   const int32_t* q_starts, const int32_t* kv_lens, const int32_t* table, int64_t table_stride,
                                   int64_t tokens, int batch, int heads, int kv_heads, int dim, int64_t max_q, int64_t max_kv,
                                   const uint8_t* k_levels, const float* k_scale, const uint8_t* v_levels, const float* v_scale,
                                   int bits, int64_t pages, int page_size,
                                   int causal, int64_t window, float scale,
                                   void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                                   void* workspace, int64_t workspace_bytes, void* stream) {
    if (tokens != 0 && (!q || !q_starts || !kv_lens || !table || !k_levels || !k_scale || !v_levels || !v_scale || !out)) return MPQ_ERR_NULL;
    if ((dtype != MPQ_F16 && dtype != MPQ_BF16) || (bits != 8 && bits != 4) || (dim != 64 && dim != 128)) return MPQ_ERR_UNSUPPORTED;
    if (tokens < 0 || batch <= 0 || heads <= 0 || heads > 65536 || tokens > 0x7fffffff / heads || kv_heads <= 0 || heads % kv_heads || kv_heads > 65535 ||
        table_stride <= 0 || pages <= 0 || pages > 0x7fffffff || page_size <= 0 || max_q < 0 || max_kv < 0 || window < 0 ||
        (heads > 1 && out_head_stride < dim) || (tokens > 1 && out_token_stride < dim)) return MPQ_ERR_BAD_SHAPE;
    if (!(scale == scale) || scale - scale != 0.0f) return MPQ_ERR_UNSUPPORTED;
    if (!aligned16(k_levels) || !aligned16(v_levels) || !aligned_to(k_scale, 4) || !aligned_to(v_scale, 4) || !aligned_to(q, 2) ||
        !aligned_to(out, 2) || !aligned_to(lse, 4) || !aligned_to(q_starts, 4) || !aligned_to(kv_lens, 4) || !aligned_to(table, 4)) return MPQ_ERR_ALIGN;
    if (tokens == 0) return MPQ_OK;
    const int group = heads / kv_heads;
    AttnPlan p = attn_plan(tokens, batch, group, kv_heads, max_q, max_kv);
    if (p.tiles > 0x7fffffff) return MPQ_ERR_BAD_SHAPE;
    // A window leaves a tile less of its context than that: plan for what it sees, within the workspace's splits (a
    // ragged batch of 1 to 511 tokens over 5000 with a window of 1500: 61 us planned for 5000, 47 for what a tile sees).
    if (window > 0 && window < max_kv && p.splits > 1) {
        const int64_t seen = window + (causal ? p.rows / group + 1 : max_q < tokens ? max_q : tokens);
        const AttnPlan w = attn_plan(tokens, batch, group, kv_heads, max_q, seen < max_kv ? seen : max_kv);
        if (w.splits <= p.splits) { p.splits = w.splits; p.split_tokens = w.split_tokens; p.joined = w.joined; }
    }
    int page_shift = -1;
    if ((page_size & (page_size - 1)) == 0) for (page_shift = 0; (1 << page_shift) < page_size; ++page_shift) {}
    AttnArgs g = {q, q_token_stride, q_head_stride, q_starts, kv_lens, table, table_stride, tokens, batch, heads, kv_heads, heads / kv_heads,
                  k_levels, k_scale, v_levels, v_scale, pages, page_size, page_shift, causal != 0, window, scale * 1.4426950408889634f,
                  out, out_token_stride, out_head_stride, lse, nullptr, nullptr, p.splits, p.split_tokens, p.joined, wait_limit()};
    if (p.splits > 1 && !p.joined) {
        if (!workspace) return MPQ_ERR_NULL;
        if (!aligned16(workspace)) return MPQ_ERR_ALIGN;
        if (workspace_bytes < mpq_cache_attention_workspace(tokens, batch, heads, kv_heads, dim, max_q, max_kv)) return MPQ_ERR_WORKSPACE;
        g.part_o = static_cast<float*>(workspace);
        g.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + up16(tokens * heads * p.splits * dim * 4));
    }
    cudaStream_t st = (cudaStream_t)stream;
    const bool bf = dtype == MPQ_BF16;
    if (dim == 128) return bf ? launch_attention<__nv_bfloat16, 128>(g, p, dtype, bits, st) : launch_attention<__half, 128>(g, p, dtype, bits, st);
    return bf ? launch_attention<__nv_bfloat16, 64>(g, p, dtype, bits, st) : launch_attention<__half, 64>(g, p, dtype, bits, st);
}
