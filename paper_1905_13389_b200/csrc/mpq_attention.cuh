// Attention of new tokens over a paged cache of levels: what its kernels share.
//
// Mathematics.  A key or value of the cache is (2u - L) s / L with one range s per (token, head).  For a
// query row (token, head) with scores x_j = scale log2(e) q . k_j,
//   out = sum_j 2^x_j v_j / sum_j 2^x_j.
// The ranges never touch the level bytes: levels are small integers, exact in fp16, so both products run
// on the fp16 tensor pipes over the bare levels, and
//   x_j = (q . levels_j) (s^k_j / L) scale log2(e)          one fp32 multiply per score,
//   2^x_j v_j = 2^(x_j + log2 s^v_j) levels_j / L           the value's range moves into the exponent.
// With y_j = x_j + log2 s^v_j and a reference m at most 2^3 below the running maximum of y, the weights
// w_j = 2^(y_j - m + 12) lie in [0, 2^15] whatever the ranges are: that is what makes fp16 weights safe (what
// is lost is a weight below 2^-36 of the row's largest CONTRIBUTION, never a token whose score alone is small).
// The reference moves only when the maximum has outgrown it by more than 2^3, so a step usually needs neither
// a reduction of the maximum over lanes nor a rescaling of what has been summed.  The denominator is kept in fp32:
//   l = sum_j w_j / s^v_j = 2^(12 - m) sum_j 2^x_j,
// where a token drops out only if its contribution lies 2^138 below the row's largest one.
// Queries are scaled by a power of two per row before they become fp16, so nothing overflows or is lost
// beside the row's largest element.  Ranges below 2^-90 (all-zero values among them) count as 2^-90
// in the exponent, and a result below 2^-89 in magnitude is stored as 0.
// What is rounded, and what it costs.  Weights become fp16 for the tensor pipes: 2^-11 of each, of random sign, in the
// numerator alone (the denominator sums them unrounded).  Scores carry the 2 units of ex2.approx and of __log2f.  Queries
// are exact in fp16 beside the row's largest element and lose bits 2^14 below it.  On fp16 results the error against 64
// bits is 2.65e-4 of them in the root mean square where a 32-bit form has 2.07e-4, the result's own rounding; on bf16
// results 1.67e-3 and 1.66e-3 (a ragged batch over 4-bit pages; a decode step).  Weights in two fp16 parts would double the
// second product; the levels they weigh have 8 bits.
// What is not finite comes out where it is seen.  A token's NaN (or a key's infinite) range makes the scores of the
// rows that see it NaN, and with them l; maxima ignore NaNs, so a part of a row whose scores are ALL NaN has no
// reference and l = NaN, and hands its sums on with the reference +infinity, which wins every join and turns the row
// into NaNs (part_reference).  A query row that is not finite takes part as zeros, so that masks and missing tokens
// need no care, and its denominator becomes NaN at the end if it has seen anything.
#pragma once
#include "mpq_levels.cuh"
#include "mpq_tensor.cuh"

namespace mpq {

struct AttnArgs {
    const void* q; int64_t q_ts, q_hs;
    const int32_t* q_starts; const int32_t* kv_lens; const int32_t* table; int64_t table_stride;
    int64_t tokens; int batch, heads, kv_heads, group;
    const uint8_t* k_levels; const float* k_scale; const uint8_t* v_levels; const float* v_scale;
    int64_t pages; int page_size, page_shift;   // shift: log2 of a page size that is a power of two, else -1
    int causal; int64_t window;
    float scale_log2;                       // scale * log2(e)
    void* out; int64_t o_ts, o_hs; float* lse;
    float* part_o; float2* part_ml;         // [tokens][heads][splits](dim), (m, l) of each split; used where a tile has more than one split
    int splits, split_tokens;               // launch grid's splits; context tokens of one split
    int joined;                             // the splits of a tile are one cluster, which joins them (no workspace)
    uint32_t polls;                         // limit of a wait (the tensor-core form)
};

// One tile of query rows of one sequence: row r is token r / group, head kv_head * group + r % group.
struct AttnTile {
    int b, q0, n_q, rows, row0;             // sequence, its first token, tokens, n_q * group, first row of the tile
    int kv_len;
    int lo, hi;                             // context tokens that some row of the tile may see, lo a multiple of the chunk
};

// Visible range of row r: [first, last].
__device__ __forceinline__ void row_range(const AttnArgs& g, const AttnTile& t, int token, int& first, int& last) {
    const int pos = t.kv_len - t.n_q + token;
    last = g.causal ? min(pos, t.kv_len - 1) : t.kv_len - 1;
    first = g.window > 0 ? (int)max((int64_t)0, (int64_t)pos - g.window + 1) : 0;
}

// The sequence and rows of tile number `index` of R rows each, tiles counted over the sequences in order
// (all 32 lanes call; the result is the same in every lane).  False: no such tile.  Tokens past the last sequence (the
// padding of a captured step) are one sequence more, without a context: their rows see nothing and are stored as such.
template <int R>
__device__ __forceinline__ bool find_tile(const AttnArgs& g, int index, AttnTile& t) {
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int base = 0; base <= g.batch; base += 32) {
        const int b = base + lane;
        int q0 = 0, n = 0, kv = 0;
        if (b <= g.batch) {
            if (b < g.batch) kv = g.kv_lens[b];
            q0 = (int)min((int64_t)max(g.q_starts[b], 0), g.tokens);
            const int64_t next = b < g.batch ? max(g.q_starts[b + 1], q0) : g.tokens;
            n = (int)min(next, g.tokens) - q0;
        }
        const int tiles = (int)(((int64_t)n * g.group + R - 1) / R);
        int upto = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + upto > index);
        if (past) {
            const int src = __ffs(past) - 1;
            t.b = base + src;
            t.q0 = __shfl_sync(0xffffffffu, q0, src);
            t.n_q = __shfl_sync(0xffffffffu, n, src);
            t.kv_len = __shfl_sync(0xffffffffu, kv, src);
            t.row0 = (index - before - __shfl_sync(0xffffffffu, upto - tiles, src)) * R;
            t.rows = t.n_q * g.group;
            return true;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    return false;
}

// Context range of a tile of R rows (t.kv_len as the caller gave it), its start rounded down to a multiple of CHUNK.
template <int R, int CHUNK>
__device__ __forceinline__ void tile_range(const AttnArgs& g, AttnTile& t) {
    t.kv_len = (int)max((int64_t)0, min((int64_t)t.kv_len, min(g.table_stride * g.page_size, (int64_t)0x7fff0000)));
    int first, last, unused;
    row_range(g, t, t.row0 / g.group, first, unused);
    row_range(g, t, (min(t.row0 + R, t.rows) - 1) / g.group, unused, last);
    t.hi = max(last + 1, 0);
    t.lo = min(first, t.hi) / CHUNK * CHUNK;
}

// Splits that a tile with context range [lo, hi) really uses, and the tokens of split s.
__device__ __forceinline__ int tile_splits(const AttnArgs& g, const AttnTile& t) {
    return max(1, min(g.splits, (t.hi - t.lo + g.split_tokens - 1) / g.split_tokens));
}
// The last split of the grid takes whatever is left, so any split count covers the whole context.
__device__ __forceinline__ void split_range(const AttnArgs& g, const AttnTile& t, int s, int used, int& begin, int& end) {
    begin = t.lo + s * g.split_tokens;
    end = s == used - 1 ? t.hi : min(t.hi, begin + g.split_tokens);
}

// Row number in the cache (in tokens) of context token j, or 0xffffffff when its page number lies outside
// the cache.  Cache rows are counted in 32 bits: 2^32 rows of 32 bytes are more than the device holds.
__device__ __forceinline__ uint32_t context_row(const AttnArgs& g, const int32_t* pages_of, int j, int kv_head) {
    const int p = g.page_shift >= 0 ? j >> g.page_shift : j / g.page_size;
    const int32_t page = __ldg(pages_of + p);
    if ((uint32_t)page >= (uint32_t)g.pages) return 0xffffffffu;          // g.pages is below 2^31
    return ((uint32_t)page * (uint32_t)g.kv_heads + (uint32_t)kv_head) * (uint32_t)g.page_size + (uint32_t)(j - p * g.page_size);
}

constexpr float kTinyRange = 8.077935669463161e-28f;        // 2^-90
constexpr float kLag = 3.0f;                                // the reference may lie this far (log2) below a row's maximum,
constexpr float kBoost = 12.0f;                             // and weights are scaled by 2^12: up to half of fp16's largest number

// 2^x to 2 units in the last place or so; 2^-infinity = 0.
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// log2 of a value's range and the reciprocal that belongs to it (2^-that, so that rounding the logarithm
// cancels in the denominator).  The reciprocal is always finite (a NaN range gives 0): a masked token's weight
// of 0 may be multiplied by it; a row that does see such a token gets its NaN from the exponent.
__device__ __forceinline__ void range_exponent(float s, float& lg, float& inv) {
    lg = __log2f(s < kTinyRange ? kTinyRange : s);           // NaN passes through
    inv = lg == lg ? exp2f(-lg) : 0.0f;                      // may be subnormal
}
// Factor of a key's range: range / L, NaN for an infinite range (0 * infinity): a score of minus infinity would hide it.
template <int BITS>
__device__ __forceinline__ float key_factor(float s) {
    const float f = s * (1.0f / (float)((1 << BITS) - 1));
    return fmaf(s, 0.0f, f);
}
// Reference that a part of a row hands on with its denominator l: -infinity where it has seen nothing.
__device__ __forceinline__ float part_reference(float m, float l) { return m == -INFINITY && l != 0.0f ? INFINITY : m; }

__device__ __forceinline__ float final_value(float o) { return fabsf(o) < 2.0f * kTinyRange ? 0.0f : o; }

// Power of two that brings a row's largest magnitude into [1, 2), and its inverse.
__device__ __forceinline__ void row_power(float amax, float& down, float& up) {
    int e = amax > 0.0f ? (int)((__float_as_uint(amax) >> 23) & 0xff) - 127 : 0;
    e = min(max(e, -100), 126);
    down = __uint_as_float((uint32_t)(127 - e) << 23);
    up = __uint_as_float((uint32_t)(127 + e) << 23);
}
// Factor of a query row's scores, finite: times a score of 0 it has to stay 0.
__device__ __forceinline__ float row_factor(float up, float scale_log2) { return fminf(fmaxf(up * scale_log2, -3.402823466e38f), 3.402823466e38f); }

constexpr int kJoined = 8;                                // splits that a cluster can hold
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
// Joins the rows of a tile over the splits of a cluster's first `used` CTAs, at most SPLITS: warp `index` of `warps` takes
// every warps-th row.  ml_at(r) is the shared-memory address of row r's (reference, denominator), o_at(r, d) that of its
// element d, the same in every CTA.  (Two or four rows at once were slower: their registers spill.)
template <typename T, int D, int SPLITS, typename MlAt, typename OAt>
__device__ __forceinline__ void join_rows(const AttnArgs& g, const AttnTile& t, int kv_head, int rows, int used, int index, int warps, MlAt ml_at, OAt o_at) {
    const int lane = threadIdx.x & 31;
    for (int r = index; r < rows; r += warps) {
        float part[SPLITS][D / 32], ref = -INFINITY, den = 0.0f;
        if (lane < used) {
            const uint32_t at = map_to_cta(ml_at(r), lane);
            ref = ld_cluster(at);
            den = ld_cluster(at + 4);
        }
#pragma unroll
        for (int s = 0; s < SPLITS; ++s)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) part[s][i] = s < used ? ld_cluster(map_to_cta(o_at(r, i * 32 + lane), s)) : 0.0f;
        float top = ref;
#pragma unroll
        for (int o = 1; o < SPLITS; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        top = __shfl_sync(0xffffffffu, top, 0);
        const float f = ref == -INFINITY ? 0.0f : fast_exp2(ref - top);
        den = ref == -INFINITY ? 0.0f : den * f;
#pragma unroll
        for (int o = 1; o < SPLITS; o <<= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
        den = __shfl_sync(0xffffffffu, den, 0);
        float acc[D / 32] = {};
#pragma unroll
        for (int s = 0; s < SPLITS; ++s) {
            const float fs = __shfl_sync(0xffffffffu, f, s);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) acc[i] = s < used ? fmaf(part[s][i], fs, acc[i]) : acc[i];
        }
        const int row = t.row0 + r, token = t.q0 + row / g.group, head = kv_head * g.group + row % g.group;
        T* out = static_cast<T*>(g.out) + (int64_t)token * g.o_ts + (int64_t)head * g.o_hs;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) out[i * 32 + lane] = from_f32<T>(top == -INFINITY ? 0.0f : final_value(acc[i] / den));
        if (g.lse && lane == 0)
            g.lse[(int64_t)token * g.heads + head] = top == -INFINITY ? -INFINITY : (top - kBoost + log2f(den)) * 0.6931471805599453f;
    }
}

// The tensor-core form for many query rows (mpq_attention_tiles.cu).
constexpr int kTileRows = 256, kStepTokens = 128;         // rows of a CTA, context tokens of a step
int attention_tiles(const AttnArgs& g, int dtype, int dim, int bits, int64_t tiles, cudaStream_t st);
int attention_wait_failures(unsigned int* count_host, cudaStream_t st);

}  // namespace mpq
