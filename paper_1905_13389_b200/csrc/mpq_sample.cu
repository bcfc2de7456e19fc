// Drawing one token a row from logits: temperature, top-k, top-p, min-p, given random numbers (mpq_sample).
//
// Which token is drawn hangs on where a running sum passes a border, so weights are 64-bit fixed-point numbers
// (whole multiples of 2^-shift of the largest weight, the nearest ones, made from 64-bit exponentials): their sums are exact whatever
// the order and borders are exact products with the row's own numbers.  shift is 62 less log2(vocab) rounded up, 50 at most, so
// that a row's sum fits: 45 for 131,072 tokens, 42 for 786,432.  A weight is off by 2^-42 of itself and half a multiple, and by no more than
// itself: what is less than half a multiple weighs nothing and is never drawn, however much of it there is.
// (With 32-bit weights a tail token of a flat row of 131,072 is another one in some percent of the draws.)
// Bound by issuing: some 30 instructions an element for a weight, 11 of them FP64.  256 x 131072 in bfloat16 by temperature take
// 87 us (memory would take 10), top-p over 256 x 151000 in 32 bits 204; a row alone is bound by latency, 30 us with every rule.
//
// A row belongs to one CTA, or where there are few rows to a cluster of up to four.  Shares that are small enough stay in shared
// memory; of larger ones only the first look goes to memory, the later ones find the row in L2.  Nothing is sorted.  Where
// top-k or top-p ends is found in three looks.  The first finds the largest logit.  The second counts elements by their distance
// from it, in 2048 steps of 1/64, which says in which steps the end lies: exactly for top-k, by counts times weights for top-p.
// The third adds up the weights -- of all, and of what lies above those steps -- and hands what lies in them (where few
// are kept: all that are kept) to every CTA of the row.  There it is counted by the bits of a code, key (the logit's bits in
// their order) before place, which no two elements share.  Where the second look was too far off the sums show it, and
// it is looked at again with the difference known.
// Where that fails (more than 2048 equals, say) the row is searched by the bits of its keys: two passes count by 11 bits each --
// exactly for top-k, with rounded weights for top-p --, and a third takes the exact sum of all above the 2^10 keys found
// and counts their members; equals have equal weights, so count times weight is exact.  Where rounding had led astray the
// search goes on from there, on the right side.
#include "mpq_attention.cuh"
#include "mpq_tensor.cuh"

namespace mpq {

typedef unsigned long long u64;

struct SampleArgs {
    const void* logits; int64_t ld;
    int vocab;
    const float *temperature; const int32_t* top_k; const float *top_p, *min_p, *uniform;
    int64_t* tokens; float* logprob;
    int shift;                                            // weights are multiples of 2^-shift: vocab 2^shift <= 2^62
    int ctas, warp_chunks;                                // CTAs of a row; 16-byte chunks that are a warp's share
    int cached;                                           // whether shares stay in shared memory
};

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;
constexpr int kSampleBins = 2048, kLowBits = 10;          // 11 + 11 + 10 bits of a key
constexpr int kSampleGroups = kSampleBins / 32;
constexpr int kSampleOwn = 4, kSampleMembers = 1024;      // members that a thread holds, and one of several CTAs hands out

// Whole numbers in the order of the logits; -0 and 0 are the same number.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// f s for 0 <= f < 1, rounded down or up to a whole number, exactly.
__device__ __forceinline__ u64 share_of(u64 s, float f, bool up) {
    const uint32_t b = __float_as_uint(f), e = b >> 23;
    const u64 m = e ? (b & 0x7fffffu) | 0x800000u : b;
    const int shift = 150 - (int)(e ? e : 1);             // f = m 2^-shift, shift >= 24
    const u64 lo = m * s, hi = __umul64hi(m, s);
    if (m == 0) return 0;
    u64 q, rest;
    if (shift < 64) { q = hi << (64 - shift) | lo >> shift; rest = lo << (64 - shift); }
    else if (shift == 64) { q = hi; rest = lo; }
    else if (shift < 128) { q = hi >> (shift - 64); rest = lo | hi << (128 - shift); }
    else { q = 0; rest = 1; }
    return q + (up && rest ? 1 : 0);
}

__device__ __forceinline__ u64 ld_cluster64(uint32_t addr) {
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_cluster32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld_cluster32x2(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}

struct SampleBorder {                                      // the bin in which a sum is reached: the sums before and with it, the counts
    u64 above, above_to;
    uint32_t digit, count, count_to;
    float edge;                                           // the smallest number in it, or over it
};
// What passes between a row's CTAs, two of each: one is written while others may still read the one before.
struct SampleShared {
    u64 parts[2][2][kSampleWarps];
    uint32_t bins[2][kSampleBins];
    uint32_t offsets[kSampleBins];                        // sums of 1/256 of a step by which a bin's members lie behind its beginning
    u64 coarse[2][2][kSampleGroups];                      // what groups of 32 bins are worth, and their counts
    int noted[2], found;                                  // members a CTA hands out; a place
    double rest[kSampleWarps], rest_all;                  // (the latter of a CTA, for the others)
    // within a CTA
    SampleBorder border[2];
    u64 scan[kSampleWarps], sums[2][kSampleWarps];
    double powers[16];                                    // 2^(i / 16 + shift): sixteen, so that lanes never ask one bank for two of them
    uint32_t digit, differ[2];
    u64 above, weight, members, member;
    u64 codes[kSampleThreads], ordered[kSampleThreads];   // few members, one to a thread: their codes, their weights in the codes' order
};

// The largest element of a chunk, NaN if one is.
__device__ __forceinline__ float chunk_max(const uint4& r, const float*) {
    return max_nan(max_nan(__uint_as_float(r.x), __uint_as_float(r.y)), max_nan(__uint_as_float(r.z), __uint_as_float(r.w)));
}
template <typename T, typename Two>
__device__ __forceinline__ float chunk_max_pairs(const uint4& r) {
    const Two* e = reinterpret_cast<const Two*>(&r);
    const Two m = __hmax2_nan(__hmax2_nan(e[0], e[1]), __hmax2_nan(e[2], e[3]));
    return max_nan(to_f32(m.x), to_f32(m.y));
}
__device__ __forceinline__ float chunk_max(const uint4& r, const __half*) { return chunk_max_pairs<__half, __half2>(r); }
__device__ __forceinline__ float chunk_max(const uint4& r, const __nv_bfloat16*) { return chunk_max_pairs<__nv_bfloat16, __nv_bfloat162>(r); }

// exp((x - top) / warm) 2^shift, rounded: 2^(t / 16) with t = n + f is 2^(n / 16) from the table and the exponent, times
// the series of 2^(f / 16), |f| <= 1/2, off by 2^-42 of itself at most.
struct SampleWeight {
    float top, cool2, lowest;                             // 2 / temperature; below `lowest` weights are less than a quarter of a multiple
    double dtop, cool;
    const double* powers;
    static constexpr u64 kBias = 0x433ull << 52;          // 2^52: on top of it, the low bits of a number are its whole part

    __device__ SampleWeight(float largest, float warm, int shift, const double* table)
        : top(largest), cool2(fminf(2.0f / warm, 3e38f)), lowest((float)((double)largest - 0.69314718055994530942 * (double)(shift + 2) * (double)warm)),
          dtop(largest), cool(16.0 * 1.4426950408889634073599 / (double)warm), powers(table) {}
    __device__ __forceinline__ u64 biased(float x) const {
        constexpr double kMagic = 6755399441055744.0;     // 1.5 2^52: on top of it, the low bits are the nearest whole number
        constexpr double kLog = 0.69314718055994530942 / 16;
        const double d = (double)x - dtop, m = fma(d, cool, kMagic), f = fma(d, cool, -(m - kMagic));
        const int n = __double2loint(m);
        const double a = powers[n & 15];
        double q = fma(f, kLog * kLog * kLog * kLog * kLog / 120, kLog * kLog * kLog * kLog / 24);
        q = fma(f, q, kLog * kLog * kLog / 6);
        q = fma(f, q, kLog * kLog / 2);
        q = fma(f, q, kLog);
        const double scaled = __hiloint2double(__double2hiint(a) + (n & ~15) * 65536, __double2loint(a));
        return (u64)__double_as_longlong(fma(scaled * f, q, scaled) + 4503599627370496.0);
    }
    __device__ __forceinline__ bool small(float x) const { return x < lowest; }
    // In 32 bits, as a share of the largest; a guess (at temperatures below 2^-127 a poor one).  Two logits can lie farther apart than
    // the largest number, half of that cannot.
    __device__ __forceinline__ float guess(float x) const { return fast_exp2(fmaf(0.5f, x, -0.5f * top) * cool2 * 1.4426950408889634f); }
    __device__ __forceinline__ u64 operator()(float x) const {
        u64 w = 0;
        if (!small(x)) w = biased(x) - kBias;
        return x > -INFINITY ? w : 0ull;
    }
};

template <typename T>
struct SampleRow {
    static constexpr int E = 16 / (int)sizeof(T);         // elements of a chunk
    SampleShared& sh;
    const T* x0;                                          // the row
    const int vocab, skew;                                // skew: place of its first element; places count from the 16-byte boundary before it
    uint4* chunks;                                        // this warp's share, where it is cached
    const bool cached;
    const int ctas, rank, warp, lane, warp_chunks;
    const int v0;                                         // place of the share's first element
    int turn = 0;                                         // which of the two exchange buffers comes next

    __device__ SampleRow(SampleShared& s, uint4* data, const SampleArgs& g)
        : sh(s), x0(static_cast<const T*>(g.logits) + (int64_t)(blockIdx.x / (unsigned)g.ctas) * g.ld), vocab(g.vocab),
          skew((int)(reinterpret_cast<uintptr_t>(x0) & 15) / (int)sizeof(T)), cached(g.cached != 0), ctas(g.ctas), rank(g.ctas > 1 ? (int)cluster_rank() : 0),
          warp(__shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0)), lane(threadIdx.x & 31), warp_chunks(g.warp_chunks),
          v0((rank * kSampleWarps + warp) * g.warp_chunks * E) {
        chunks = data + warp * warp_chunks;
    }

    __device__ __forceinline__ void sync() {
        if (ctas > 1) cluster_sync_all();
        else __syncthreads();
    }
    __device__ __forceinline__ uint32_t peer(const void* p, int cta) const { return ctas > 1 ? map_to_cta(smem_addr(p), (uint32_t)cta) : smem_addr(p); }

    static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[E]) {
        const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = to_f32(e[i]);
    }
    // Chunk c of the share from memory, -infinity where the row is not.
    __device__ __forceinline__ uint4 read_chunk(int c) const {
        const int i = v0 + c * E - skew;
        if (i >= 0 && i + E <= vocab) return *reinterpret_cast<const uint4*>(x0 + i);
        uint4 r;
        T* e = reinterpret_cast<T*>(&r);
#pragma unroll
        for (int q = 0; q < E; ++q) e[q] = i + q >= 0 && i + q < vocab ? x0[i + q] : from_f32<T>(-INFINITY);
        return r;
    }
    // Chunks c, c + 32, .. of the share, asked for together.
    template <int N>
    __device__ __forceinline__ void read_chunks(int c, uint4 (&in)[N], bool from_memory) const {
        if (!from_memory) {
#pragma unroll
            for (int j = 0; j < N; ++j) in[j] = chunks[c + 32 * j];
        } else if (v0 >= skew && v0 + warp_chunks * E - skew <= vocab) {         // every share but a row's first and last ones
            const uint4* from = reinterpret_cast<const uint4*>(x0 + (v0 - skew)) + c;
#pragma unroll
            for (int j = 0; j < N; ++j) in[j] = from[32 * j];
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) in[j] = read_chunk(c + 32 * j);
        }
    }
    // f(v, values) for this lane's elements of the share, eight at a time (a share is whole groups of them), the next eight on
    // their way; place_of(v, i) is where the i-th of them lies.
    static constexpr int kParts = 8 / E, kGroup = 32 * kParts;             // chunks of a warp's step
    static __device__ __forceinline__ int place_of(int v, int i) { return v + i % E + i / E * 32 * E; }
    template <typename F>
    __device__ __forceinline__ void each_group(F f) const {
        uint4 next[kParts];
        read_chunks(lane, next, !cached);
#pragma unroll 1
        for (int c = lane; c < warp_chunks; c += kGroup) {
            float x[8];
#pragma unroll
            for (int j = 0; j < kParts; ++j) {
                float e[E];
                unpack(next[j], e);
#pragma unroll
                for (int i = 0; i < E; ++i) x[j * E + i] = e[i];
            }
            read_chunks(c + kGroup < warp_chunks ? c + kGroup : lane, next, !cached);
            f(v0 + c * E, x);
        }
    }
    // Element i of the share of warp w of this CTA.
    __device__ __forceinline__ void element(int w, int i, int& place, float& x) const {
        place = v0 + (w - warp) * warp_chunks * E + i;
        if (cached) x = to_f32(reinterpret_cast<const T*>(chunks + (w - warp) * warp_chunks)[i]);
        else x = place >= skew && place - skew < vocab ? to_f32(x0[place - skew]) : -INFINITY;
    }
    // f(place, value) for all elements of the share.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        each_group([&](int v, const float (&x)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (x[i] > -INFINITY) f(place_of(v, i), x[i]);
        });
    }

    // Every warp's numbers -> all of the row's warps, four to a lane, the same in all warps of all CTAs.
    __device__ __forceinline__ void collect(int which, int of_turn, u64 (&v)[4]) const {
        const u64* part = sh.parts[of_turn][which];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = lane * 4 + i;
            v[i] = n < ctas * kSampleWarps ? ld_cluster64(peer(part + n % kSampleWarps, n / kSampleWarps)) : 0;
        }
    }
    __device__ __forceinline__ void gather(u64 mine, u64 (&v)[4]) {
        if (lane == 0) sh.parts[turn][0][warp] = mine;
        sync();
        collect(0, turn, v);
        turn ^= 1;
    }
    static __device__ __forceinline__ u64 warp_sum(u64 s) {
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        return s;
    }
    __device__ __forceinline__ u64 warp_scan(u64 x) const {
        for (int o = 1; o < 32; o <<= 1) {
            const u64 below = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += below;
        }
        return x;
    }
    __device__ __forceinline__ u64 block_scan(u64 x) {
        x = warp_scan(x);
        if (lane == 31) sh.scan[warp] = x;
        __syncthreads();
        const u64 before = warp_sum(lane < warp ? sh.scan[lane] : 0);
        __syncthreads();
        return x + before;
    }
    __device__ __forceinline__ u64 row_sum(u64 s) {
        u64 v[4];
        gather(warp_sum(s), v);
        return warp_sum(v[0] + v[1] + v[2] + v[3]);
    }
    // Sum of f over the share.
    template <typename F>
    __device__ __forceinline__ u64 sum(F f) const {
        u64 s = 0;
        each([&](int place, float x) { s += f(place, x); });
        return s;
    }
    // A group's weights, f(i, weight + kBias) each: sums of them are corrected once, modulo 2^64.
    template <typename F>
    static __device__ __forceinline__ void weigh(const SampleWeight& weight, const float (&x)[8], F f) {
        float low = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) low = fminf(low, x[i]);
        if (!weight.small(low) && low > -INFINITY) {      // (without a branch between them they are made side by side)
#pragma unroll
            for (int i = 0; i < 8; ++i) f(i, weight.biased(x[i]));
            return;
        }
        float live[8], least = weight.top;                 // forbidden tokens among ordinary ones: the same beside a choice
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            live[i] = x[i] > -INFINITY ? x[i] : weight.top;
            least = fminf(least, live[i]);
        }
        if (!weight.small(least)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const u64 w = weight.biased(live[i]);
                f(i, x[i] > -INFINITY ? w : SampleWeight::kBias);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f(i, weight(x[i]) + SampleWeight::kBias);
        }
    }

    // The lowest place at which the running sum of f exceeds goal(sum of all), in the one thread that finds it (-1 elsewhere).
    // `s`: this thread's part of the sum of f over its warp.  The warp in whose share it lies is found first, then that
    // share is gone through by all warps of its CTA, a sixteenth each, then a sixteenth by one warp.
    template <typename F, typename Goal>
    __device__ __forceinline__ int running(u64 s, F f, Goal goal_of) {
        u64 v[4];
        gather(warp_sum(s), v);
        const u64 here = v[0] + v[1] + v[2] + v[3], upto = warp_scan(here), all = __shfl_sync(0xffffffffu, upto, 31), goal = goal_of(all);
        const int in = __ffs(__ballot_sync(0xffffffffu, upto > goal)) - 1;      // the lane that holds the warp in question
        if (in < 0) return -1;
        u64 before = upto - here;
        int which = lane * 4;
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (which == lane * 4 + i && before + v[i] <= goal) { before += v[i]; ++which; }
        which = __shfl_sync(0xffffffffu, which, in);
        before = __shfl_sync(0xffffffffu, before, in);
        if (which / kSampleWarps != rank) return -1;
        which %= kSampleWarps;
        // a sixteenth by each warp, several reads under way
        const int n = warp_chunks * E, per = (n + kSampleWarps - 1) / kSampleWarps, from = min(n, warp * per), to = min(n, from + per);
        u64 part = 0;
        constexpr int kAtOnce = 8;
#pragma unroll 1
        for (int i = from + lane; i < to; i += 32 * kAtOnce) {
            int place[kAtOnce];
            float x[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) element(which, min(i + 32 * j, to - 1), place[j], x[j]);
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) part += i + 32 * j < to ? f(place[j], x[j]) : 0;
        }
        part = warp_sum(part);
        if (lane == 0) sh.scan[warp] = part;
        __syncthreads();
        const u64 sums_to = warp_scan(lane < kSampleWarps ? sh.scan[lane] : 0) + before;
        const int sixteenth = __ffs(__ballot_sync(0xffffffffu, sums_to > goal)) - 1;
        if (sixteenth < 0) return -1;
        if (sixteenth > 0) before = __shfl_sync(0xffffffffu, sums_to, sixteenth - 1);
        __syncthreads();
        // ... and that one by all threads, in their order
        const int last = min(n, (sixteenth + 1) * per);
#pragma unroll 1
        for (int i0 = sixteenth * per; i0 < last; i0 += kSampleThreads) {
            const int i = i0 + (int)threadIdx.x;
            int place = 0;
            float x = 0.0f;
            u64 w = 0;
            if (i < last) {
                element(which, i, place, x);
                w = f(place, x);
            }
            const u64 upto_here = before + block_scan(w);
            if (threadIdx.x == kSampleThreads - 1) sh.above = upto_here;
            __syncthreads();
            before = sh.above;
            if (before > goal) return upto_here > goal && upto_here - w <= goal ? place : -1;
            __syncthreads();
        }
        return -1;
    }

    __device__ __forceinline__ uint32_t* clear_bins() {
        uint32_t* bins = sh.bins[turn];
        for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) bins[i] = 0;
        __syncthreads();
        return bins;
    }
    // Adds up what the CTAs have counted by bins, worth(bin, count, offsets) of each, and finds, from the highest bin down, those in
    // which the sum reaches goals(sum of all, ..) (the lowest that has anything, if none does): sh.border, N of them.  Groups of
    // 32 bins are summed by each CTA and looked at first, so that little passes between the CTAs.
    template <int N, typename Worth, typename Goals, typename Edge>
    __device__ __forceinline__ void find_borders(Worth worth, Goals goals, Edge edge) {
        __syncthreads();
        for (int i = warp; i < kSampleGroups; i += kSampleWarps) {
            const int bin = i * 32 + lane;
            const u64 n = sh.bins[turn][bin], value = warp_sum(worth(bin, (uint32_t)n, sh.offsets[bin])), all = warp_sum(n);
            if (lane == 0) { sh.coarse[turn][0][i] = value; sh.coarse[turn][1][i] = all; }
        }
        sync();
        if (warp < N) {                                   // a warp for each
            // two groups a lane, the highest first
            u64 value[2] = {}, n[2] = {};
            for (int c = 0; c < ctas; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int group = kSampleGroups - 1 - 2 * lane - i;
                    value[i] += ld_cluster64(peer(&sh.coarse[turn][0][group], c));
                    n[i] += ld_cluster64(peer(&sh.coarse[turn][1][group], c));
                }
            const u64 to = warp_scan(value[0] + value[1]), n_to = warp_scan(n[0] + n[1]);
            u64 goal[N];
            goals(__shfl_sync(0xffffffffu, to, 31), goal);
            const uint32_t any = __ballot_sync(0xffffffffu, (n[0] | n[1]) != 0);
            const u64 here_goal = warp == 0 ? goal[0] : goal[N - 1];
            const uint32_t reach = __ballot_sync(0xffffffffu, to >= here_goal);
            const int in = reach ? __ffs(reach) - 1 : 31 - __clz(any);          // something has been counted
            const bool second = reach ? to - value[1] < here_goal : n[1] != 0;
            const int group = __shfl_sync(0xffffffffu, kSampleGroups - 1 - 2 * lane - (second ? 1 : 0), in);
            const u64 before = __shfl_sync(0xffffffffu, to - value[1] - (second ? 0 : value[0]), in);
            const u64 n_before = __shfl_sync(0xffffffffu, n_to - n[1] - (second ? 0 : n[0]), in);
            const int bin = group * 32 + 31 - lane;
            u64 here = 0, w = 0;
            for (int c = 0; c < ctas; ++c) {
                const uint32_t one = ld_cluster32(peer(&sh.bins[turn][bin], c));
                here += one;
                w += worth(bin, one, ld_cluster32(peer(&sh.offsets[bin], c)));
            }
            const u64 upto = before + warp_scan(w), n_upto = n_before + warp_scan(here);
            const uint32_t reaches = __ballot_sync(0xffffffffu, upto >= here_goal), anything = __ballot_sync(0xffffffffu, here != 0);
            const int at = reaches ? __ffs(reaches) - 1 : 31 - __clz(anything);
            const float number = edge(warp, (uint32_t)__shfl_sync(0xffffffffu, bin, at));
            if (lane == at) sh.border[warp] = SampleBorder{upto - w, upto, (uint32_t)bin, (uint32_t)here, (uint32_t)n_upto, number};
        }
        __syncthreads();
        turn ^= 1;
    }

    // Distance of an element from the largest in steps (of which `twice` are two logits), rounded the same way for equals and never
    // against the order (NaN only for what is not over -infinity).  Bins count the steps down from the highest, the lowest one for
    // all beyond.
    static __device__ __forceinline__ float distance(float x, float top, float twice) { return fmaf(-0.5f, x, 0.5f * top) * twice; }
    // The smallest number whose distance is below `limit` (1 or more), by a warp: distances never grow with the number.
    __device__ __forceinline__ float nearest_below(float top, float twice, float limit) const {
        uint32_t lo = 0x00800000u, hi = order_key(top);   // from the lowest finite number on; hi's distance is 0
        for (int turn = 0; lo < hi && turn < 16; ++turn) {                 // (eight turns at most)
            const uint32_t step = (hi - lo) / 32 + 1, at = min(lo + lane * step, hi);
            const uint32_t yes = __ballot_sync(0xffffffffu, at == hi || distance(key_value(at), top, twice) < limit);
            if (yes == 0) {
                lo += 31 * step + 1;
            } else {
                const uint32_t f = (uint32_t)__ffs(yes) - 1;
                hi = min(lo + f * step, hi);
                lo = f == 0 ? hi : min(hi, lo + (f - 1) * step + 1);
            }
        }
        return key_value(hi);
    }
    // What lies in bins from `digit` up is this number or more.
    __device__ __forceinline__ float least_of(float top, float twice, uint32_t digit) const {
        return digit == 0 ? key_value(0x00800000u) : digit >= kSampleBins ? INFINITY : nearest_below(top, twice, (float)(kSampleBins - (int)digit));
    }
    // Where members are handed out: in the exchange's bins, both of them where there is no exchange.
    __device__ __forceinline__ u64* members_of(int of_turn) const { return reinterpret_cast<u64*>(sh.bins[ctas > 1 ? of_turn : 0]); }
    __device__ __forceinline__ int most_members() const { return ctas > 1 ? kSampleMembers : 2 * kSampleMembers; }
    // Hands out those of a group that `mask` names (called by whole warps: one of them is asked for room).
    __device__ __forceinline__ void note(uint32_t mask, int v, const float (&x)[8]) {
        if (!__any_sync(0xffffffffu, mask)) return;
        const int mine = __popc(mask);
        int at = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int below = __shfl_up_sync(0xffffffffu, at, o);
            if (lane >= o) at += below;
        }
        int from = 0;
        if (lane == 31) from = atomicAdd(&sh.noted[turn], at);
        at += __shfl_sync(0xffffffffu, from, 31) - mine;
        u64* members = members_of(turn);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (mask >> i & 1) {
                if (at < most_members()) members[at] = code_of(place_of(v, i), x[i]);
                ++at;
            }
    }
    // An element's place in the order, the larger the earlier.
    static __device__ __forceinline__ u64 code_of(int place, float x) { return (u64)order_key(x) << 32 | (uint32_t)~place; }

    // Sum of a number over the CTA's threads, the same in all of them.
    __device__ __forceinline__ u64 block_sum(u64 v, int& phase) {
        v = warp_sum(v);
        if (lane == 0) sh.sums[phase][warp] = v;
        __syncthreads();
        v = sh.sums[phase][lane % kSampleWarps];
        for (int o = kSampleWarps / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        phase ^= 1;
        return v;
    }
    // The largest code at which the sum of f over the codes from it on reaches goal, where that of all does: ten bits at a
    // time, from the highest one in which those with f differ, until one is left.
    __device__ __forceinline__ u64 resolve(const u64 (&code)[kSampleOwn], const u64 (&f)[kSampleOwn], u64 goal) {
        constexpr int kBits = 10, kPer = (1 << kBits) / kSampleThreads;
        u64* bins = reinterpret_cast<u64*>(sh.bins[turn]);
        if (threadIdx.x == 0) {
            sh.differ[0] = sh.differ[1] = 0;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSampleOwn; ++i) if (f[i]) sh.member = code[i];            // any one
        __syncthreads();
        const u64 ref = sh.member;
        u64 other = 0;
#pragma unroll
        for (int i = 0; i < kSampleOwn; ++i) if (f[i]) other |= code[i] ^ ref;
        const uint32_t hi = __reduce_or_sync(0xffffffffu, (uint32_t)(other >> 32)), lo = __reduce_or_sync(0xffffffffu, (uint32_t)other);
        if (lane == 0) {
            if (hi) atomicOr(&sh.differ[0], hi);
            if (lo) atomicOr(&sh.differ[1], lo);
        }
        __syncthreads();
        const u64 differ = (u64)sh.differ[0] << 32 | sh.differ[1];
        if (differ == 0) return ref;
        int at = 64 - __clzll((long long)differ);         // all codes agree from this bit up
        u64 prefix = at < 64 ? ref >> at : 0;
        for (;;) {
            const int shift = max(at - kBits, 0), width = at - shift;
#pragma unroll
            for (int i = 0; i < kPer; ++i) bins[threadIdx.x + i * kSampleThreads] = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kSampleOwn; ++i)
                if (f[i] && (at == 64 || code[i] >> at == prefix)) atomicAdd(bins + (code[i] >> shift & ((1u << width) - 1)), f[i]);
            __syncthreads();
            u64 n[kPer], mine = 0;
            const int first = (1 << kBits) - 1 - (int)threadIdx.x * kPer;
#pragma unroll
            for (int i = 0; i < kPer; ++i) { n[i] = bins[first - i]; mine += n[i]; }
            u64 before = block_scan(mine) - mine;
            if (before < goal && before + mine >= goal) {
                bool open = true;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    if (open && before + n[i] >= goal) { sh.digit = (uint32_t)(first - i); sh.above = before; open = false; }
                    before += n[i];
                }
            }
            __syncthreads();
            prefix = prefix << width | sh.digit;
            goal -= sh.above;
            at = shift;
            const u64 below = differ & (((u64)1 << at) - 1);
            const int next = 64 - __clzll((long long)below);                // bits that none differ in are passed over
            int left = 0;
#pragma unroll
            for (int i = 0; i < kSampleOwn; ++i)
                if (f[i] && code[i] >> at == prefix) { ++left; sh.member = code[i]; }
            const bool one = __syncthreads_or(left > 1) == 0 && __syncthreads_count(left == 1) == 1;
            if (one || below == 0) return sh.member;
            prefix = prefix << (at - next) | (ref >> next & (((u64)1 << (at - next)) - 1));
            at = next;
        }
    }
    // How many of the members, one to a thread, have a larger code.
    __device__ __forceinline__ int rank_of(u64 code, int members) {
        sh.codes[threadIdx.x] = code;
        __syncthreads();
        int rank = 0;
        if (warp * 32 < members)
#pragma unroll 4
            for (int i = 0; i < members; ++i) rank += sh.codes[i] > code;
        return rank;
    }
    // resolve() of as many members as threads, one to a thread: by their ranks.
    __device__ __forceinline__ u64 resolve_few(u64 code, u64 f, int members, u64 goal) {
        const int rank = rank_of(code, members);
        sh.ordered[threadIdx.x] = 0;
        __syncthreads();
        if (code) sh.ordered[rank] = f;
        __syncthreads();
        const u64 here = sh.ordered[threadIdx.x], upto = block_scan(here);
        if (upto >= goal && upto - here < goal) sh.digit = threadIdx.x;
        __syncthreads();
        if (code && rank == (int)sh.digit) sh.member = code;
        __syncthreads();
        return sh.member;
    }
    // Whether no CTA has been given more than it can hand out, nor all together more than one can take.
    __device__ __forceinline__ bool can_take(int noted_turn) const {
        const uint32_t n = lane < ctas ? ld_cluster32(peer(&sh.noted[noted_turn], lane)) : 0;
        return __all_sync(0xffffffffu, n <= (uint32_t)most_members()) && __reduce_add_sync(0xffffffffu, min(n, 4096u)) <= kSampleThreads * kSampleOwn;
    }
    __device__ __forceinline__ int handed(int noted_turn) const {
        int n = 0;
        for (int c = 0; c < ctas; ++c) n += (int)ld_cluster32(peer(&sh.noted[noted_turn], c));
        return n;
    }
    // Takes the members that the CTAs have noted, OWN to a thread in their order; 0 behind the last.
    template <int OWN>
    __device__ __forceinline__ void take_members(int noted_turn, u64 (&code)[OWN]) {
        int end = 0, c = -1, n = 0;
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int at = (int)threadIdx.x * OWN + i;
            while (at >= end && c + 1 < ctas) { n = (int)ld_cluster32(peer(&sh.noted[noted_turn], ++c)); end += n; }
            code[i] = at < end ? ld_cluster64(peer(members_of(noted_turn) + (at - (end - n)), c)) : 0;
        }
    }
};

// PER_SM: CTAs to a multiprocessor, one where there are no more (some of what it holds does not fit the registers of half of one).
template <typename T, int PER_SM>
__global__ void __launch_bounds__(kSampleThreads, PER_SM) sample_kernel(const SampleArgs g) {
    extern __shared__ uint4 held[];
    __shared__ SampleShared sh;
    constexpr int E = SampleRow<T>::E;
    SampleRow<T> r(sh, held, g);
    const int lane = r.lane, skew = r.skew;
    if (threadIdx.x < 16) sh.powers[threadIdx.x] = exp2((double)threadIdx.x / 16.0 + (double)g.shift);
    chain_entry();
    const int64_t row = blockIdx.x / g.ctas;
    const float warm = g.temperature ? g.temperature[row] : 1.0f;
    const int k = g.top_k ? g.top_k[row] : 0;
    const float p = g.top_p ? g.top_p[row] : 1.0f, least = g.min_p ? g.min_p[row] : 0.0f, u = g.uniform[row];

    // the first of the row's order, and NaNs
    float best = -INFINITY;
    int best_chunk = 0;
    bool nan = false;
    constexpr int kLoads = 4;
    auto ask = [&](int c0, uint4 (&in)[kLoads]) {         // (what is not there is asked for twice instead)
#pragma unroll
        for (int j = 0; j < kLoads; j += SampleRow<T>::kParts) {
            uint4 some[SampleRow<T>::kParts];
            r.read_chunks(c0 + 32 * j < g.warp_chunks ? c0 + 32 * j : lane, some, true);
#pragma unroll
            for (int i = 0; i < SampleRow<T>::kParts; ++i) in[j + i] = some[i];
        }
    };
    uint4 next[kLoads];
    ask(lane, next);
#pragma unroll 1
    for (int c0 = lane; c0 < g.warp_chunks; c0 += 32 * kLoads) {
        uint4 in[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) in[j] = next[j];
        ask(c0 + 32 * kLoads, next);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int c = c0 + 32 * j;
            if (c >= g.warp_chunks) break;
            if (r.cached) r.chunks[c] = in[j];
            const float top = chunk_max(in[j], static_cast<const T*>(nullptr));
            if (!(top <= best)) {
                nan |= top != top;
                best = top;
                best_chunk = c;
            }
        }
    }
    // Small k: where m warps have j elements each that are no smaller than some number, and m j is k or more, the first k are no
    // smaller either.  The number is the m-th largest of the warps' j-th largest among their threads' own largest elements;
    // with m three quarters of the warps it leaves some two or three times k.
    const bool some = k > 0 && k < g.vocab;
    const int warps = min((int)(((int64_t)g.vocab + skew + g.warp_chunks * E - 1) / (g.warp_chunks * E)), g.ctas * kSampleWarps);      // that have elements
    const int per_warp = (int)min((4 * (int64_t)k + 3 * warps - 1) / (3 * warps), (int64_t)64);
    const bool by_threads = some && per_warp <= 24;
    u64 last = 0;                                         // the key of that element
    if (by_threads) {
        uint32_t key = order_key(best);
#pragma unroll
        for (int size = 2; size <= 32; size *= 2)         // sorted by the warp, the largest first
#pragma unroll
            for (int o = size / 2; o > 0; o >>= 1) {
                const uint32_t other = __shfl_xor_sync(0xffffffffu, key, o);
                const bool falling = (lane & size) == 0 || size == 32;
                key = ((lane & o) == 0) == falling ? max(key, other) : min(key, other);
            }
        last = __shfl_sync(0xffffffffu, key, per_warp - 1);
    }
    u64 code = 0;                                         // 0: nothing over -infinity; all ones: a NaN
    if (best > -INFINITY) {
        float x[E];
        SampleRow<T>::unpack(r.cached ? r.chunks[best_chunk] : r.read_chunk(best_chunk), x);
        int at = E - 1;
#pragma unroll
        for (int q = E - 1; q >= 0; --q) if (x[q] == best) at = q;
        code = (u64)order_key(best) << 32 | (uint32_t)~(r.v0 + best_chunk * E + at);
    }
    if (nan) code = ~0ull;
    float reach = -INFINITY;
    {
        u64 v[4];
        for (int o = 16; o > 0; o >>= 1) code = max(code, __shfl_xor_sync(0xffffffffu, code, o));
        if (lane == 0) sh.parts[r.turn][1][r.warp] = last;
        const int turn = r.turn;
        r.gather(code, v);
        code = max(max(v[0], v[1]), max(v[2], v[3]));
        for (int o = 16; o > 0; o >>= 1) code = max(code, __shfl_xor_sync(0xffffffffu, code, o));
        if (by_threads) {
            r.collect(1, turn, v);
            const int m = (k + per_warp - 1) / per_warp;
            int over[4] = {}, from[4] = {};                // how many are larger, and no smaller
            for (int l = 0; l < g.ctas * kSampleWarps / 4; ++l)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t other = __shfl_sync(0xffffffffu, (uint32_t)v[i], l);
#pragma unroll
                    for (int q = 0; q < 4; ++q) { over[q] += other > (uint32_t)v[q]; from[q] += other >= (uint32_t)v[q]; }
                }
            uint32_t mth = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) if (over[q] < m && from[q] >= m) mth = (uint32_t)v[q];
            reach = key_value(max(__reduce_max_sync(0xffffffffu, mth), 0x00800000u));      // (finite, where there are fewer than k)
        }
    }
    const float top = key_value((uint32_t)(code >> 32));
    const int first = (int)~(uint32_t)code;
    const bool greedy = warm <= 0.0f;
    const bool bad = code == 0 || code == ~0ull || warm != warm || p != p || least != least || u != u || (!greedy && top == INFINITY);
    if (bad) {
        if (r.rank == 0 && threadIdx.x == 0) {
            g.tokens[row] = -1;
            if (g.logprob) g.logprob[row] = kNaN;
        }
        if (g.ctas > 1) cluster_sync_all();               // nobody leaves while others read its numbers
        return;
    }

    const bool top_p = p < 1.0f;
    const bool cut_off = !greedy && ((some && !by_threads) || (top_p && !some));
    const SampleWeight weight(top, warm, g.shift, sh.powers);
    const u64 floor_w = least > 0.0f ? (u64)ceil(fmin((double)least, 4.0) * exp2((double)g.shift)) : 0ull;
    const bool all_stay = !some && !top_p && floor_w <= 1;
    const float twice = some ? 128.0f : 64.0f * fminf(weight.cool2, 2e30f);
    // The second look, for whatever is wanted: counts of distances; the sum of all weights; and what the others weigh together at
    // temperature 1, the first one's weight being 1 -- where it has nearly all of the probability its logarithm is
    // -log(1 + rest).  That one in 32 bits: a term is off by (2.5 |d| + 4) 2^-24 of itself at most, d its distance from the first.
    constexpr uint32_t kNear = 512 << 8;                   // eight steps of a factor e
    u64 weights = 0;
    auto look = [&](bool distances, bool sums, bool others) {
        uint32_t* bins = sh.bins[r.turn];
        if (distances) {
            for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) bins[i] = sh.offsets[i] = 0;
            __syncthreads();
        }
        float rest = 0.0f;
        auto one = [&](int v, const float (&x)[8]) {
            if (distances) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (x[i] > -INFINITY) {
                        // in 1/256 of a step, rounded down: on top of 2^23 the low bits are whole numbers
                        const uint32_t away = __float_as_uint(__fadd_rd(fminf(r.distance(x[i], top, twice), (float)kSampleBins - 0.25f) * 256.0f, 8388608.0f)) - 0x4b000000u;
                        const uint32_t bin = kSampleBins - 1 - (away >> 8);
                        atomicAdd(bins + bin, 1u);
                        // 32-bit logits that many share a bin lie anywhere in it
                        if (!some && (sizeof(T) == 2 || away < kNear)) atomicAdd(sh.offsets + bin, away & 255u);
                    }
            }
            if (sums) {
                r.weigh(weight, x, [&](int, u64 w) { weights += w; });
                weights -= 8 * SampleWeight::kBias;
            }
            if (others) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = fast_exp2((x[i] - top) * 1.4426950408889634f);
                if (first >= v && first <= r.place_of(v, 7)) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) if (r.place_of(v, i) == first) e[i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) rest += e[i];
            }
        };
        if (distances || sums || others) r.each_group(one);
        if (others) {
            double sum = rest;
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) sh.rest[r.warp] = sum;
            __syncthreads();
            sum = sh.rest[lane % kSampleWarps];
            for (int o = kSampleWarps / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (threadIdx.x == 0) sh.rest_all = sum;
        }
    };
    look(cut_off, !greedy && all_stay, g.logprob != nullptr);
    // by one thread of the row, after an exchange between its CTAs
    auto finish = [&](int v, float x) {
        g.tokens[row] = v - skew;
        if (!g.logprob) return;
        double rest = 0.0;
        for (int c = 0; c < g.ctas; ++c) rest += __longlong_as_double((long long)ld_cluster64(r.peer(&sh.rest_all, c)));
        g.logprob[row] = (float)(((double)x - (double)top) - log1p(rest));
    };
    if (greedy) {
        r.sync();
        if (r.rank == 0 && threadIdx.x == 0) finish(first, top);
        if (g.ctas > 1) cluster_sync_all();
        return;
    }

    // kept: keys over `edge`, and those equal to it up to place `cut`
    uint32_t edge = 0;
    int cut = 0x7fffffff;
    auto kept = [&](int v, float x) { const uint32_t key = order_key(x); return key > edge || (key == edge && v <= cut); };
    // The key, and the place among the equals of it, at which the sum of f from the top reaches `goal`: edge and cut.
    // f: one, or (weights) the weight -- that is guessed at first, one at least, in 32 bits that hold the sum of what is open.
    const float unit = exp2f((float)g.shift);
    auto narrow = [&](u64 goal, auto f, bool weights) {
        const u64 total = r.row_sum(r.sum([&](int v, float x) { return kept(v, x) ? f(x) : 0ull; }));
        if (total <= goal) return;                        // all of it stays
        uint32_t over = 1u << (32 - kLowBits), under = 0xffffffffu;        // the border lies below `over` and above `under` (key >> kLowBits)
        u64 base = 0;                                     // f's sum from `over` on
        int64_t bias = 0;                                 // by how much the guesses above `under` fall short
        auto as_counted = [](uint32_t, uint32_t n, uint32_t) { return (u64)n; };
        for (int turns = 0; turns < 1 << 16; ++turns) {   // (each one takes at least one occupied key off the open ones)
            auto open = [&](uint32_t key) { const uint32_t high = key >> kLowBits; return high < over && (under == 0xffffffffu || high > under); };
            const float scale = weights ? 4.2e9f / ((float)(total - base) * 1.0001f) : 1.0f, per = scale * unit;
            auto guess = [&](float x) { return weights ? max(1u, __float2uint_rn(weight.guess(x) * per)) : 1u; };
            const u64 want = (u64)max((int64_t)((double)(goal - base) * (double)scale) - bias, (int64_t)1);
            u64 above1 = 0, above2 = 0;
            uint32_t high = 0;
#pragma unroll 1
            for (int level = 0; level < 2; ++level) {
                uint32_t* bins = r.clear_bins();
                r.each([&](int v, float x) {
                    const uint32_t key = order_key(x);
                    if ((level == 0 || key >> 21 == high) && open(key) && kept(v, x)) {
                        atomicAdd(bins + (level ? key >> kLowBits & (kSampleBins - 1) : key >> 21), guess(x));
                    }
                });
                above1 += above2;
                const u64 left = want > above1 ? want - above1 : 1;
                r.template find_borders<1>(as_counted, [&](u64, u64 (&goal)[1]) { goal[0] = left; }, [](int, uint32_t) { return 0.0f; });
                above2 = sh.border[0].above;
                high = level ? high << 11 | sh.border[0].digit : sh.border[0].digit;
            }
            high = min(high, (1u << (32 - kLowBits)) - 1);
            // exactly: what lies above, and how many have each of the keys found
            uint32_t* bins = r.clear_bins();
            u64 s = 0;
            r.each([&](int v, float x) {
                const uint32_t key = order_key(x);
                if (key >> kLowBits >= high && kept(v, x)) {
                    if (key >> kLowBits == high) atomicAdd(bins + (key & ((1 << kLowBits) - 1)), 1u);
                    else s += f(x);
                }
            });
            const int turn = r.turn;
            const u64 sum = r.row_sum(s);
            const int lo = (1 << kLowBits) - 1 - 2 * (int)threadIdx.x;     // this thread's keys: lo, lo - 1
            u64 n[2] = {0, 0}, w[2];
            for (int c = 0; c < g.ctas; ++c) {
                const uint2 two = ld_cluster32x2(r.peer(&sh.bins[turn][lo - 1], c));
                n[0] += two.y;
                n[1] += two.x;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = n[i] ? f(key_value(high << kLowBits | (uint32_t)(lo - i))) : 0;
            const u64 mine = n[0] * w[0] + n[1] * w[1], upto = sum + r.block_scan(mine);
            if (threadIdx.x == kSampleThreads - 1) sh.above = upto;
            __syncthreads();
            const u64 down_to = sh.above;                 // f's sum from the lowest of these keys on
            __syncthreads();
            if (sum >= goal) { under = high; bias = (int64_t)((double)(sum - base) * (double)scale) - (int64_t)(above1 + above2); continue; }
            if (down_to < goal) { over = high; base = down_to; bias = 0; continue; }
            if (upto >= goal && upto - mine < goal) {
                const int i = upto - n[1] * w[1] >= goal ? 0 : 1;
                sh.digit = (uint32_t)(lo - i);
                sh.above = upto - n[1] * w[1] - (i ? 0 : n[0] * w[0]);
                sh.weight = w[i];
                sh.members = n[i];
            }
            __syncthreads();
            const uint32_t e = high << kLowBits | sh.digit;
            const u64 wanted = (goal - sh.above + sh.weight - 1) / sh.weight;
            int c = e == edge ? cut : 0x7fffffff;
            if (wanted < sh.members) {                    // the place of the last one wanted
                auto equal = [&](int v, float x) { return (u64)(order_key(x) == e && kept(v, x)); };
                const int place = r.running(r.sum(equal), equal, [&](u64) { return wanted - 1; });
                if (place >= 0)
                    for (int q = 0; q < g.ctas; ++q) st_cluster(r.peer(&sh.found, q), (uint32_t)place);
                r.sync();
                c = sh.found;
                r.turn ^= 1;
            }
            edge = e;
            cut = c;
            __syncthreads();
            break;
        }
    };
    auto drawn = [&](u64 all) { return u >= 1.0f ? all - 1 : u > 0.0f ? share_of(all, u, false) : 0ull; };
    auto share = [&](u64 all) { return max(p > 0.0f ? share_of(all, p, true) : 0ull, 1ull); };
    u64 all = 0;                                          // top-p without top-k: what the row weighs, once it is known
    bool open = !all_stay;                                // whether it is still to be found what stays
    bool summed = all_stay;                               // whether `weights` is the sum of what stays
    int64_t bias = 0;
    int phase = 0;
    const bool least_only = !some && !top_p;              // min-p alone: two steps below its border at most
    bool by_reach = by_threads;
#pragma unroll 1
    for (int tries = 0; open && tries < 4; ++tries) {
        float outer, inner = INFINITY;                    // what is handed out is `outer` or more and below `inner`
        bool few = true;                                  // ... is all that can stay
        u64 above = 0, above_to = 0;
        if (by_reach) {
            outer = reach;
        } else if (least_only) {
            outer = r.nearest_below(top, twice, least >= 1.0f ? 3.0f : -64.0f * logf(least) + 2.0f);
        } else {
            if (tries > 0) look(true, false, false);
            // the weight of a bin's members is that of their mean distance, off by some 2^-15 of itself; 2^-12 on both sides
            auto worth = [&](uint32_t bin, uint32_t n, uint32_t offsets) -> u64 {
                if (some) return n;
                if (bin == 0 || n == 0) return 0ull;
                const bool exact = sizeof(T) == 2 || kSampleBins - 1 - bin < (kNear >> 8);
                const float away = (float)(kSampleBins - 1 - bin) + (exact ? ((float)offsets / (float)n + 0.5f) * (1.0f / 256.0f) : 0.5f);
                return (u64)((float)n * (fast_exp2(away * (-1.4426950408889634f / 64.0f)) * unit));
            };
            r.template find_borders<2>(worth, [&](u64 guessed, u64 (&goal)[2]) {
                if (some) { goal[0] = goal[1] = (u64)k; return; }
                const int64_t margin = (int64_t)(guessed >> 12), aim = (int64_t)(tries == 0 ? share(guessed) : share(all)) + bias;
                goal[0] = (u64)max(aim - margin, (int64_t)1);
                goal[1] = (u64)max(aim + margin, (int64_t)1);
            }, [&](int which, uint32_t digit) { return r.least_of(top, twice, which == 0 ? digit + 1 : digit); });
            const SampleBorder hi = sh.border[0], lo = sh.border[1];
            above = hi.above;
            above_to = lo.above_to;
            const uint32_t most = (uint32_t)(kSampleThreads * kSampleOwn);
            few = lo.count_to <= most;
            outer = lo.edge;
            if (!few) {
                inner = hi.edge;
                if (lo.count_to - (hi.count_to - hi.count) > most) break;
            }
        }
        // The third look.
        const int turn = r.turn;
        if (threadIdx.x == 0) sh.noted[turn] = 0;
        __syncthreads();
        u64 s = 0, total = 0;                             // of what lies above `inner`, of all
        const bool sums = top_p && !some;
        if (sums) {
            r.each_group([&](int v, const float (&x)[8]) {
                uint32_t mask = 0;
                uint32_t over = 0;
                r.weigh(weight, x, [&](int i, u64 w) {
                    total += w;
                    if (x[i] >= inner) { s += w; ++over; }
                    mask |= x[i] >= outer && x[i] < inner ? 1u << i : 0u;
                });
                total -= 8 * SampleWeight::kBias;
                s -= over * SampleWeight::kBias;
                r.note(mask, v, x);
            });
        } else {
            uint32_t n = 0;
            r.each_group([&](int v, const float (&x)[8]) {
                uint32_t mask = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    n += x[i] >= inner;
                    mask |= x[i] >= outer && x[i] < inner ? 1u << i : 0u;
                }
                r.note(mask, v, x);
            });
            s = n;
        }
        __syncthreads();
        const u64 mine = SampleRow<T>::warp_sum(s);
        total = SampleRow<T>::warp_sum(total);
        if (lane == 0) sh.parts[turn][1][r.warp] = total;
        u64 v[4];
        r.gather(mine, v);
        if (!r.can_take(turn)) {
            if (!by_reach) break;
            by_reach = false;                             // the largest ones lie with few threads: they are counted after all
            continue;
        }
        const u64 sum = SampleRow<T>::warp_sum(v[0] + v[1] + v[2] + v[3]);
        if (sums && tries == 0) {
            r.collect(1, turn, v);
            all = SampleRow<T>::warp_sum(v[0] + v[1] + v[2] + v[3]);
        }
        const int handed = r.handed(turn);
        if (few && handed <= kSampleThreads) {
            // A member a thread.  Its rank among the codes orders the weights, sums over that order say where top-k and top-p end,
            // and sums over the smaller places which one is drawn.
            u64 own[1];
            r.take_members(turn, own);
            const u64 mine = own[0], w = mine ? weight(key_value((uint32_t)(mine >> 32))) : 0;
            const int rank = r.rank_of(mine, handed);
            const int kept = some ? min(k, handed) : handed;
            sh.ordered[threadIdx.x] = 0;
            __syncthreads();
            if (mine && rank < kept) sh.ordered[rank] = w;
            __syncthreads();
            const u64 at_rank = sh.ordered[threadIdx.x];
            const u64 upto = r.block_scan(at_rank);
            if (threadIdx.x == kSampleThreads - 1) sh.above = upto;
            if (threadIdx.x == 0) sh.digit = (uint32_t)kept;
            __syncthreads();
            if (top_p) {
                const u64 whole = sh.above, goal = share(some ? whole : all);
                if (whole < goal) { bias += (int64_t)(above_to - whole); continue; }       // (top-p alone: too short a guess)
                if (at_rank && upto >= goal && upto - at_rank < goal) sh.digit = threadIdx.x + 1;
                __syncthreads();
            }
            const bool stays = mine && rank < (int)sh.digit && (w >= floor_w || rank == 0);
            sh.ordered[threadIdx.x] = stays ? w : 0;       // (now beside the codes; nobody reads the ranks' any more)
            __syncthreads();
            u64 before = 0;                                // what stays at smaller places
            if (r.warp * 32 < handed)
#pragma unroll 4
                for (int i = 0; i < handed; ++i) before += (uint32_t)sh.codes[i] > (uint32_t)mine ? sh.ordered[i] : 0ull;
            const u64 point = drawn(r.block_sum(stays ? w : 0, phase));
            if (r.rank == 0 && stays && before <= point && before + w > point) {
                const int place = (int)~(uint32_t)mine;
                finish(place, to_f32(r.x0[place - skew]));
            }
            if (g.ctas > 1) cluster_sync_all();
            return;
        }
        u64 code[kSampleOwn], w[kSampleOwn], f[kSampleOwn], whole = 0;
        if (handed <= kSampleThreads) {
            u64 own[1];
            r.take_members(turn, own);
#pragma unroll
            for (int i = 0; i < kSampleOwn; ++i) code[i] = i == 0 ? own[0] : 0ull;
        } else {
            r.take_members(turn, code);
        }
#pragma unroll
        for (int i = 0; i < kSampleOwn; ++i) {
            w[i] = code[i] ? weight(key_value((uint32_t)(code[i] >> 32))) : 0;
            f[i] = some ? (u64)(code[i] != 0) : w[i];
            whole += f[i];
        }
        whole = r.block_sum(whole, phase);
        u64 e = 0;
        if (!least_only) {
            const u64 goal = some ? (u64)k : share(all);
            if (sum + whole < goal) {                     // fewer over -infinity than top-k lets stay, or too short a guess
                if (!some) { bias += (int64_t)(above_to - (sum + whole)); continue; }
            } else if (sum >= goal) {
                bias += (int64_t)(above - sum);
                continue;
            } else {
                e = handed <= kSampleThreads ? r.resolve_few(code[0], f[0], handed, goal - sum) : r.resolve(code, f, goal - sum);
            }
        }
        open = false;
        if (!few) {
            edge = (uint32_t)(e >> 32);
            cut = (int)~(uint32_t)e;
            if (sums && floor_w <= 1) {                   // what lies above, and the kept ones of what was handed out
                if (threadIdx.x < kSampleWarps) sh.sums[0][threadIdx.x] = 0;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kSampleOwn; ++i) {
                    const int owner = (int)~(uint32_t)code[i] / (g.warp_chunks * E) - r.rank * kSampleWarps;
                    if (code[i] >= e && code[i] && owner >= 0 && owner < kSampleWarps) atomicAdd(&sh.sums[0][owner], w[i]);
                }
                __syncthreads();
                weights = s + (lane == 0 ? sh.sums[0][r.warp] : 0ull);
                summed = true;
            }
            break;
        }
        if (some && top_p) {
            u64 left = 0;
#pragma unroll
            for (int i = 0; i < kSampleOwn; ++i) {
                f[i] = code[i] >= e ? w[i] : 0;
                left += f[i];
            }
            left = r.block_sum(left, phase);
            e = max(e, r.resolve(code, f, share(left)));
        }
        u64 left = 0;
#pragma unroll
        for (int i = 0; i < kSampleOwn; ++i) {
            f[i] = code[i] >= e && (w[i] >= floor_w || (int)~(uint32_t)code[i] == first) ? w[i] : 0;
            left += f[i];
            if (!f[i]) code[i] = 0;
            code[i] &= 0xffffffffull;                     // in the order of the places from here on
        }
        left = r.block_sum(left, phase);
        const int place = (int)~(uint32_t)r.resolve(code, f, drawn(left) + 1);
        if (r.rank == 0 && threadIdx.x == 0) finish(place, to_f32(r.x0[place - skew]));
        if (g.ctas > 1) cluster_sync_all();
        return;
    }
    if (open && some) narrow((u64)k, [](float) { return 1ull; }, false);
    if (top_p && (some || open)) {
        const u64 left = r.row_sum(r.sum([&](int v, float x) { return kept(v, x) ? weight(x) : 0ull; }));
        narrow(share(left), weight, true);
    }
    auto stays = [&](int v, float x) {
        if (!kept(v, x)) return 0ull;
        const u64 w = weight(x);
        return w >= floor_w || v == first ? w : 0ull;
    };
    const int place = r.running(summed ? weights : r.sum(stays), stays, drawn);
    if (place >= 0) finish(place, to_f32(r.x0[place - skew]));
    if (g.ctas > 1) cluster_sync_all();
}

constexpr int kSampleMost = 786432;                       // elements of a row (half of that in 32 bits)
constexpr int kSampleHeld = 76 * 1024;                    // bytes of shares with which two CTAs fit a multiprocessor

template <typename T>
int launch_sample(SampleArgs g, int64_t rows, cudaStream_t st) {
    constexpr int E = 16 / (int)sizeof(T);
    const int sms = sm_count();
    if (sms == 0) return MPQ_ERR_CUDA;
    // More CTAs to a row, up to four, while the device has room for all rows' at once and a CTA 8192 elements.  Many CTAs that wait for one another
    // cost more than they bring: us with 1 / 2 / 4 / 8 of them, 1 x 131072 in 32 bits 47 / 36 / 32 / 39, 7 x 50021 72 / 52 / 45 / 48,
    // 64 x 131072 in 16 bits 203 / 134 / 106 / 141, 256 x 151000 205 / 216 / 278 / 519.
    const bool aligned = aligned16(g.logits) && (rows == 1 || g.ld % E == 0);
    const int64_t chunks = ceil_div((int64_t)g.vocab + (aligned ? 0 : E - 1), E);
    g.ctas = 1;
    while (g.ctas < 4 && rows * g.ctas <= sms && g.vocab / g.ctas >= 8192) g.ctas *= 2;
    constexpr int kGroup = SampleRow<T>::kGroup;
    g.warp_chunks = (int)ceil_div(chunks, g.ctas * kSampleWarps * kGroup) * kGroup;
    const int share = g.warp_chunks * kSampleWarps * 16;
    g.cached = share <= kSampleHeld;
    if (rows * g.ctas > 0x7fffffff) return MPQ_ERR_BAD_SHAPE;
    static PerDeviceOnce once[2];
    const bool alone = rows * g.ctas <= sms;
    auto* kernel = alone ? sample_kernel<T, 1> : sample_kernel<T, 2>;
    const int rc = once[alone].raise_smem_limit(kernel, kSampleHeld);
    if (rc != MPQ_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * g.ctas), 1, 1);
    cfg.blockDim = dim3(kSampleThreads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)(g.cached ? share : 0);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)g.ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kernel, g) != cudaSuccess) { cudaGetLastError(); return MPQ_ERR_CUDA; }
    return launch_status();
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_sample(const void* logits, int64_t ld, int dtype, int64_t rows, int64_t vocab,
                          const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* uniform,
                          int64_t* tokens, float* logprob, void* stream) {
    if (rows != 0 && (!logits || !uniform || !tokens)) return MPQ_ERR_NULL;
    if (rows < 0 || rows > 0x7fffffff || vocab <= 0 || (rows > 1 && ld < vocab)) return MPQ_ERR_BAD_SHAPE;
    if (!dtype_ok(dtype) || vocab > kSampleMost / (dtype == MPQ_F32 ? 2 : 1)) return MPQ_ERR_UNSUPPORTED;
    if (!aligned_to(logits, dtype_size(dtype)) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) || !aligned_to(top_p, 4) || !aligned_to(min_p, 4) ||
        !aligned_to(uniform, 4) || !aligned_to(tokens, 8) || !aligned_to(logprob, 4)) return MPQ_ERR_ALIGN;
    if (rows == 0) return MPQ_OK;
    int bits = 0;
    while ((int64_t)1 << bits < vocab) ++bits;
    const SampleArgs g = {logits, ld, (int)vocab, temperature, top_k, top_p, min_p, uniform, tokens, logprob, 62 - bits > 50 ? 50 : 62 - bits, 1, 0, 0};
    if (dtype == MPQ_F32) return launch_sample<float>(g, rows, (cudaStream_t)stream);
    if (dtype == MPQ_F16) return launch_sample<__half>(g, rows, (cudaStream_t)stream);
    return launch_sample<__nv_bfloat16>(g, rows, (cudaStream_t)stream);
}
