// Low-rank adapters of a product of level bytes: what its two kernels share.
#pragma once
#include <type_traits>

#include "mpq_levels.cuh"

namespace mpq {

// What the first kernel leaves for the second, per token: its adapter (-1: none), z in 32 bits for the forms that multiply with
// it one by one, and z 2^-e in parts of the adapters' type for the matrix instructions, with 2^e beside them.  bfloat16: three
// parts, e = 0, together z whole.  float16, whose range is shorter than z's: two parts and an e that brings the row's
// largest near 2^15, together z to 2^-22 of itself or 2^-39 of the row's largest.
constexpr int kLowParts = 3;
struct LowWorkspace {
    float* z;                                             // [m][rank]
    uint16_t* parts;                                      // [kLowParts][m][rank]
    float* scale;                                         // [m]
    int32_t* chosen;                                      // [m]
    static int64_t bytes(int64_t m, int rank) { return (m * ((int64_t)rank * (4 + 2 * kLowParts) + 8) + 15) / 16 * 16; }
    LowWorkspace() = default;
    LowWorkspace(void* p, int64_t m, int rank) {          // rank is a multiple of 16, so every part starts at 16 bytes
        z = static_cast<float*>(p);
        parts = reinterpret_cast<uint16_t*>(z + m * rank);
        scale = reinterpret_cast<float*>(parts + kLowParts * m * rank);
        chosen = reinterpret_cast<int32_t*>(scale + m);
    }
};

struct AdapterArgs {
    const uint8_t* a; const float* a_scale; int La;       // the product's activations
    int64_t m, row_bytes;
    const void* down; const float* factor;                // [adapters][rank][row_bytes] elements; [adapters] or null
    int adapters, rank;                                   // rank: a multiple of 16
    const int32_t *starts, *ids; int batch;
    LowWorkspace low;
};
int adapter_down(const AdapterArgs& g, int dtype, cudaStream_t st);

// d += a b^T on 16 x 8 x 16 of W, in 32 bits.
template <typename W>
__device__ __forceinline__ void mma_16x8x16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same_v<W, __half>)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The two halves of a chain's launch (chain_entry): let the next kernel's blocks come, and wait for the kernel before.  That one may
// be writing while this one already runs, so what it makes is read by ordinary loads, which the wait orders: the read-only path
// (__ldg) is for memory that nobody writes as long as the kernel runs -- `up`, which the product multiplies z with: the kernel before
// lets the product in only when all earlier ones have ended.
__device__ __forceinline__ void chain_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void chain_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// An ordinary load that keeps its place behind the wait, but not behind stores: several can be on their way.
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

}  // namespace mpq
