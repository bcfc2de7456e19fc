// Low-rank adapters of a product of level bytes: what its two kernels share.
#pragma once
#include <type_traits>

#include "mpq_levels.cuh"

namespace mpq {

struct AdapterArgs {
    const uint8_t* a; const float* a_scale; int La;       // the product's activations
    int64_t m, k, row_bytes;
    const void* down; const float* factor;                // [adapters][rank][row_bytes] elements; [adapters] or null
    int adapters, rank;                                   // rank: a multiple of 16
    const int32_t *starts, *ids; int batch;
    float* z; int32_t* chosen;                            // workspace: [m][rank]; the adapter of each token, -1 for none
};
int adapter_down(const AdapterArgs& g, int dtype, cudaStream_t st);

}  // namespace mpq
