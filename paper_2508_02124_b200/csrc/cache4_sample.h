// Where the selection's sample lies in a row (cache4_select.cu). Plain C++: a host can compile it too.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define DMA_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define DMA_HOST_DEVICE inline
#endif

namespace dma {

// The i-th of `groups` places in a row of `quads` quads: the row is cut into as many strata, each of which has one, at a distance from its first that a multiplicative hash of i
// (2^32 by the golden ratio) gives. The product of hash and stratum takes 64 bits: rows have up to 2^28 quads.
DMA_HOST_DEVICE uint32_t sample_quad(uint32_t i, uint32_t quads, uint32_t groups) {
    const uint32_t step = quads / groups;
    return (uint32_t)((uint64_t)i * quads / groups) + (uint32_t)((uint64_t)(i * 2654435761u) * step >> 32);
}

}  // namespace dma
