// The product's forms, as its entry point chooses among them.
#pragma once

#include "enec_micro.cuh"

namespace enec {

struct MicroProduct {
    int dt;
    const uint8_t* x;
    uint64_t ld_x;
    uint32_t tokens;
    const uint8_t* w;
    MicroShape s;      // of w
    uint8_t* y;
    uint64_t ld_y;
    int* status;
};

constexpr uint32_t kFewMostShared = 226 * 1024;   // the kernels have a little static shared memory beside it

// Whether the form for few tokens takes a call (up to 16 tokens, as long as their digits fit into a cluster's shared memory).
bool micro_few_takes(uint32_t tokens, uint32_t col_tiles);
enec_status micro_few(const MicroProduct& p, const MicroDevice& dev, cudaStream_t stream);
// All tokens of the product, on the tensor cores.
enec_status micro_many(const MicroProduct& p, const MicroDevice& dev, cudaStream_t stream);

}  // namespace enec
