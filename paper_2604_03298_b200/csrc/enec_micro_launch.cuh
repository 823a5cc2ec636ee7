// The product's forms, as its entry point chooses among them.
#pragma once

#include <mutex>

#include "enec_micro.cuh"

namespace enec {

// Clusters of `size` CTAs of a kernel that run at the same time, asked once per kernel, device and sizes; the last 32 answers are kept.
// (A part's groups of SMs are not multiples of a cluster: of 148 SMs clusters of 4 fill 132 and clusters of 8 fill 120.)
template <class Kernel>
bool resident_clusters(Kernel* kernel, const MicroDevice& dev, uint32_t size, uint32_t threads, uint32_t bytes, uint32_t& out) {
    struct Answer {
        Kernel* kernel;
        int ordinal;
        uint32_t size, bytes;
        int clusters;
    };
    static std::mutex mu;
    static Answer known[32] = {};
    static uint32_t next = 0;
    std::lock_guard<std::mutex> lock(mu);
    for (const Answer& a : known) {
        if (a.kernel != kernel || a.ordinal != dev.ordinal || a.size != size || a.bytes != bytes) continue;
        out = uint32_t(a.clusters);
        return true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(size);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = bytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) return false;
    known[next++ % 32] = Answer{kernel, dev.ordinal, size, bytes, n};
    out = uint32_t(n);
    return true;
}

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
// Products of no columns: zeros, if the streams' headers say what the call says. x: null or a stream too.
enec_status micro_no_columns(const uint8_t* x, const MicroShape& sx, const uint8_t* w, const MicroShape& sw, uint64_t tokens, void* y, uint64_t ld_y,
                             int* status, cudaStream_t stream);
// All tokens of the product, on the tensor cores.
enec_status micro_many(const MicroProduct& p, const MicroDevice& dev, cudaStream_t stream);

}  // namespace enec
