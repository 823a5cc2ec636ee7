// y = x W^T for few tokens, W a microscaled stream: one launch that reads every weight once (see enec_micro_few.cuh).
//
// A CTA takes strips of 16 rows, one after another, and shares a strip's columns among its eight warps. The activations it
// needs stand in its shared memory, 2 bytes a value and token. Where they would not fit, a cluster of CTAs shares the columns and the
// first of them adds the others' sums, in their order. No sum depends on which CTA was faster.
#include "enec_micro_few.cuh"

#include <cooperative_groups.h>

#include "enec_micro_launch.cuh"

namespace enec {
namespace {

struct FewJob {
    const uint8_t* x;
    uint64_t ld_x;
    const uint8_t* w;
    MicroShape s;
    uint8_t* y;
    uint64_t ld_y;
    uint32_t tokens;
    uint32_t strips;      // that hold rows of the matrix
    uint32_t share;       // units of 128 columns that a CTA of the cluster takes
    uint32_t cluster;
    int* status;
};

__host__ __device__ constexpr uint32_t few_inverse_bytes(int nt) { return kFewWarps * 8 * nt * 4; }
__host__ __device__ constexpr uint32_t few_fixed_bytes(int nt) { return few_ring_bytes(1) + few_sum_bytes(nt, 1) + few_inverse_bytes(nt); }

template <int DT, int NT>
__global__ void __launch_bounds__(kFewThreads, 2) enec_micro_few_kernel(const __grid_constant__ FewJob job) {
    extern __shared__ __align__(128) uint8_t smem[];
    using T = typename MicroType<DT>::T;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const MicroShape& s = job.s;
    const uint32_t rank = job.cluster > 1 ? blockIdx.x % job.cluster : 0, team = blockIdx.x / job.cluster, teams = gridDim.x / job.cluster;
    float* sums = reinterpret_cast<float*>(smem + few_ring_bytes(1));
    float* inverse = reinterpret_cast<float*>(smem + few_ring_bytes(1) + few_sum_bytes(NT, 1)) + warp * 8 * NT;
    const uint32_t ring = smem_u32(smem) + warp * kFewStages * few_stage_bytes(1);
    const uint32_t staged = smem_u32(smem) + few_fixed_bytes(NT);

    const uint32_t all_units = (s.cols + kUnitCols - 1) / kUnitCols;
    const uint32_t unit0 = rank * job.share;
    const uint32_t units = unit0 < all_units ? min(job.share, all_units - unit0) : 0;

    pdl_wait();
    pdl_launch_dependents();
    // what this warp asks for next: unit ask_u of strip ask_strip
    uint32_t ask_strip = team, ask_u = warp, slot = 0;
    auto ask = [&]() {
        if (ask_strip < job.strips && ask_u < units) {
            ask_unit(job.w + kMicroHeaderBytes + uint64_t(ask_strip >> 3) * s.col_tiles * kMicroRecordBytes, ask_strip & 7, unit0 + ask_u,
                     ring + slot * few_stage_bytes(1), lane);
            ask_u += kFewWarps;
            if (ask_u >= units) ask_u = warp, ask_strip += teams;
        }
        cp_async_commit();
        slot = slot + 1 == kFewStages ? 0 : slot + 1;
    };
#pragma unroll
    for (uint32_t i = 0; i < kFewStages - 1; ++i) ask();
    const bool good = micro_header_ok(job.w, s);
    if (lane < 8 * NT) inverse[lane] = 0.f;
    __syncwarp();
    stage_share<DT>([&](uint32_t i) { return job.x + uint64_t(i) * job.ld_x * sizeof(T); }, job.tokens, units, unit0 * kUnitCols, s.cols, staged,
                    inverse, warp, lane);
    if (!good && blockIdx.x == 0 && threadIdx.x == 0) report(job.status, ENEC_ERR_BAD_STREAM);

    const uint32_t block_bytes = job.tokens * 64;
    const uint32_t columns = staged + g * 64 + t * 16;
    bool exists[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) exists[nt] = nt * 8 + g < job.tokens;
    uint32_t from = 0, set = 0;
    for (uint32_t strip = team; strip < job.strips; strip += teams) {
        float acc[NT][4] = {};
        for (uint32_t u = warp; u < units; u += kFewWarps) {
            cp_async_wait<kFewStages - 2>();
            __syncwarp();
            ask();   // into the slot that the unit before was read from, by all lanes
            add_unit<NT>(acc, ring + from * few_stage_bytes(1), columns + u * 4 * block_bytes, block_bytes, exists, lane);
            from = from + 1 == kFewStages ? 0 : from + 1;
        }
        float* mine = sums + set * (few_sum_bytes(NT, 1) / 8);
        put_sums<NT>(mine + warp * 16 * few_sum_row(NT), acc, inverse, lane);
        if (job.cluster > 1) cooperative_groups::this_cluster().sync();
        else __syncthreads();
        if (rank == 0) {
            for (uint32_t i = threadIdx.x; i < 16 * job.tokens; i += kFewThreads) {
                const uint32_t m = i & 15, token = i >> 4;
                const uint32_t row = (strip >> 3) * kMicroRows + strip_row(strip & 7, m);
                float v = 0.f;
                for (uint32_t r = 0; r < job.cluster; ++r) {
                    const float* theirs = r ? cooperative_groups::this_cluster().map_shared_rank(mine, r) : mine;
#pragma unroll
                    for (uint32_t k = 0; k < kFewWarps; ++k) v += theirs[(k * 16 + m) * few_sum_row(NT) + token];
                }
                if (row < s.rows && good) reinterpret_cast<T*>(job.y)[uint64_t(token) * job.ld_y + row] = MicroType<DT>::one(v);
            }
        }
        set ^= 1;   // the sums are written again only behind the next barrier but one's strip
    }
    cp_async_wait<0>();
    if (job.cluster > 1) cooperative_groups::this_cluster().sync();   // no CTA ends while its sums are read
}

template <int DT, int NT>
enec_status launch(FewJob job, const MicroDevice& dev, cudaStream_t stream) {
    const uint32_t all_units = (job.s.cols + kUnitCols - 1) / kUnitCols;
    const uint32_t per_unit = job.tokens * kUnitCols * 2;
    uint32_t cluster = 1;
    while (cluster < 8 && few_fixed_bytes(NT) + (all_units + cluster - 1) / cluster * per_unit > kFewMostShared) cluster *= 2;
    job.cluster = cluster;
    job.share = (all_units + cluster - 1) / cluster;
    const uint32_t bytes = few_fixed_bytes(NT) + job.share * per_unit;
    if (bytes > kFewMostShared) return ENEC_ERR_TOO_LARGE;
    static std::atomic<uint64_t> allowed{0};
    if (!allow_shared(allowed, dev, enec_micro_few_kernel<DT, NT>, kFewMostShared)) return ENEC_ERR_CUDA;
    const uint32_t resident = uint32_t(dev.sms) * (bytes <= kFewHalfShared ? 2 : 1) / cluster;
    const uint32_t teams = job.strips < resident ? job.strips : resident;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(teams * cluster);
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, enec_micro_few_kernel<DT, NT>, job);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

template <int DT>
enec_status launch_any(const FewJob& job, const MicroDevice& dev, cudaStream_t stream) {
    return job.tokens <= 8 ? launch<DT, 1>(job, dev, stream) : job.tokens <= 16 ? launch<DT, 2>(job, dev, stream) : launch<DT, 4>(job, dev, stream);
}

}  // namespace

uint32_t micro_few_most_tokens(uint32_t cols) {
    const uint32_t share = ((cols + kUnitCols - 1) / kUnitCols + 7) / 8;
    for (uint32_t tokens : {32u, 16u, 8u, 4u, 2u, 1u}) {
        const int nt = tokens > 16 ? 4 : tokens > 8 ? 2 : 1;
        if (few_fixed_bytes(nt) + uint64_t(share) * tokens * kUnitCols * 2 <= kFewMostShared) return tokens;
    }
    return 0;
}

enec_status micro_few(const MicroProduct& p, const MicroDevice& dev, cudaStream_t stream) {
    FewJob job;
    job.x = p.x;
    job.ld_x = p.ld_x;
    job.w = p.w;
    job.s = p.s;
    job.y = p.y;
    job.ld_y = p.ld_y;
    job.tokens = p.tokens;
    const uint32_t last = p.s.rows - (p.s.row_tiles - 1) * kMicroRows;   // rows of the last record
    job.strips = (p.s.row_tiles - 1) * 8 + (last >= 32 ? 8 : (last + 3) / 4);
    job.status = p.status;
    return p.dt == ENEC_BF16 ? launch_any<ENEC_BF16>(job, dev, stream) : launch_any<ENEC_FP16>(job, dev, stream);
}

}  // namespace enec
