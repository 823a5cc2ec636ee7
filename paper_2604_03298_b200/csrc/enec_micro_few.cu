// y = x W^T for few tokens, W a microscaled stream: one launch that reads every weight once (see enec_micro_few.cuh).
//
// A CTA's teams take strips of 16 rows, one after another. The activations stand in its shared memory, 2 bytes a value and token. Where
// they would not fit, a cluster of CTAs shares the columns and the first of them adds the others' sums, in their order. No sum
// depends on which team or CTA was faster.
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
    uint32_t team;        // warps
    int* status;
};

template <int DT, int NT>
__global__ void __launch_bounds__(kFewThreads, 1) enec_micro_few_kernel(const __grid_constant__ FewJob job) {
    extern __shared__ __align__(128) uint8_t smem[];
    using T = typename MicroType<DT>::T;
    constexpr uint32_t kStages = few_stages(1), kSums = few_sum_words(NT, 1);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const MicroShape& s = job.s;
    const uint32_t rank = job.cluster > 1 ? blockIdx.x % job.cluster : 0;
    const uint32_t all_units = (s.cols + kUnitCols - 1) / kUnitCols;
    const uint32_t unit0 = min(rank * job.share, all_units), units = min(job.share, all_units - unit0);
    const uint32_t per_cta = kFewWarps / job.team, team = warp / job.team, in_team = warp % job.team;
    const uint32_t first = blockIdx.x / job.cluster * per_cta + team, step = gridDim.x / job.cluster * per_cta;
    float* sums = reinterpret_cast<float*>(smem + few_ring_bytes(1)) + team * job.team * kSums;
    float* inverse = reinterpret_cast<float*>(smem + few_fixed_bytes(NT, 1));
    const uint32_t ring = smem_u32(smem) + warp * kStages * few_stage_bytes(1);
    const uint32_t staged = smem_u32(inverse + job.share * 8 * NT);

    pdl_wait();
    pdl_launch_dependents();
    // what this warp asks for next: unit ask_u of strip ask_strip
    uint32_t ask_strip = first, ask_u = in_team, slot = 0;
    auto ask = [&]() {
        if (ask_strip < job.strips && ask_u < units) {
            ask_unit(job.w + kMicroHeaderBytes + uint64_t(ask_strip >> 3) * s.col_tiles * kMicroRecordBytes, ask_strip & 7, unit0 + ask_u,
                     ring + slot * few_stage_bytes(1), lane);
            ask_u += job.team;
            if (ask_u >= units) ask_u = in_team, ask_strip += step;
        }
        cp_async_commit();
        slot = slot + 1 == kStages ? 0 : slot + 1;
    };
#pragma unroll
    for (uint32_t i = 0; i < kStages - 1; ++i) ask();
    const bool good = micro_header_ok(job.w, s);
    stage_columns<DT>([&](uint32_t i) { return job.x + uint64_t(i) * job.ld_x * sizeof(T); }, job.tokens, units, unit0 * kUnitCols, s.cols, staged,
                      inverse, 8 * NT);
    __syncthreads();
    if (!good && blockIdx.x == 0 && threadIdx.x == 0) report(job.status, ENEC_ERR_BAD_STREAM);

    const uint32_t values = staged + g * 64 + t * 16;
    bool exists[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) exists[nt] = nt * 8 + g < job.tokens;
    uint32_t from = 0;
    // clusters meet at every strip, so all their teams go round equally often
    for (uint32_t strip = first; job.cluster > 1 ? strip - team < job.strips : strip < job.strips; strip += step) {
        float acc[NT][4] = {};
        for (uint32_t u = in_team; strip < job.strips && u < units; u += job.team) {
            cp_async_wait<kStages - 2>();
            __syncwarp();
            ask();   // into the slot that the unit before was read from, by all lanes
            add_unit<NT>(acc, ring + from * few_stage_bytes(1), values + u * 4 * job.tokens * 64, inverse + u * 8 * NT + 2 * t, job.tokens, exists, lane);
            from = from + 1 == kStages ? 0 : from + 1;
        }
        put_sums<NT>(sums + in_team * kSums, acc, lane);
        if (job.cluster > 1) cooperative_groups::this_cluster().sync();
        else team_sync(team, job.team * 32);
        if (rank == 0 && strip < job.strips) {
            for (uint32_t i = in_team * 32 + lane; i < 16 * job.tokens; i += job.team * 32) {
                const uint32_t m = i & 15, token = i >> 4;
                const uint32_t row = (strip >> 3) * kMicroRows + strip_row(strip & 7, m);
                float v = 0.f;
                for (uint32_t r = 0; r < job.cluster; ++r) {
                    const float* theirs = r ? cooperative_groups::this_cluster().map_shared_rank(sums, r) : sums;
                    for (uint32_t k = 0; k < job.team; ++k) v += theirs[k * kSums + m * few_sum_row(NT) + token];
                }
                if (row < s.rows && good) reinterpret_cast<T*>(job.y)[uint64_t(token) * job.ld_y + row] = MicroType<DT>::one(v);
            }
        }
        // the sums have been read before they are written again, and before a CTA ends
        if (job.cluster > 1) cooperative_groups::this_cluster().sync();
        else team_sync(team, job.team * 32);
    }
    cp_async_wait<0>();
}

template <int DT, int NT>
enec_status launch(FewJob job, const MicroDevice& dev, cudaStream_t stream) {
    const uint32_t all_units = (job.s.cols + kUnitCols - 1) / kUnitCols;
    const uint32_t per_unit = few_unit_bytes(NT, job.tokens), fixed = few_fixed_bytes(NT, 1);
    uint32_t cluster = 1;
    while (cluster < 8 && fixed + uint64_t(all_units + cluster - 1) / cluster * per_unit > kFewMostShared) cluster *= 2;
    job.cluster = cluster;
    job.share = (all_units + cluster - 1) / cluster;
    const uint32_t bytes = fixed + job.share * per_unit;
    if (bytes > kFewMostShared) return ENEC_ERR_TOO_LARGE;
    static std::atomic<uint64_t> allowed{0};
    if (!allow_shared(allowed, dev, enec_micro_few_kernel<DT, NT>, kFewMostShared)) return ENEC_ERR_CUDA;
    const uint32_t places = uint32_t(dev.sms) / cluster;
    job.team = few_team(job.strips, job.share, places);
    const uint32_t per_cta = kFewWarps / job.team, needed = (job.strips + per_cta - 1) / per_cta;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((needed < places ? needed : places) * cluster);
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
        if (few_fixed_bytes(nt, 1) + uint64_t(share) * few_unit_bytes(nt, tokens) <= kFewMostShared) return tokens;
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
