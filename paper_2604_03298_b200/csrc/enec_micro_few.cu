// y = x W^T for few tokens, W a microscaled stream: one launch that reads every weight once (see enec_micro_pieces.cuh).
//
// A CTA takes row tiles of W, one after another. Where there are fewer of them than SMs, or where the digits of whole rows of x would not
// fit into shared memory, a cluster of CTAs shares the columns: each sends its sums to the CTA that adds up the token's, in the
// order of the CTAs. No sum depends on which CTA was faster.
#include "enec_micro_pieces.cuh"

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
    uint32_t share;       // records of columns that a CTA of the cluster takes
    uint32_t cluster;
    uint32_t stages;
    int* status;
};

struct FewTasks {
    PieceTask task;
    uint64_t step;       // bytes from a row tile to the CTA's next one
    __device__ __forceinline__ PieceTask get() const { return task; }
    __device__ __forceinline__ void next() { task.records += step; }
};

template <int DT>
__global__ void __launch_bounds__(kPieceThreads, 1) enec_micro_few_kernel(const __grid_constant__ FewJob job) {
    extern __shared__ uint8_t raw[];
    __shared__ PieceShared sh;
    using T = typename MicroType<DT>::T;
    uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = job.cluster > 1 ? blockIdx.x % job.cluster : 0;
    const uint32_t first_tile = blockIdx.x / job.cluster, step = gridDim.x / job.cluster;
    const uint32_t n_tasks = (job.s.row_tiles - first_tile + step - 1) / step;
    const uint32_t first = min(rank * job.share, job.s.col_tiles), count = min(job.share, job.s.col_tiles - first);
    const uint64_t tile_bytes = uint64_t(job.s.col_tiles) * kMicroRecordBytes;
    // two sets of [CTA][token][row]
    float* sums = reinterpret_cast<float*>(smem + job.stages * kMicroRecordBytes + job.share * piece_record_bytes(job.tokens));
    // other CTAs' shared memory may be written once they have begun
    if (job.cluster > 1) cooperative_groups::this_cluster().barrier_arrive();
    piece_setup(sh, job.stages);
    pdl_wait();
    pdl_launch_dependents();
    const MicroProbe header(job.w);
    const uint32_t owned = (job.tokens + job.cluster - 1) / job.cluster;   // tokens that a CTA of the cluster adds up, at most
    const uint32_t worker = warp - 2, row_in = (warp & 3) * 32 + lane;
    if (job.cluster > 1) cooperative_groups::this_cluster().barrier_wait();
    piece_products(
        sh, smem, job.stages, n_tasks, job.s.cols,
        FewTasks{PieceTask{job.w + kMicroHeaderBytes + first_tile * tile_bytes, first, count, 0, job.tokens}, step * tile_bytes},
        [&](uint32_t token, uint32_t col, float* x) {
            uint32_t w[4];
            load_eight<DT>(job.x + (uint64_t(token) * job.ld_x + col) * 2, col < job.s.cols ? int(min(job.s.cols - col, 8u)) : 0, w);
            as_floats<DT>(w, x);
        },
        [&](uint32_t i, uint32_t tmem, bool ok) {
            const uint32_t row = (first_tile + i * step) * kMicroRows + row_in;
            for (uint32_t token = worker >> 2; token < job.tokens; token += kPieceWorkers / 4) {
                const float v = count ? take_sum(tmem, token) : 0.f;
                if (job.cluster > 1) {   // to the CTA that adds up this token
                    float* to = cooperative_groups::this_cluster().map_shared_rank(sums, token % job.cluster);
                    to[(((i & 1) * job.cluster + rank) * owned + token / job.cluster) * kMicroRows + row_in] = v;
                } else if (header.fits(job.s) && ok && row < job.s.rows) {
                    reinterpret_cast<T*>(job.y)[uint64_t(token) * job.ld_y + row] = MicroType<DT>::one(v);
                }
            }
        },
        [](uint32_t, bool) {}, job.cluster > 1,
        [&](uint32_t i) {
            // a set of sums is written again behind the next one of these, and has been read by then; nothing comes from other CTAs behind
            // the last one
            cooperative_groups::this_cluster().sync();
            const uint32_t r = threadIdx.x & 127, row = (first_tile + i * step) * kMicroRows + r;
            if (threadIdx.x >= 512 || row >= job.s.rows || !header.fits(job.s) || sh.failed) return;
            for (uint32_t t = threadIdx.x >> 7; t * job.cluster + rank < job.tokens; t += 4) {
                const float* from = sums + ((i & 1) * job.cluster * owned + t) * kMicroRows + r;
                float v = 0.f;
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k)
                    if (k < job.cluster) v += from[k * owned * kMicroRows];
                reinterpret_cast<T*>(job.y)[uint64_t(t * job.cluster + rank) * job.ld_y + row] = MicroType<DT>::one(v);
            }
        });
    if (threadIdx.x == 0) {
        if (sh.failed) report(job.status, ENEC_ERR_TIMEOUT);
        else if (!header.fits(job.s) && blockIdx.x == 0) report(job.status, ENEC_ERR_BAD_STREAM);
    }
}

// Shared memory of a CTA that takes `share` records with four stages, or 0 where it does not fit.
uint32_t few_bytes(uint32_t share, uint32_t tokens, uint32_t cluster, uint32_t& stages) {
    const uint64_t others = 1024 + uint64_t(share) * piece_record_bytes(tokens) + (cluster > 1 ? (tokens + cluster - 1) / cluster * cluster * kMicroRows * 8 : 0);
    if (others + 4 * kMicroRecordBytes > kFewMostShared) return 0;
    const uint64_t fit = (kFewMostShared - others) / kMicroRecordBytes;
    stages = fit < kPieceMostStages ? uint32_t(fit) : kPieceMostStages;
    const uint32_t bytes = uint32_t(others + stages * kMicroRecordBytes);
    return bytes < kTmemAloneShared ? kTmemAloneShared : bytes;
}

template <int DT>
enec_status launch(FewJob job, const MicroDevice& dev, cudaStream_t stream) {
    // the smallest cluster whose CTAs have room; a larger one as long as all of them work at the same time
    uint32_t bytes = 0;
    job.cluster = 0;
    for (uint32_t cluster = 1; cluster <= 8; cluster *= 2) {
        const uint32_t share = (job.s.col_tiles + cluster - 1) / cluster;
        uint32_t stages = 0;
        const uint32_t need = few_bytes(share, job.tokens, cluster, stages);
        if (need == 0) continue;
        if (job.cluster && (uint64_t(job.s.row_tiles) * cluster > uint64_t(dev.sms) || cluster > job.s.col_tiles)) break;
        job.cluster = cluster, job.share = share, job.stages = stages, bytes = need;
    }
    if (job.cluster == 0) return ENEC_ERR_TOO_LARGE;
    static std::atomic<uint64_t> allowed{0};
    if (!allow_shared(allowed, dev, enec_micro_few_kernel<DT>, kFewMostShared)) return ENEC_ERR_CUDA;
    uint32_t places = uint32_t(dev.sms);
    if (job.cluster > 1 && !resident_clusters(enec_micro_few_kernel<DT>, dev, job.cluster, kPieceThreads, bytes, places)) return ENEC_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((job.s.row_tiles < places ? job.s.row_tiles : places) * job.cluster);
    cfg.blockDim = dim3(kPieceThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = job.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = job.cluster > 1 ? 2 : 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, enec_micro_few_kernel<DT>, job);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

}  // namespace

bool micro_few_takes(uint32_t tokens, uint32_t col_tiles) {
    uint32_t stages;
    return tokens <= kPieceTokens && few_bytes((col_tiles + 7) / 8, tokens, 8, stages) != 0;
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
    job.status = p.status;
    return p.dt == ENEC_BF16 ? launch<ENEC_BF16>(job, dev, stream) : launch<ENEC_FP16>(job, dev, stream);
}

}  // namespace enec
