// y = X W^T with both operands as microscaled streams: tcgen05.mma with block scales (kind::mxf4), four times the rate of bf16.
//
// Lanes of the accumulator are rows of W, its columns tokens: 128 x up to 192, twice, so that a tile's results leave while the next one's
// products run. A CTA takes tile after tile. A stage is one record's 256 columns: a record lies in memory as the tensor cores want it in
// shared memory, so a stage is a handful of bulk copies without a tensor map, and its scales go on to tensor memory as they are
// (tcgen05.cp). At this rate a tile is bound by shared memory: a stage's 44 KB are written once, and its 4 matrix instructions read 10 KB
// each, 85 KB in all or 664 clocks at 128 bytes a clock, for 392 clocks of instructions (98 each, measured); the kernel takes 870.
// 256 x 192 would need 548 for the same work, but only three such stages fit, and no second set of sums: 2048 x 14336 x 4096 took
// 85 us (1300 clocks a stage, and 9000 a tile for storing behind the products) where this form took 68 (it takes that with
// the streams in L2, 74 us cold). Pairs of CTAs that share the tokens' operand would read 57 KB.
#include "enec_micro_mma.cuh"

#include "enec_micro_launch.cuh"

namespace enec {
namespace {

constexpr uint32_t kBothMostStages = 5;
constexpr uint32_t kBothThreads = 320;       // copies, matrix instructions, eight warps that store
constexpr uint32_t kBothMostTokens = 192;    // of a tile
constexpr uint32_t kScaleColumns = 24;       // of a stage in tensor memory: 8 for the rows of W, 16 for the tokens

struct BothJob {
    const uint8_t* x;
    const uint8_t* w;
    MicroShape sx, sw;
    uint8_t* y;
    uint64_t ld_y;
    uint32_t tile_tokens;
    uint32_t tiles;
    uint32_t stages;
    int* status;
};

__host__ __device__ constexpr uint32_t both_stage_bytes(uint32_t tokens) { return kMicroElemBytes + tokens * 128 + 3 * 1024; }

// A tile's place: rows 128 row_tile .., tokens first .., which are the rows skip .. of one record, and where there is one, of the next.
struct BothTile {
    uint32_t row_tile, token0, x_tile, skip, first_rows;
    bool second;
    __device__ __forceinline__ BothTile(const BothJob& job, uint32_t t) {
        row_tile = t % job.sw.row_tiles;
        token0 = t / job.sw.row_tiles * job.tile_tokens;
        x_tile = token0 / kMicroRows, skip = token0 % kMicroRows;
        first_rows = min(job.tile_tokens, kMicroRows - skip);
        second = first_rows < job.tile_tokens && x_tile + 1 < job.sx.row_tiles;
    }
};

template <int DT>
__global__ void __launch_bounds__(kBothThreads, 1) enec_micro_both_kernel(const __grid_constant__ BothJob job) {
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[kBothMostStages], empty[kBothMostStages], done[2], drained[2];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int failed;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    const uint32_t n = job.tile_tokens, stage_bytes = both_stage_bytes(n);
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < job.stages; ++i) mbar_init(full + i, 1), mbar_init(empty + i, 1);
        for (uint32_t i = 0; i < 2; ++i) mbar_init(done + i, 1), mbar_init(drained + i, kBothThreads / 32 - 2);
        mbar_fence_init();
        failed = 0;
    }
    if (warp == 1) tmem_alloc(&tmem_at, 512);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_at;
    pdl_wait();
    pdl_launch_dependents();

    const uint32_t records = job.sw.col_tiles;
    const uint64_t strip = uint64_t(records) * kMicroRecordBytes;
    const uint32_t leader = elected();
    if (warp == 0) {
        uint32_t asked = 0, s = 0, phase = 1;
        for (uint32_t t = blockIdx.x; t < job.tiles; t += gridDim.x) {
            const BothTile tile(job, t);
            const uint32_t bytes = kMicroRecordBytes + tile.first_rows * 128 + 1024 + (tile.second ? (n - tile.first_rows) * 128 + 1024 : 0);
            const uint8_t* wr = job.w + kMicroHeaderBytes + tile.row_tile * strip;
            const uint8_t* xr = job.x + kMicroHeaderBytes + tile.x_tile * strip;
            for (uint32_t k = 0; k < records; ++k, wr += kMicroRecordBytes, xr += kMicroRecordBytes) {
                if (asked >= job.stages && !warp_wait(empty + s, phase, &failed)) {
                    failed = 1;
                    break;
                }
                if (leader) {
                    uint8_t* a = smem + s * stage_bytes;
                    uint8_t* b = a + kMicroElemBytes;
                    uint8_t* scales = b + n * 128;
                    mbar_expect_tx(full + s, bytes);
                    bulk_g2s(a, wr, kMicroElemBytes, full + s);
                    bulk_g2s(b, xr + tile.skip * 128, tile.first_rows * 128, full + s);
                    if (tile.second) bulk_g2s(b + tile.first_rows * 128, xr + strip, (n - tile.first_rows) * 128, full + s);
                    bulk_g2s(scales, wr + kMicroElemBytes, 1024, full + s);
                    bulk_g2s(scales + 1024, xr + kMicroElemBytes, 1024, full + s);
                    if (tile.second) bulk_g2s(scales + 2048, xr + strip + kMicroElemBytes, 1024, full + s);
                }
                ++asked;
                if (++s == job.stages) s = 0, phase ^= 1;
            }
        }
        // nothing may be in flight when the CTA ends
        for (uint32_t i = asked > job.stages ? asked - job.stages : 0; i < asked; ++i) mbar_wait_bounded(full + i % job.stages, (i / job.stages) & 1);
    } else if (warp == 1) {
        const uint32_t idesc = scaled_idesc(n);
        const uint64_t operands = operand_desc(smem_u32(smem)), scales = scale_desc(smem_u32(smem) + kMicroElemBytes + n * 128);
        uint32_t s = 0, phase = 0, i = 0, there = mbar_complete(full, 0);
        for (uint32_t t = blockIdx.x; t < job.tiles; t += gridDim.x, ++i) {
            const BothTile tile(job, t);
            const uint32_t set = i & 1, sums = tmem + set * kBothMostTokens;
            if (i >= 2 && !suspended_wait(drained + set, ((i >> 1) - 1) & 1, &failed)) failed = 1;
            for (uint32_t k = 0; k < records && !failed; ++k) {
                if (!there && !suspended_wait(full + s, phase, &failed)) {
                    failed = 1;
                    break;
                }
                const uint32_t now = s;
                if (++s == job.stages) s = 0, phase ^= 1;
                there = mbar_complete(full + s, phase);
                tcgen05_fence_after();
                const uint64_t a = operands + now * (stage_bytes / 16), b = a + kMicroElemBytes / 16, sc = scales + now * (stage_bytes / 16);
                // tensor memory of a stage's scales: of the columns' four chunks h, 4 columns for the rows of W, and 8 for the tokens
                const uint32_t to = tmem + 2 * kBothMostTokens + now * kScaleColumns;
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) {
                    copy_scales(leader, to + h * 4, sc + h * 32);
                    copy_scales(leader, to + 8 + h * 8, sc + 64 + h * 32);
                    copy_scales(tile.second ? leader : 0, to + 8 + h * 8 + 4, sc + 128 + h * 32);
                }
                const uint32_t steps = (job.sw.cols - k * kMicroCols + 63) / 64;
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) {
                    const uint32_t h = q >> 1, pair = (q & 1) * 2;
                    mma_scaled(q < steps ? leader : 0, sums, a + q * 2, b + q * 2, idesc | pair << 4 | pair << 29, to + h * 4,
                               to + 8 + h * 8 + tile.skip / 32, k > 0 || q > 0);
                }
                tcgen05_commit(leader, empty + now);
            }
            tcgen05_commit(leader, done + set);
        }
        // no instruction may be under way when tensor memory is given back
        for (uint32_t k = i > 2 ? i - 2 : 0; k < i; ++k) mbar_wait_bounded(done + (k & 1), (k >> 1) & 1);
        __syncwarp();
    } else {
        const MicroProbe w_header(job.w), x_header(job.x);
        const bool good = w_header.fits(job.sw) && x_header.fits(job.sx);
        const uint32_t quarter = warp & 3, half = (warp - 2) >> 2;   // the lanes of tensor memory that this warp may read; which 16 tokens in 32
        uint32_t i = 0;
        for (uint32_t t = blockIdx.x; t < job.tiles; t += gridDim.x, ++i) {
            const BothTile tile(job, t);
            const uint32_t set = i & 1, row = tile.row_tile * kMicroRows + quarter * 32 + lane;
            wait_or_fail(done + set, (i >> 1) & 1, &failed);
            tcgen05_fence_after();
            if (good && !warp_failed(&failed)) {
                for (uint32_t c = half * 16; c < n; c += 32) {
                    if (tile.token0 + c >= job.sx.rows) break;
                    uint32_t v[16];
                    tmem_load16(tmem + (quarter * 32 << 16) + set * kBothMostTokens + c, v);
                    tmem_load_wait();
                    store_tile16<DT>(job.y, job.ld_y, tile.token0 + c, job.sx.rows, row, job.sw.rows, v, 1.f, lane);
                }
            }
            tcgen05_fence_before();
            warp_arrive(drained + set);
        }
        if (!good && blockIdx.x == 0 && warp == 2 && lane == 0) report(job.status, ENEC_ERR_BAD_STREAM);
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    if (failed && threadIdx.x == 0) report(job.status, ENEC_ERR_TIMEOUT);
    if (warp == 1) tmem_free(tmem, 512);
}

template <int DT>
enec_status launch_both(BothJob job, const MicroDevice& dev, cudaStream_t stream) {
    static std::atomic<uint64_t> allowed{0};
    if (!allow_shared(allowed, dev, enec_micro_both_kernel<DT>, kFewMostShared)) return ENEC_ERR_CUDA;
    const uint32_t fit = (kFewMostShared - 1024) / both_stage_bytes(job.tile_tokens);
    job.stages = fit < kBothMostStages ? fit : kBothMostStages;
    uint32_t bytes = job.stages * both_stage_bytes(job.tile_tokens) + 1024;
    if (bytes < kTmemAloneShared) bytes = kTmemAloneShared;
    const uint32_t grid = job.tiles < uint32_t(dev.sms) ? job.tiles : uint32_t(dev.sms);
    const cudaError_t err = launch_pdl(enec_micro_both_kernel<DT>, grid, kBothThreads, bytes, stream, job);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

}  // namespace
}  // namespace enec

using namespace enec;

extern "C" enec_status enec_matmul_microscaled_both(const void* d_x, size_t x_size, size_t tokens, const void* d_w, size_t w_size, size_t rows,
                                                    size_t cols, enec_dtype dt, void* d_y, size_t ld_y, int* d_status, enec_stream_t stream) {
    if (dt != ENEC_BF16 && dt != ENEC_FP16) return ENEC_ERR_UNSUPPORTED_DTYPE;
    BothJob job;
    if (!make_micro_shape(1, tokens, cols, job.sx) || !make_micro_shape(1, rows, cols, job.sw)) return ENEC_ERR_TOO_LARGE;
    if (tokens == 0 || rows == 0) return ENEC_OK;
    if (!d_x || !d_w || !d_y || !micro_aligned16(d_x) || !micro_aligned16(d_w) || !micro_aligned16(d_y) || ld_y < rows || (uint64_t(ld_y) >> 36))
        return ENEC_ERR_INVALID_ARG;
    if (x_size < job.sx.total || w_size < job.sw.total) return ENEC_ERR_BUFFER_TOO_SMALL;
    if (cols == 0)
        return micro_no_columns(static_cast<const uint8_t*>(d_x), job.sx, static_cast<const uint8_t*>(d_w), job.sw, tokens, d_y, ld_y, d_status, stream);
    MicroDevice dev;
    if (!micro_device(dev)) return ENEC_ERR_CUDA;
    job.x = static_cast<const uint8_t*>(d_x);
    job.w = static_cast<const uint8_t*>(d_w);
    job.y = static_cast<uint8_t*>(d_y);
    job.ld_y = ld_y;
    job.status = d_status;
    // the tile whose rounds over the SMs cost least: a stage's time is that of its matrix instructions or of shared memory's bytes, whichever is
    // longer, and a CTA has some 5000 clocks of filling the ring and of storing its last tile. Tokens in steps of 64:
    // a tile then begins at row 0 or 64 of a record, and its scales at an even column of tensor memory.
    uint64_t least = ~uint64_t(0), tiles = 0;
    for (uint32_t k = kBothMostTokens; k >= 64; k -= 64) {
        const uint64_t all = uint64_t(job.sw.row_tiles) * ((tokens + k - 1) / k), rounds = (all + dev.sms - 1) / dev.sms;
        const uint32_t instructions = 4 * (k > 128 ? k / 2 + 2 : 65), bytes = 4 * (4096 + k * 32) + both_stage_bytes(k);
        const uint64_t cost = rounds * job.sw.col_tiles * (instructions > bytes / 128 ? instructions : bytes / 128) + 5000;
        if (cost < least) least = cost, job.tile_tokens = k, tiles = all;
    }
    if (tiles >> 31) return ENEC_ERR_TOO_LARGE;
    job.tiles = uint32_t(tiles);
    return dt == ENEC_BF16 ? launch_both<ENEC_BF16>(job, dev, stream) : launch_both<ENEC_FP16>(job, dev, stream);
}
