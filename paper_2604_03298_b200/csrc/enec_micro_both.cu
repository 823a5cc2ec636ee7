// y = X W^T with both operands as microscaled streams: tcgen05.mma with block scales (kind::mxf4), four times the rate of bf16.
//
// Lanes of the accumulator are rows of W, its columns tokens. A stage is one record's 256 columns: a record lies in memory as the
// tensor cores want it in shared memory, so a stage is a handful of bulk copies without a tensor map, and its scales go on to
// tensor memory as they are (tcgen05.cp). At this rate what bounds a tile is how fast L2 refills shared memory: 256 rows x 192
// tokens take 60 KB a stage for 786 clocks of matrix instructions (98 each, measured), 76 bytes a clock, of which L2 gave 84 at
// most; 128 x 128 would take 134. So the tile is the largest whose accumulators (2 x 192 columns) leave room for three stages'
// scales in the 512 columns of tensor memory, or the smaller one with which the SMs' last round is fuller.
#include "enec_micro_mma.cuh"

#include "enec_micro_launch.cuh"

namespace enec {
namespace {

constexpr uint32_t kBothMostStages = 8;
constexpr uint32_t kBothThreads = 320;       // copies, matrix instructions, eight warps that store
constexpr uint32_t kBothMostTokens = 192;    // of a tile
constexpr uint32_t kScaleColumns = 32;       // of a stage in tensor memory: 8 for each 128 rows of W, 16 for the tokens

struct BothJob {
    const uint8_t* x;
    const uint8_t* w;
    MicroShape sx, sw;
    uint8_t* y;
    uint64_t ld_y;
    uint32_t tile_tokens;
    uint32_t row_tiles;      // tiles along the rows of W
    uint32_t stages;
    int* status;
};

template <int MT>
__host__ __device__ constexpr uint32_t both_stage_bytes(uint32_t tokens) { return MT * kMicroElemBytes + tokens * 128 + (MT + 2) * 1024; }

template <int DT, int MT>
__global__ void __launch_bounds__(kBothThreads, 1) enec_micro_both_kernel(const __grid_constant__ BothJob job) {
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[kBothMostStages], empty[kBothMostStages], done;
    __shared__ uint32_t tmem_at;
    __shared__ volatile int failed;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    const uint32_t n = job.tile_tokens, stage_bytes = both_stage_bytes<MT>(n);
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < job.stages; ++i) mbar_init(full + i, 1), mbar_init(empty + i, 1);
        mbar_init(&done, 1);
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

    const uint32_t row_tile = blockIdx.x % job.row_tiles * MT;                    // in units of 128 rows
    const uint32_t token0 = blockIdx.x / job.row_tiles * n;
    const uint32_t mt = min(uint32_t(MT), job.sw.row_tiles - row_tile);            // of them that the matrix has
    const uint32_t records = job.sw.col_tiles;
    // the tokens' records: rows skip .. of the first, the rest of the second where there is one
    const uint32_t x_tile = token0 / kMicroRows, skip = token0 % kMicroRows, first_rows = min(n, kMicroRows - skip);
    const bool second = first_rows < n && x_tile + 1 < job.sx.row_tiles;
    const uint8_t* wr = job.w + kMicroHeaderBytes + uint64_t(row_tile) * records * kMicroRecordBytes;
    const uint8_t* xr = job.x + kMicroHeaderBytes + uint64_t(x_tile) * records * kMicroRecordBytes;
    const uint64_t strip = uint64_t(records) * kMicroRecordBytes;

    const uint32_t leader = elected();
    if (warp == 0) {
        const uint32_t bytes = mt * kMicroRecordBytes + first_rows * 128 + 1024 + (second ? (n - first_rows) * 128 + 1024 : 0);
        uint32_t k = 0, s = 0, phase = 1;
        for (; k < records; ++k) {
            if (k >= job.stages && !suspended_wait(empty + s, phase, &failed)) {
                failed = 1;
                break;
            }
            uint8_t* a = smem + s * stage_bytes;
            uint8_t* b = a + MT * kMicroElemBytes;
            uint8_t* scales = b + n * 128;
            const uint64_t at = uint64_t(k) * kMicroRecordBytes;
            if (leader) {
                mbar_expect_tx(full + s, bytes);
                for (uint32_t i = 0; i < mt; ++i) {
                    bulk_g2s(a + i * kMicroElemBytes, wr + i * strip + at, kMicroElemBytes, full + s);
                    bulk_g2s(scales + i * 1024, wr + i * strip + at + kMicroElemBytes, 1024, full + s);
                }
                bulk_g2s(b, xr + at + skip * 128, first_rows * 128, full + s);
                bulk_g2s(scales + MT * 1024, xr + at + kMicroElemBytes, 1024, full + s);
                if (second) {
                    bulk_g2s(b + first_rows * 128, xr + strip + at, (n - first_rows) * 128, full + s);
                    bulk_g2s(scales + MT * 1024 + 1024, xr + strip + at + kMicroElemBytes, 1024, full + s);
                }
            }
            if (++s == job.stages) s = 0, phase ^= 1;
        }
        // nothing may be in flight when the CTA ends
        for (uint32_t i = k > job.stages ? k - job.stages : 0; i < k; ++i) mbar_wait_bounded(full + i % job.stages, (i / job.stages) & 1);
    } else if (warp == 1) {
        const uint32_t idesc = scaled_idesc(n);
        const uint64_t operands = operand_desc(smem_u32(smem)), scales = scale_desc(smem_u32(smem) + MT * kMicroElemBytes + n * 128);
        uint32_t s = 0, phase = 0;
        for (uint32_t k = 0; k < records; ++k) {
            if (!suspended_wait(full + s, phase, &failed)) {
                failed = 1;
                break;
            }
            tcgen05_fence_after();
            const uint64_t a = operands + s * (stage_bytes / 16), b = a + MT * (kMicroElemBytes / 16), sc = scales + s * (stage_bytes / 16);
            // tensor memory of a stage's scales: of the columns' four chunks h, 4 columns per 128 rows of W, and 8 for the tokens
            const uint32_t to = tmem + MT * kBothMostTokens + s * kScaleColumns;
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
#pragma unroll
                for (uint32_t i = 0; i < MT; ++i) copy_scales(i < mt ? leader : 0, to + (2 * i + h) * 4, sc + i * 64 + h * 32);
                copy_scales(leader, to + MT * 8 + h * 8, sc + MT * 64 + h * 32);
                copy_scales(second ? leader : 0, to + MT * 8 + h * 8 + 4, sc + (MT + 1) * 64 + h * 32);
            }
            const uint32_t steps = (job.sw.cols - k * kMicroCols + 63) / 64;
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                const uint32_t h = q >> 1, pair = (q & 1) * 2;
                const uint32_t scale_x = to + MT * 8 + h * 8 + skip / 32;
#pragma unroll
                for (uint32_t i = 0; i < MT; ++i)
                    mma_scaled(q < steps && i < mt ? leader : 0, tmem + i * kBothMostTokens, a + i * (kMicroElemBytes / 16) + q * 2, b + q * 2,
                               idesc | pair << 4 | pair << 29, to + (2 * i + h) * 4, scale_x, k > 0 || q > 0);
            }
            tcgen05_commit(leader, empty + s);
            if (++s == job.stages) s = 0, phase ^= 1;
        }
        tcgen05_commit(leader, &done);
        mbar_wait_bounded(&done, 0);   // no instruction may be under way when tensor memory is given back
    } else {
        const bool good = micro_header_ok(job.w, job.sw) && micro_header_ok(job.x, job.sx);
        if (!suspended_wait(&done, 0, &failed)) failed = 1;
        tcgen05_fence_after();
        const uint32_t quarter = warp & 3, half = (warp - 2) >> 2;   // the lanes of tensor memory that this warp may read; which 16 tokens in 32
        if (good && !failed) {
            for (uint32_t i = 0; i < mt; ++i) {
                const uint32_t row = (row_tile + i) * kMicroRows + quarter * 32 + lane;
                for (uint32_t c = half * 16; c < n; c += 32) {
                    if (token0 + c >= job.sx.rows) break;
                    uint32_t v[16];
                    tmem_load16(tmem + (quarter * 32 << 16) + i * kBothMostTokens + c, v);
                    tmem_load_wait();
                    store_tile16<DT>(job.y, job.ld_y, token0 + c, job.sx.rows, row, job.sw.rows, v, 1.f, lane);
                }
            }
        }
        if (!good && blockIdx.x == 0 && warp == 2 && lane == 0) report(job.status, ENEC_ERR_BAD_STREAM);
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    if (failed && threadIdx.x == 0) report(job.status, ENEC_ERR_TIMEOUT);
    if (warp == 1) tmem_free(tmem, 512);
}

template <int DT, int MT>
enec_status launch_both(BothJob job, uint32_t grid, const MicroDevice& dev, cudaStream_t stream) {
    static std::atomic<uint64_t> allowed{0};
    if (!allow_shared(allowed, dev, enec_micro_both_kernel<DT, MT>, kFewMostShared)) return ENEC_ERR_CUDA;
    // as many stages as fit into shared memory, and their scales beside the sums in tensor memory: three of the largest tile
    const uint32_t fit = (kFewMostShared - 1024) / both_stage_bytes<MT>(job.tile_tokens), columns = (512 - MT * kBothMostTokens) / kScaleColumns;
    job.stages = fit < columns ? fit : columns;
    if (job.stages > kBothMostStages) job.stages = kBothMostStages;
    uint32_t bytes = job.stages * both_stage_bytes<MT>(job.tile_tokens) + 1024;
    if (bytes < kTmemAloneShared) bytes = kTmemAloneShared;
    const cudaError_t err = launch_pdl(enec_micro_both_kernel<DT, MT>, grid, kBothThreads, bytes, stream, job);
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
    if (cols == 0) return cudaMemset2DAsync(d_y, ld_y * 2, 0, rows * 2, tokens, stream) == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
    MicroDevice dev;
    if (!micro_device(dev)) return ENEC_ERR_CUDA;
    job.x = static_cast<const uint8_t*>(d_x);
    job.w = static_cast<const uint8_t*>(d_w);
    job.y = static_cast<uint8_t*>(d_y);
    job.ld_y = ld_y;
    job.status = d_status;
    // the tile whose rounds over the SMs cost least: a tile's time is that of its matrix instructions or of refilling shared memory at 84
    // bytes a clock, whichever is longer, over its records, and some 3000 clocks for filling the ring and storing. Tokens in steps of 64:
    // a tile then begins at row 0 or 64 of a record, and its scales at an even column of tensor memory
    uint32_t mt = 2, n = kBothMostTokens;
    uint64_t least = ~uint64_t(0);
    for (uint32_t m = 2; m >= 1; --m) {
        for (uint32_t k = kBothMostTokens; k >= 64; k -= 64) {
            const uint64_t all = uint64_t((job.sw.row_tiles + m - 1) / m) * ((tokens + k - 1) / k);
            const uint32_t instructions = 4 * m * (k > 128 ? k / 2 + 2 : 65), refill = (m * kMicroRecordBytes + k * 128 + 2048) / 84;
            const uint64_t cost = (all + dev.sms - 1) / dev.sms * (uint64_t(job.sw.col_tiles) * (instructions > refill ? instructions : refill) + 3000);
            if (cost < least) least = cost, mt = m, n = k;
        }
    }
    auto tiles = [&]() { return uint64_t((job.sw.row_tiles + mt - 1) / mt) * ((tokens + n - 1) / n); };
    job.tile_tokens = n;
    job.row_tiles = (job.sw.row_tiles + mt - 1) / mt;
    if (tiles() >> 31) return ENEC_ERR_TOO_LARGE;
    const uint32_t grid = uint32_t(tiles());
    if (dt == ENEC_BF16) return mt == 2 ? launch_both<ENEC_BF16, 2>(job, grid, dev, stream) : launch_both<ENEC_BF16, 1>(job, grid, dev, stream);
    return mt == 2 ? launch_both<ENEC_FP16, 2>(job, grid, dev, stream) : launch_both<ENEC_FP16, 1>(job, grid, dev, stream);
}
