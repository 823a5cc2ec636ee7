// enec_matmul_microscaled: arguments, and which form of the product takes a call.
#include "enec_micro_launch.cuh"

namespace enec {
namespace {

constexpr uint32_t kZeroThreads = 256;

__global__ void __launch_bounds__(kZeroThreads)
    enec_micro_no_columns_kernel(const uint8_t* x, MicroShape sx, const uint8_t* w, MicroShape sw, uint64_t tokens, uint16_t* y, uint64_t ld_y, int* status) {
    pdl_wait();
    pdl_launch_dependents();
    if (!micro_header_ok(w, sw) || (x && !micro_header_ok(x, sx))) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(status, ENEC_ERR_BAD_STREAM);
        return;
    }
    const uint64_t all = tokens * sw.rows;   // below 2^62
    for (uint64_t i = uint64_t(blockIdx.x) * kZeroThreads + threadIdx.x; i < all; i += uint64_t(gridDim.x) * kZeroThreads) {
        const uint64_t token = i / sw.rows;
        y[token * ld_y + (i - token * sw.rows)] = 0;
    }
}

}  // namespace

enec_status micro_no_columns(const uint8_t* x, const MicroShape& sx, const uint8_t* w, const MicroShape& sw, uint64_t tokens, void* y, uint64_t ld_y,
                             int* status, cudaStream_t stream) {
    const uint64_t blocks = (tokens * sw.rows + kZeroThreads - 1) / kZeroThreads;
    const cudaError_t err = launch_pdl(enec_micro_no_columns_kernel, uint32_t(blocks < 4096 ? blocks : 4096), kZeroThreads, 0, stream, x, sx, w, sw, tokens,
                                       static_cast<uint16_t*>(y), ld_y, status);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

}  // namespace enec

using namespace enec;

extern "C" enec_status enec_matmul_microscaled(const void* d_x, enec_dtype dt, size_t tokens, size_t ld_x, const void* d_w, size_t w_size,
                                               size_t rows, size_t cols, void* d_y, size_t ld_y, int* d_status, enec_stream_t stream) {
    if (dt != ENEC_BF16 && dt != ENEC_FP16) return ENEC_ERR_UNSUPPORTED_DTYPE;
    MicroProduct p;
    if (!make_micro_shape(1, rows, cols, p.s) || (tokens >> 31)) return ENEC_ERR_TOO_LARGE;
    if (tokens == 0 || rows == 0) return ENEC_OK;
    if ((!d_x && cols) || !d_w || !d_y || !micro_aligned16(d_x) || !micro_aligned16(d_w) || !micro_aligned16(d_y) || ld_x < cols ||
        ld_y < rows || (uint64_t(ld_x) >> 36) || (uint64_t(ld_y) >> 36))
        return ENEC_ERR_INVALID_ARG;
    if (w_size < p.s.total) return ENEC_ERR_BUFFER_TOO_SMALL;
    if (cols == 0) return micro_no_columns(nullptr, p.s, static_cast<const uint8_t*>(d_w), p.s, tokens, d_y, ld_y, d_status, stream);
    MicroDevice dev;
    if (!micro_device(dev)) return ENEC_ERR_CUDA;
    p.dt = dt;
    p.x = static_cast<const uint8_t*>(d_x);
    p.ld_x = ld_x;
    p.tokens = uint32_t(tokens);
    p.w = static_cast<const uint8_t*>(d_w);
    p.y = static_cast<uint8_t*>(d_y);
    p.ld_y = ld_y;
    p.status = d_status;
    return micro_few_takes(p.tokens, p.s.col_tiles) ? micro_few(p, dev, stream) : micro_many(p, dev, stream);
}
