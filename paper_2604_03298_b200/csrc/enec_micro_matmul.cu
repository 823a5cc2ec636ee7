// enec_matmul_microscaled: arguments, and which form of the product takes a call.
#include "enec_micro_launch.cuh"

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
    if (cols == 0)   // sums of nothing
        return cudaMemset2DAsync(d_y, ld_y * 2, 0, rows * 2, tokens, stream) == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
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
