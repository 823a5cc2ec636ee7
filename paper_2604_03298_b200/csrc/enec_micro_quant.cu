// Quantisation into microscaled 4-bit streams and back (layout: enec_micro.cuh).
//
// For a block of 32 values with a = max |x|: the scale is 2^s, s = clamp(floor(log2 a) - 2, -127, 127) (2 is the exponent of
// E2M1's largest power of two), every value x 2^-s is rounded once to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even
// code, above 6 to 6, sign kept), and a block with a NaN or an infinity is one of NaN (scale byte 255). x 2^-s is exact in
// fp32 wherever it is not far below the smallest rounding border, so the code is the one of exact arithmetic.
//
// Both directions are bound by memory: 16 bytes (bf16) in, 4.25 out for every 8 values, some 50 instructions between them.
// A warp takes one row of a record at a time (256 columns: 512 bytes of bf16 on one side, one 128-byte line of the record on the
// other), eight values a lane, four lanes a block. It does so for rows r, r + 32, r + 64 and r + 96 together: four independent
// loads in flight per lane, and the four rows' scales are neighbours in the record (16 bytes per four chunks).
#include "enec_micro.cuh"

#include <mutex>

namespace enec {

bool micro_device(MicroDevice& out) {
    static std::mutex mu;
    static MicroDevice infos[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
    std::lock_guard<std::mutex> lock(mu);
    MicroDevice& d = infos[dev];
    if (d.sms == 0 && cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return false;
    d.ordinal = dev;
    out = d;
    return true;
}

namespace {

constexpr uint32_t kQuantThreads = 256;
constexpr uint32_t kTasksPerCta = kQuantThreads / 32;          // a warp's task: four rows of a record
constexpr uint32_t kCtasPerRecord = 32 / kTasksPerCta;

struct RecordPlace {
    uint32_t matrix, row_tile, col_tile;
};
__device__ __forceinline__ RecordPlace record_place(uint32_t record, const MicroShape& s) {
    RecordPlace p;
    p.col_tile = record % s.col_tiles;
    const uint32_t strip = record / s.col_tiles;
    p.row_tile = strip % s.row_tiles;
    p.matrix = strip / s.row_tiles;
    return p;
}

// Eight codes, the first in the low four bits (round to nearest even, above the largest to the largest).
__device__ __forceinline__ uint32_t e2m1_codes(const float* x) {
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w)
        : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return w;
}

template <int DT>
__global__ void __launch_bounds__(kQuantThreads) enec_micro_quantize_kernel(const uint8_t* in, uint64_t ld, MicroShape s, uint8_t* out) {
    constexpr int kElem = DT == ENEC_FP32 ? 4 : 2;
    constexpr int kWords = 2 * kElem;
    pdl_wait();
    pdl_launch_dependents();
    const uint32_t lane = threadIdx.x & 31, chunk = lane >> 2, part = lane & 3;
    if (blockIdx.x == 0 && threadIdx.x < kMicroHeaderBytes / 16) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (threadIdx.x == 0) v = make_uint4(kMicroMagic, kMicroVersion, s.batch, s.rows);
        if (threadIdx.x == 1) v = make_uint4(s.cols, 0, uint32_t(s.total), uint32_t(s.total >> 32));
        *reinterpret_cast<uint4*>(out + 16 * threadIdx.x) = v;
    }
    if (s.records == 0) return;
    const uint32_t record = blockIdx.x / kCtasPerRecord;
    const uint32_t low = (blockIdx.x % kCtasPerRecord) * kTasksPerCta + (threadIdx.x >> 5);   // r mod 32 of the warp's rows
    const RecordPlace p = record_place(record, s);
    const uint32_t col = p.col_tile * kMicroCols + 8 * lane;
    const int valid_cols = col < s.cols ? int(min(s.cols - col, 8u)) : 0;
    const uint32_t row0 = p.row_tile * kMicroRows + low;
    const uint8_t* from = in + ((uint64_t(p.matrix) * s.rows + row0) * ld + col) * kElem;
    uint32_t w[4][kWords];
#pragma unroll
    for (int q = 0; q < 4; ++q)
        load_eight<DT>(from + uint64_t(q) * 32 * ld * kElem, row0 + 32 * q < s.rows ? valid_cols : 0, w[q]);
    uint8_t* rec = out + kMicroHeaderBytes + uint64_t(record) * kMicroRecordBytes;
    uint32_t bytes = 0;   // the four rows' scale bytes of this lane's block
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float x[8];
        as_floats<DT>(w[q], x);
        uint32_t top = 0;   // the order of magnitudes is the order of their bits; a NaN's are the largest
        if constexpr (DT == ENEC_FP32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, w[q][i] & 0x7FFFFFFFu);
        } else {   // two at a time, in their own type
            uint32_t two = __vmaxu2(__vmaxu2(w[q][0] & 0x7FFF7FFFu, w[q][1] & 0x7FFF7FFFu), __vmaxu2(w[q][2] & 0x7FFF7FFFu, w[q][3] & 0x7FFF7FFFu));
            two = max(two >> 16, two & 0xFFFFu);
            top = DT == ENEC_BF16 ? two << 16 : __float_as_uint(MicroType<ENEC_FP16>::unpack(two).x);
        }
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t exponent = top >> 23;   // floor(log2) + 127, and 0 for zero and subnormal numbers
        const uint32_t byte = exponent == 255 ? 255u : exponent < 2 ? 0u : exponent - 2;
        const float inverse = __uint_as_float((254u - min(byte, 253u)) << 23);   // 2^(127 - byte)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= inverse;
        const uint32_t codes = byte == 255 ? 0u : e2m1_codes(x);
        const uint32_t row = low + 32 * q;
        *reinterpret_cast<uint32_t*>(rec + row * 128 + ((chunk ^ (row & 7)) << 4) + part * 4) = codes;
        bytes |= byte << (8 * q);
    }
    // lane (chunk 4a, part q) stores the four bytes of row q's chunks 4a .. 4a + 3
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t theirs = __shfl_sync(0xFFFFFFFFu, bytes, ((chunk & 4) + j) * 4);
        word |= ((theirs >> (8 * part)) & 0xFFu) << (8 * j);
    }
    if ((chunk & 3) == 0) *reinterpret_cast<uint32_t*>(rec + kMicroElemBytes + (chunk >> 2) * 512 + low * 16 + part * 4) = word;
}

// Rows of 8 values a lane, from word to word the warp's columns in order, to a row that begins `off` bytes behind a 16-byte
// boundary: every lane stores the whole granule that holds its first element, with the last `off` bytes of the lane before; what
// a granule lacks at either end of the row goes out element by element. valid: elements of this lane inside the matrix.
template <int DT>
__device__ __forceinline__ void store_eight(uint8_t* p, int valid, const uint32_t* w, uint32_t lane) {
    constexpr int kElem = DT == ENEC_FP32 ? 4 : 2;
    constexpr int kWords = 2 * kElem;
    const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p)) & 15u;   // the same for all lanes of the warp
    auto element = [&](int j) {
        if constexpr (kElem == 4) *reinterpret_cast<uint32_t*>(p + 4 * j) = w[j];
        if constexpr (kElem == 2) *reinterpret_cast<uint16_t*>(p + 2 * j) = uint16_t(j & 1 ? w[j / 2] >> 16 : w[j / 2]);
    };
    if (off == 0) {
        if (kElem == 4 && valid == 8 && (reinterpret_cast<uintptr_t>(p) & 31) == 0) {
            // 32 bytes a lane in one instruction: two of 16 touch every sector twice (8192 x 2048 values: 20.3 us)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                         "r"(w[kWords - 4]), "r"(w[kWords - 3]), "r"(w[kWords - 2]), "r"(w[kWords - 1])
                         : "memory");
        } else if (valid == 8) {
#pragma unroll
            for (int g = 0; g < kWords / 4; ++g)
                *reinterpret_cast<uint4*>(p + 16 * g) = make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < valid) element(j);
        }
        return;
    }
    // a: the lane before's last 16 bytes, then this lane's; shifted up by off bytes, its granules begin at word 4
    uint32_t a[kWords + 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __shfl_up_sync(0xFFFFFFFFu, w[kWords - 4 + i], 1);
#pragma unroll
    for (int i = 0; i < kWords; ++i) a[4 + i] = w[i];
    if (off & 8) {
#pragma unroll
        for (int i = kWords + 3; i >= 2; --i) a[i] = a[i - 2];
    }
    if (off & 4) {
#pragma unroll
        for (int i = kWords + 3; i >= 1; --i) a[i] = a[i - 1];
    }
    if (off & 2) {
#pragma unroll
        for (int i = kWords + 3; i >= 1; --i) a[i] = __funnelshift_l(a[i - 1], a[i], 16);
    }
    const int head = (8 * kElem - int(off)) / kElem;         // elements that end at this lane's last granule boundary
    const bool whole = lane > 0 && valid >= head;
    const bool next_whole = __shfl_down_sync(0xFFFFFFFFu, int(whole), 1) && lane < 31;
    if (whole) {
#pragma unroll
        for (int g = 0; g < kWords / 4; ++g)
            *reinterpret_cast<uint4*>(p - off + 16 * g) = make_uint4(a[4 + 4 * g], a[5 + 4 * g], a[6 + 4 * g], a[7 + 4 * g]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < valid && (j < head ? !whole : !next_whole)) element(j);
}

template <int DT>
__global__ void __launch_bounds__(kQuantThreads)
    enec_micro_dequantize_kernel(const uint8_t* in, MicroShape s, uint8_t* out, uint64_t ld, int* status) {
    constexpr int kElem = DT == ENEC_FP32 ? 4 : 2;
    constexpr int kWords = 2 * kElem;
    pdl_wait();
    pdl_launch_dependents();
    if (s.records == 0) {
        if (threadIdx.x == 0 && !micro_header_ok(in, s)) report(status, ENEC_ERR_BAD_STREAM);
        return;
    }
    const uint32_t lane = threadIdx.x & 31, chunk = lane >> 2, part = lane & 3;
    const uint32_t record = blockIdx.x / kCtasPerRecord;
    const uint32_t low = (blockIdx.x % kCtasPerRecord) * kTasksPerCta + (threadIdx.x >> 5);
    const RecordPlace p = record_place(record, s);
    const uint8_t* rec = in + kMicroHeaderBytes + uint64_t(record) * kMicroRecordBytes;
    const uint4 scales = __ldg(reinterpret_cast<const uint4*>(rec + kMicroElemBytes + (chunk >> 2) * 512 + low * 16));
    uint32_t codes[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t row = low + 32 * q;
        codes[q] = __ldg(reinterpret_cast<const uint32_t*>(rec + row * 128 + ((chunk ^ (row & 7)) << 4) + part * 4));
    }
    if (!micro_header_ok(in, s)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(status, ENEC_ERR_BAD_STREAM);
        return;
    }
    const uint32_t col = p.col_tile * kMicroCols + 8 * lane;
    const int valid = col < s.cols ? int(min(s.cols - col, 8u)) : 0;
    const uint32_t row0 = p.row_tile * kMicroRows + low;
    uint8_t* to = out + ((uint64_t(p.matrix) * s.rows + row0) * ld + col) * kElem;
    const uint32_t of_row[4] = {scales.x, scales.y, scales.z, scales.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (row0 + 32 * q >= s.rows) break;   // the same for the whole warp
        const uint32_t byte = (of_row[q] >> (8 * (chunk & 3))) & 0xFFu;
        const float scale = micro_scale(byte);
        const uint4 h = e2m1_values(codes[q]);
        const uint32_t hw[4] = {h.x, h.y, h.z, h.w};
        uint32_t w[kWords];
        if (DT == ENEC_FP16 && __all_sync(0xFFFFFFFFu, byte - 113u < 30u)) {
            // scales of 2^-14 .. 2^15 are fp16 numbers, and a product of two is rounded once: half the instructions
            const uint32_t factor = ((byte - 112) << 10) * 0x10001u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __half2 v = __hmul2(reinterpret_cast<const __half2&>(hw[i]), reinterpret_cast<const __half2&>(factor));
                w[i] = reinterpret_cast<const uint32_t&>(v);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 v = MicroType<ENEC_FP16>::unpack(hw[i]);
                if constexpr (DT == ENEC_FP32) {
                    w[2 * i] = __float_as_uint(v.x * scale);
                    w[2 * i + 1] = __float_as_uint(v.y * scale);
                } else {
                    w[i] = MicroType<DT>::pack(v.x * scale, v.y * scale);
                }
            }
        }
        store_eight<DT>(to + uint64_t(q) * 32 * ld * kElem, valid, w, lane);
    }
}

}  // namespace
}  // namespace enec

using namespace enec;

extern "C" {

size_t enec_microscaled_size(size_t batch, size_t rows, size_t cols) {
    MicroShape s;
    return make_micro_shape(batch, rows, cols, s) ? size_t(s.total) : 0;
}

enec_status enec_quantize_microscaled(const void* d_in, enec_dtype dt, size_t batch, size_t rows, size_t cols, size_t ld, void* d_out,
                                      size_t out_capacity, int* d_status, enec_stream_t stream) {
    (void)d_status;   // nothing in the values can make this call fail; kept for the one manner of all calls
    if (!known_dtype(dt)) return ENEC_ERR_UNSUPPORTED_DTYPE;
    MicroShape s;
    if (!make_micro_shape(batch, rows, cols, s)) return ENEC_ERR_TOO_LARGE;
    if ((!d_in && s.records) || !d_out || !micro_aligned16(d_in) || !micro_aligned16(d_out) || ld < cols || (uint64_t(ld) >> 36))
        return ENEC_ERR_INVALID_ARG;
    if (out_capacity < s.total) return ENEC_ERR_BUFFER_TOO_SMALL;
    const uint32_t grid = s.records ? uint32_t(s.records) * kCtasPerRecord : 1;
    const uint8_t* in = static_cast<const uint8_t*>(d_in);
    uint8_t* out = static_cast<uint8_t*>(d_out);
    const cudaError_t err =
        dt == ENEC_BF16   ? launch_pdl(enec_micro_quantize_kernel<ENEC_BF16>, grid, kQuantThreads, 0, stream, in, uint64_t(ld), s, out)
        : dt == ENEC_FP16 ? launch_pdl(enec_micro_quantize_kernel<ENEC_FP16>, grid, kQuantThreads, 0, stream, in, uint64_t(ld), s, out)
                          : launch_pdl(enec_micro_quantize_kernel<ENEC_FP32>, grid, kQuantThreads, 0, stream, in, uint64_t(ld), s, out);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

enec_status enec_dequantize_microscaled(const void* d_in, size_t in_size, enec_dtype dt, size_t batch, size_t rows, size_t cols,
                                        void* d_out, size_t ld, int* d_status, enec_stream_t stream) {
    if (!known_dtype(dt)) return ENEC_ERR_UNSUPPORTED_DTYPE;
    MicroShape s;
    if (!make_micro_shape(batch, rows, cols, s)) return ENEC_ERR_TOO_LARGE;
    if (!d_in || (!d_out && s.records) || !micro_aligned16(d_in) || !micro_aligned16(d_out) || ld < cols || (uint64_t(ld) >> 36))
        return ENEC_ERR_INVALID_ARG;
    if (in_size < s.total) return ENEC_ERR_BUFFER_TOO_SMALL;
    const uint32_t grid = s.records ? uint32_t(s.records) * kCtasPerRecord : 1;
    const uint8_t* in = static_cast<const uint8_t*>(d_in);
    uint8_t* out = static_cast<uint8_t*>(d_out);
    const cudaError_t err =
        dt == ENEC_BF16 ? launch_pdl(enec_micro_dequantize_kernel<ENEC_BF16>, grid, kQuantThreads, 0, stream, in, s, out, uint64_t(ld), d_status)
        : dt == ENEC_FP16
            ? launch_pdl(enec_micro_dequantize_kernel<ENEC_FP16>, grid, kQuantThreads, 0, stream, in, s, out, uint64_t(ld), d_status)
            : launch_pdl(enec_micro_dequantize_kernel<ENEC_FP32>, grid, kQuantThreads, 0, stream, in, s, out, uint64_t(ld), d_status);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

}  // extern "C"
