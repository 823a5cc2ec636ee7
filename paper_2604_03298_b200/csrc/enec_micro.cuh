// Microscaled 4-bit streams: layout, and what their kernels share.
//
// A stream holds `batch` matrices of rows x cols values in E2M1 (sign, two exponent bits, one mantissa bit) with one
// E8M0 scale (a power of two) for every 32 neighbouring values of a row: the MXFP4 form of the OCP microscaling formats.
// Behind a header of 128 bytes, each matrix is cut into records of 128 rows x 256 columns, the records of 128 rows one after
// another along the columns. A record is what one stage of a matrix kernel takes: 16384 bytes of elements in the order in
// which the tensor cores read a K-major operand from shared memory (rows of 128 bytes whose 16-byte chunks are exchanged by
// the row's number mod 8), and 1024 bytes of scales in the order in which they go to tensor memory (512 bytes for every
// four chunks: row r at 16 (r mod 32) + 4 (r / 32)). So a record is copied as it is, without a tensor map, and a chunk
// is exactly one block of 32 values with its scale. Rows and columns behind the matrix are zero bytes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "enec_common.cuh"
#include "enec_launch.cuh"

namespace enec {

constexpr uint32_t kMicroMagic = 0x344D4E45u;  // "ENM4" little-endian
constexpr uint32_t kMicroVersion = 1;
constexpr uint32_t kMicroHeaderBytes = 128;
constexpr uint32_t kMicroRows = 128;           // of a record
constexpr uint32_t kMicroCols = 256;
constexpr uint32_t kMicroElemBytes = kMicroRows * kMicroCols / 2;
constexpr uint32_t kMicroScaleBytes = kMicroRows * kMicroCols / 32;
constexpr uint32_t kMicroRecordBytes = kMicroElemBytes + kMicroScaleBytes;
constexpr uint32_t kMicroBlock = 32;

// The first 32 bytes of the header; the other 96 are zero.
struct alignas(16) MicroHeader {
    uint32_t magic;
    uint32_t version;
    uint32_t batch;
    uint32_t rows;
    uint32_t cols;
    uint32_t zero;
    uint32_t total_low, total_high;  // bytes of the stream
};
static_assert(sizeof(MicroHeader) == 32, "two 16-byte loads");

struct MicroShape {
    uint32_t batch, rows, cols;
    uint32_t row_tiles, col_tiles;   // of one matrix
    uint64_t records;                // of all matrices
    uint64_t total;                  // bytes
};

// False for more records than an index of 31 bits has room for (8 TiB and more).
__host__ inline bool make_micro_shape(uint64_t batch, uint64_t rows, uint64_t cols, MicroShape& s) {
    if ((batch >> 31) || (rows >> 31) || (cols >> 31)) return false;
    s.batch = uint32_t(batch);
    s.rows = uint32_t(rows);
    s.cols = uint32_t(cols);
    s.row_tiles = uint32_t((rows + kMicroRows - 1) / kMicroRows);
    s.col_tiles = uint32_t((cols + kMicroCols - 1) / kMicroCols);
    const uint64_t per_matrix = uint64_t(s.row_tiles) * s.col_tiles;
    if (per_matrix && batch > (uint64_t(1) << 29) / per_matrix) return false;
    s.records = batch * per_matrix;
    s.total = kMicroHeaderBytes + s.records * kMicroRecordBytes;
    return true;
}

inline bool micro_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

struct MicroDevice {
    int sms = 0;
    int ordinal = 0;
};
// Facts of the current device; false where the ordinal is beyond the library's tables.
bool micro_device(MicroDevice& out);

// Lets a kernel take `bytes` of dynamic shared memory on the current device; `done` has a bit per device and belongs to the kernel.
template <class Kernel>
inline bool allow_shared(std::atomic<uint64_t>& done, const MicroDevice& dev, Kernel* kernel, uint32_t bytes) {
    const uint64_t bit = uint64_t(1) << dev.ordinal;
    if (done.load(std::memory_order_acquire) & bit) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes)) != cudaSuccess) return false;
    done.fetch_or(bit, std::memory_order_release);
    return true;
}

#ifdef __CUDACC__

// The header's first 32 bytes, loaded early and looked at late. The host has checked the stream's size against the shape, so every read of
// the records is in bounds whatever the header holds: kernels work first and ask whether it says what the call says before they store.
struct MicroProbe {
    uint4 a, b;
    __device__ __forceinline__ explicit MicroProbe(const uint8_t* stream)
        : a(*reinterpret_cast<const uint4*>(stream)), b(*reinterpret_cast<const uint4*>(stream + 16)) {}
    __device__ __forceinline__ bool fits(const MicroShape& s) const {
        return a.x == kMicroMagic && a.y == kMicroVersion && a.z == s.batch && a.w == s.rows && b.x == s.cols && b.y == 0 &&
               b.z == uint32_t(s.total) && b.w == uint32_t(s.total >> 32);
    }
};
__device__ __forceinline__ bool micro_header_ok(const uint8_t* stream, const MicroShape& s) { return MicroProbe(stream).fits(s); }

// 2^(byte - 127); byte 0 is a subnormal number of fp32, byte 255 stands for not-a-number.
__device__ __forceinline__ float micro_scale(uint32_t byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

template <int DT>
struct MicroType;
template <>
struct MicroType<ENEC_BF16> {
    using T = __nv_bfloat16;
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return reinterpret_cast<const uint32_t&>(v);
    }
    static __device__ __forceinline__ T one(float a) { return __float2bfloat16_rn(a); }
};
template <>
struct MicroType<ENEC_FP16> {
    using T = __half;
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(reinterpret_cast<const __half2&>(w)); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __half2 v = __floats2half2_rn(a, b);
        return reinterpret_cast<const uint32_t&>(v);
    }
    static __device__ __forceinline__ T one(float a) { return __float2half_rn(a); }
};
template <>
struct MicroType<ENEC_FP32> {
    using T = float;
    static __device__ __forceinline__ T one(float a) { return a; }
};

// Eight neighbouring elements (16 or 32 bytes) from anywhere on a multiple of the element size: the 16-byte granules that hold them (one
// more than aligned ones would need; none is read that holds no element), to be shifted into words when they are needed.
template <int DT>
struct EightLoaded {
    static constexpr int kElem = DT == ENEC_FP32 ? 4 : 2;
    static constexpr int kWords = 2 * kElem;
    uint32_t a[kWords + 4];
    uint32_t off;
    int valid;   // elements, the first ones; 8 and more: all
    __device__ __forceinline__ void load(const uint8_t* p, int valid_) {
        valid = valid_;
        off = uint32_t(reinterpret_cast<uintptr_t>(p)) & 15u;
        const uint8_t* base = p - off;
        const int last = valid > 0 ? int(off) + min(valid, 8) * kElem : 0;   // bytes from base to the end of the elements
#pragma unroll
        for (int g = 0; g < kWords / 4 + 1; ++g) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (16 * g < last) v = __ldg(reinterpret_cast<const uint4*>(base + 16 * g));
            a[4 * g] = v.x, a[4 * g + 1] = v.y, a[4 * g + 2] = v.z, a[4 * g + 3] = v.w;
        }
    }
    // The elements as words, zeros behind the valid ones.
    __device__ __forceinline__ void words(uint32_t* w) {
        if (off & 8) {
#pragma unroll
            for (int i = 0; i < kWords + 2; ++i) a[i] = a[i + 2];
        }
        if (off & 4) {
#pragma unroll
            for (int i = 0; i < kWords + 1; ++i) a[i] = a[i + 1];
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = off & 2 ? __funnelshift_r(a[i], a[i + 1], 16) : a[i];
        if (valid < 8) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if (kElem == 4) w[i] = i < valid ? w[i] : 0;
                if (kElem == 2) w[i] = 2 * i + 1 < valid ? w[i] : 2 * i < valid ? w[i] & 0xFFFFu : 0;
            }
        }
    }
};
template <int DT>
__device__ __forceinline__ void load_eight(const uint8_t* p, int valid, uint32_t* w) {
    constexpr int kWords = EightLoaded<DT>::kWords;
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
    if (valid <= 0) return;
    if ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && valid >= 8) {
#pragma unroll
        for (int g = 0; g < kWords / 4; ++g) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(p + 16 * g));
            w[4 * g] = v.x, w[4 * g + 1] = v.y, w[4 * g + 2] = v.z, w[4 * g + 3] = v.w;
        }
        return;
    }
    EightLoaded<DT> eight;
    eight.load(p, valid);
    eight.words(w);
}

template <int DT>
__device__ __forceinline__ void as_floats(const uint32_t* w, float* x) {
    if constexpr (DT == ENEC_FP32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = MicroType<DT>::unpack(w[i]);
            x[2 * i] = v.x;
            x[2 * i + 1] = v.y;
        }
    }
}

// The values of eight codes, two to a word of fp16 (exact).
__device__ __forceinline__ uint4 e2m1_values(uint32_t w) {
    uint4 h;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h.x), "=r"(h.y), "=r"(h.z), "=r"(h.w)
        : "r"(w));
    return h;
}

#endif  // __CUDACC__

}  // namespace enec
