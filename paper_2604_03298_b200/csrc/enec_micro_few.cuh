// Products of a few columns with microscaled weights: what the product for few tokens and the expert layer share.
//
//   acc[row, column] = sum over blocks b of 2^s[row, b] * (sum over the 32 values of b of q[row, k] * x[column, k])
//
// Such a product reads every weight once and is bound by memory as long as the values are brought back fast enough: 4.25 bits a
// value at 6.5 TB/s are 43 values per clock and SM. One conversion instruction gives two values as fp16 (64 a clock and SM,
// measured 43 with the arithmetic around it; shifts and masks reach 19 pairs), and the inner sums go to mma.m16n8k16 (half
// an instruction a clock and SM, measured), eight columns at a time whether they are used or not; tcgen05 would want its
// operand in shared memory or tensor memory first, one store and one load for each value more. The scale is applied to the inner
// sum in fp32, so it is exact whatever its size; fp16 holds every E2M1 value exactly.
//
// The columns are fp16 too: fp16 activations as they are; bf16 ones times the power of two that takes a row's largest magnitude to
// 2^14 .. 2^15. Values down to 2^-29 of the largest keep all their bits then, below that the error is at most 2^-39 of the largest:
// far under the 2^-24 of each fp32 sum. fp32 values (an expert's hidden values) are rounded to fp16 after the same scaling: 11 bits,
// as an fp16 model keeps them and three more than a bf16 one does.
//
// A strip is 16 rows of a record: 4j .. 4j + 3, + 32, + 64, + 96, whose scales are 64 neighbouring bytes for every 128
// columns. A unit is a strip x 128 columns: 1024 bytes and 64 of scales. The warps of a CTA share a strip's units; each has
// a ring of its own in shared memory that it fills with cp.async and reads with ldmatrix, without a barrier among warps, and which
// goes on from strip to strip while sums are joined.
#pragma once

#include "enec_micro.cuh"

namespace enec {

constexpr uint32_t kFewWarps = 8;
constexpr uint32_t kFewThreads = kFewWarps * 32;
constexpr uint32_t kUnitCols = 128;
constexpr uint32_t kUnitBytes = 16 * 64;
constexpr uint32_t kUnitScales = 64;
constexpr uint32_t kFewStages = 6;

__host__ __device__ constexpr uint32_t few_stage_bytes(int mats) { return mats * (kUnitBytes + kUnitScales); }
__host__ __device__ constexpr uint32_t few_ring_bytes(int mats) { return kFewWarps * kFewStages * few_stage_bytes(mats); }
// Warps' sums of a strip, two sets: rows of 8 NT columns and a gap of 4 words against bank conflicts.
__host__ __device__ constexpr uint32_t few_sum_row(int nt) { return 8 * nt + 4; }
__host__ __device__ constexpr uint32_t few_sum_bytes(int nt, int mats) { return 2 * kFewWarps * mats * 16 * few_sum_row(nt) * 4; }

#ifdef __CUDACC__

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t a, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
                 : "r"(a)
                 : "memory");
}
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two scale bytes as the upper and the lower half of a word of bf16 (exact: 2^-127 is a subnormal number, 255 a NaN).
__device__ __forceinline__ uint32_t scale_pair(uint32_t two_bytes) {
    uint32_t d;
    asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.rn.bf16x2.ue8m0x2 %0, h;\n\t}" : "=r"(d) : "r"(two_bytes));
    return d;
}

// Asks for one unit: columns 128 u .. of strip j of the records of a row tile, which begin at `records`.
__device__ __forceinline__ void ask_unit(const uint8_t* records, uint32_t j, uint32_t u, uint32_t stage, uint32_t lane) {
    const uint8_t* rec = records + uint64_t(u >> 1) * kMicroRecordBytes;
    const uint32_t half = u & 1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t m = (lane >> 2) + 8 * i, c = lane & 3;   // row of the strip, chunk of the unit
        const uint32_t r = 4 * j + (m & 3) + 32 * (m >> 2);
        cp_async16(stage + m * 64 + ((c ^ ((m >> 1) & 3)) << 4), rec + r * 128 + (((4 * half + c) ^ (r & 7)) << 4));
    }
    if (lane < 4) cp_async16(stage + kUnitBytes + 16 * lane, rec + kMicroElemBytes + half * 512 + (4 * j + lane) * 16);
}

// Adds one unit's products to acc. columns: the address of the unit's first block in the staged columns (see stage_share), this
// lane's column and quarter added; a block is `block_bytes` long; lane's column n of tile nt exists where nt < tiles.
template <int NT>
__device__ __forceinline__ void add_unit(float (*acc)[4], uint32_t stage, uint32_t columns, uint32_t block_bytes, const bool* exists,
                                         uint32_t lane) {
    const uint32_t g = lane >> 2;
    // ldmatrix: lanes 8i .. 8i + 7 give the rows of matrix i: rows 0-7 and 8-15 of the block, then of the next one
    const uint32_t m = (lane & 7) + (lane & 8), next = lane >> 4;
    const uint32_t row = stage + m * 64, turn = (m >> 1) & 3;
    const uint32_t at = stage + kUnitBytes + (g & 3) * 16 + (g >> 2) * 4;
    const uint32_t upper = lds32(at), lower = lds32(at + 8);    // four scale bytes of rows g and g + 8
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) {
        uint32_t w[4];
        ldmatrix4(row + (((2 * pair + next) ^ turn) << 4), w[0], w[1], w[2], w[3]);
        const uint32_t su = scale_pair(pair ? upper >> 16 : upper), sl = scale_pair(pair ? lower >> 16 : lower);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint4 top = e2m1_values(w[2 * b]), bottom = e2m1_values(w[2 * b + 1]);
            const float s0 = __uint_as_float(b ? su & 0xFFFF0000u : su << 16), s1 = __uint_as_float(b ? sl & 0xFFFF0000u : sl << 16);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (exists[nt]) x = lds128(columns + (2 * pair + b) * block_bytes + nt * 8 * 64);
                float c[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(c, top.x, bottom.x, top.y, bottom.y, x.x, x.y);
                mma_f16(c, top.z, bottom.z, top.w, bottom.w, x.z, x.w);
                acc[nt][0] = fmaf(s0, c[0], acc[nt][0]);
                acc[nt][1] = fmaf(s0, c[1], acc[nt][1]);
                acc[nt][2] = fmaf(s1, c[2], acc[nt][2]);
                acc[nt][3] = fmaf(s1, c[3], acc[nt][3]);
            }
        }
    }
}

// The sums of this warp, scaled back, to shared memory: sums[row of the strip][column].
template <int NT>
__device__ __forceinline__ void put_sums(float* sums, const float (*acc)[4], const float* inverse, uint32_t lane) {
    const uint32_t g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const float2 f = *reinterpret_cast<const float2*>(inverse + nt * 8 + 2 * t);
        *reinterpret_cast<float2*>(sums + g * few_sum_row(NT) + nt * 8 + 2 * t) = make_float2(acc[nt][0] * f.x, acc[nt][1] * f.y);
        *reinterpret_cast<float2*>(sums + (g + 8) * few_sum_row(NT) + nt * 8 + 2 * t) = make_float2(acc[nt][2] * f.x, acc[nt][3] * f.y);
    }
}

// Row of the matrix (within the row tile) that row m of strip j is.
__device__ __forceinline__ uint32_t strip_row(uint32_t j, uint32_t m) { return 4 * j + (m & 3) + 32 * (m >> 2); }

// The factor of a row of activations whose largest finite magnitude has the bits `top`, and its inverse.
__device__ __forceinline__ float column_factor(uint32_t top) {
    const uint32_t field = max(top >> 23, 14u);                       // a smaller one: the factor stays at 2^127
    return __uint_as_float((127 + 14 + 127 - field) << 23);
}
__device__ __forceinline__ float column_inverse(uint32_t top) {
    const int field = int(max(top >> 23, 14u)) - 14;                  // 2^(field - 127), a subnormal number where field is 0
    return __uint_as_float(field > 0 ? uint32_t(field) << 23 : 0x00400000u);
}
// The larger of `top` and the magnitudes' bits, those of infinities and NaN left out.
__device__ __forceinline__ uint32_t larger_finite(uint32_t top, const float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        top = max(top, bits < 0x7F800000u ? bits : 0u);
    }
    return top;
}
__device__ __forceinline__ uint4 pack_half8(const float* x) {
    return make_uint4(MicroType<ENEC_FP16>::pack(x[0], x[1]), MicroType<ENEC_FP16>::pack(x[2], x[3]), MicroType<ENEC_FP16>::pack(x[4], x[5]),
                      MicroType<ENEC_FP16>::pack(x[6], x[7]));
}

// Lays this warp's share of the columns out for add_unit: units warp, warp + kFewWarps, ... below `units`, each 128 values from
// column `from` + 128 u on; values behind `cols` are zeros. Of every block of 32 values column after column, 64 bytes each, so a
// block is 64 * columns bytes; row_of(i) is where the i-th column's values come from. Each is scaled by a power of two of the
// warp's own, whose inverse goes to inverse[i]: no other warp reads these units, and sums are scaled back before they are joined.
template <int DT, class RowOf>
__device__ __forceinline__ void stage_share(RowOf row_of, uint32_t columns, uint32_t units, uint32_t from, uint32_t cols, uint32_t dst,
                                            float* inverse, uint32_t warp, uint32_t lane) {
    constexpr int kElem = DT == ENEC_FP32 ? 4 : 2;
    const uint32_t group = lane & 15;   // of eight values in a unit; half a warp takes a row
    for (uint32_t first = 0; first < columns; first += 2) {
        const uint32_t i = first + (lane >> 4);
        const bool mine = i < columns;
        const uint8_t* row = mine ? row_of(i) : nullptr;
        auto load = [&](uint32_t u, float* x) {
            uint32_t w[2 * kElem];
            const uint32_t col = from + u * kUnitCols + 8 * group;
            load_eight<DT>(row + uint64_t(col) * kElem, mine && col < cols ? int(min(cols - col, 8u)) : 0, w);
            as_floats<DT>(w, x);
        };
        uint32_t top = 0;
        if constexpr (DT != ENEC_FP16) {
#pragma unroll 4
            for (uint32_t u = warp; u < units; u += kFewWarps) {
                float x[8];
                load(u, x);
                top = larger_finite(top, x);
            }
#pragma unroll
            for (int d = 1; d < 16; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        }
        const float factor = DT == ENEC_FP16 ? 1.f : column_factor(top);
        if (mine && group == 0) inverse[i] = DT == ENEC_FP16 ? 1.f : column_inverse(top);
#pragma unroll 4
        for (uint32_t u = warp; u < units; u += kFewWarps) {
            float x[8];
            load(u, x);
            if (!mine) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= factor;
            sts128(dst + (u * 4 + (group >> 2)) * columns * 64 + i * 64 + (group & 3) * 16, pack_half8(x));
        }
    }
    __syncwarp();
}

#endif  // __CUDACC__

}  // namespace enec
