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
// The columns are fp16 too: fp16 activations as they are; bf16 ones times the power of two that takes the largest magnitude of 128
// neighbouring values to 2^14 .. 2^15. Values down to 2^-29 of the largest keep all their bits then, below that the error is at
// most 2^-39 of the largest: far under the 2^-24 of each fp32 sum. fp32 values (an expert's hidden values) are rounded to fp16 after
// the same scaling: 11 bits, as an fp16 model keeps them and three more than a bf16 one does.
//
// A strip is 16 rows of a record: 4j .. 4j + 3, + 32, + 64, + 96, whose scales are 64 neighbouring bytes for every 128
// columns. A unit is a strip x 128 columns: 1024 bytes and 64 of scales. A CTA has 16 warps (what hides a unit's chain of copy,
// ldmatrix, conversion and products is other warps: with 8 on an SM, 8 tokens x 4096 x 14336 took 32 us), in teams of 4, 8 or 16. A
// team's warps share a strip's units, its sums are joined in shared memory. Each warp has a ring of its own that it fills with
// cp.async and reads with ldmatrix, without a barrier among warps, and which goes on from strip to strip while sums are joined.
#pragma once

#include "enec_micro.cuh"

namespace enec {

constexpr uint32_t kFewWarps = 16;
constexpr uint32_t kFewThreads = kFewWarps * 32;
constexpr uint32_t kUnitCols = 128;
constexpr uint32_t kUnitBytes = 16 * 64;
constexpr uint32_t kUnitScales = 64;

__host__ __device__ constexpr uint32_t few_stages(int mats) { return mats == 2 ? 3 : 4; }
__host__ __device__ constexpr uint32_t few_stage_bytes(int mats) { return mats * (kUnitBytes + kUnitScales); }
__host__ __device__ constexpr uint32_t few_ring_bytes(int mats) { return kFewWarps * few_stages(mats) * few_stage_bytes(mats); }
// Warps' sums of a strip: rows of 8 NT columns and a gap of 4 words against bank conflicts.
__host__ __device__ constexpr uint32_t few_sum_row(int nt) { return 8 * nt + 4; }
__host__ __device__ constexpr uint32_t few_sum_words(int nt, int mats) { return mats * 16 * few_sum_row(nt); }   // of a warp
__host__ __device__ constexpr uint32_t few_fixed_bytes(int nt, int mats) { return few_ring_bytes(mats) + kFewWarps * few_sum_words(nt, mats) * 4; }
// The staged columns of a unit: 128 values of fp16 each, and room for the inverses of 8 NT factors.
__host__ __device__ constexpr uint32_t few_unit_bytes(int nt, uint32_t columns) { return columns * kUnitCols * 2 + 8 * nt * 4; }

// Warps of a team: the split that leaves the fewest warps without work, over strips (of which `ctas` CTAs work at the same time) and
// over a strip's units. strips 256, 896 and 8016 of 32 units on 148 SMs: 8, 16 and 4.
inline uint32_t few_team(uint64_t strips, uint32_t units, uint32_t ctas) {
    uint32_t best = 16;
    double most = 0;
    for (uint32_t team : {4u, 8u, 16u}) {
        const uint64_t teams = uint64_t(ctas) * (kFewWarps / team);
        const double busy = double(strips) / double((strips + teams - 1) / teams * teams) * units / ((units + team - 1) / team * team);
        if (busy > most * 1.02) most = busy, best = team;
    }
    return best;
}

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

// Asks for unit u of strip j of the records of a row tile, which begin at `records`. Row m of the strip is row 4j + m mod 4 + 32 (m / 4)
// of the record: its chunks are exchanged by (m mod 4) + 4 (j mod 2), and in the stage, where rows are 64 bytes, by (m / 2) mod 4.
__device__ __forceinline__ void ask_unit(const uint8_t* records, uint32_t j, uint32_t u, uint32_t stage, uint32_t lane) {
    const uint8_t* rec = records + uint64_t(u >> 1) * kMicroRecordBytes + j * 512;
    const uint32_t m = lane >> 2, c = lane & 3;
    const uint32_t from = ((m & 3) + 32 * (m >> 2)) * 128 + (((c ^ (m & 3)) << 4) ^ (((j ^ u) & 1) << 6));
    const uint32_t to = stage + m * 64 + ((c ^ ((m >> 1) & 3)) << 4);
    cp_async16(to, rec + from);
    cp_async16(to + 512, rec + from + 8192);   // row m + 8
    if (lane < 4) cp_async16(stage + kUnitBytes + 16 * lane, rec + kMicroElemBytes + (u & 1) * 512 - j * 448 + 16 * lane);
}

// Adds one unit's products to acc. values: the address of the unit's staged columns (see stage_columns), this lane's column and
// quarter added; factors: of its columns' inverse factors, 2 (lane mod 4) added. This lane's column n of tile nt exists where exists[nt].
template <int NT>
__device__ __forceinline__ void add_unit(float (*acc)[4], uint32_t stage, uint32_t values, const float* factors, uint32_t columns, const bool* exists,
                                         uint32_t lane) {
    const uint32_t g = lane >> 2;
    // ldmatrix: lanes 8i .. 8i + 7 give the rows of matrix i: rows 0-7 and 8-15 of the block, then of the next one
    const uint32_t m = (lane & 7) + (lane & 8), next = lane >> 4;
    const uint32_t row = stage + m * 64, turn = (m >> 1) & 3;
    const uint32_t at = stage + kUnitBytes + (g & 3) * 16 + (g >> 2) * 4;
    const uint32_t upper = lds32(at), lower = lds32(at + 8);    // four scale bytes of rows g and g + 8
    float sum[NT][4] = {};
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
                if (exists[nt]) x = lds128(values + (2 * pair + b) * columns * 64 + nt * 8 * 64);
                float c[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(c, top.x, bottom.x, top.y, bottom.y, x.x, x.y);
                mma_f16(c, top.z, bottom.z, top.w, bottom.w, x.z, x.w);
                sum[nt][0] = fmaf(s0, c[0], sum[nt][0]);
                sum[nt][1] = fmaf(s0, c[1], sum[nt][1]);
                sum[nt][2] = fmaf(s1, c[2], sum[nt][2]);
                sum[nt][3] = fmaf(s1, c[3], sum[nt][3]);
            }
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const float f0 = factors[nt * 8], f1 = factors[nt * 8 + 1];
        acc[nt][0] = fmaf(f0, sum[nt][0], acc[nt][0]);
        acc[nt][1] = fmaf(f1, sum[nt][1], acc[nt][1]);
        acc[nt][2] = fmaf(f0, sum[nt][2], acc[nt][2]);
        acc[nt][3] = fmaf(f1, sum[nt][3], acc[nt][3]);
    }
}

// The sums of this warp to shared memory: sums[row of the strip][column].
template <int NT>
__device__ __forceinline__ void put_sums(float* sums, const float (*acc)[4], uint32_t lane) {
    const uint32_t g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        *reinterpret_cast<float2*>(sums + g * few_sum_row(NT) + nt * 8 + 2 * t) = make_float2(acc[nt][0], acc[nt][1]);
        *reinterpret_cast<float2*>(sums + (g + 8) * few_sum_row(NT) + nt * 8 + 2 * t) = make_float2(acc[nt][2], acc[nt][3]);
    }
}
// A barrier of one team's warps.
__device__ __forceinline__ void team_sync(uint32_t team, uint32_t threads) {
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory");
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

// Lays columns out for add_unit, by all warps of the CTA; barriers in front and behind are the caller's. Column i's values are
// those of row_of(i) from `from` on, zeros behind `cols`. Of every 32 values column after column, 64 bytes each; half a warp takes 128
// values of a column, and their factor's inverse goes to inverse[unit * pitch + column].
template <int DT, class RowOf>
__device__ __forceinline__ void stage_columns(RowOf row_of, uint32_t columns, uint32_t units, uint32_t from, uint32_t cols, uint32_t dst,
                                              float* inverse, uint32_t pitch) {
    constexpr int kElem = DT == ENEC_FP32 ? 4 : 2;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = lane & 15;
    const uint32_t pairs = (columns + 1) / 2, tasks = pairs * units;
#pragma unroll 2
    for (uint32_t task = warp; task < tasks; task += kFewWarps) {
        const uint32_t u = task / pairs, i = task % pairs * 2 + (lane >> 4);
        const bool mine = i < columns;
        const uint32_t col = from + u * kUnitCols + 8 * group;
        uint32_t w[2 * kElem];
        load_eight<DT>(mine ? row_of(i) + uint64_t(col) * kElem : nullptr, mine && col < cols ? int(min(cols - col, 8u)) : 0, w);
        float x[8];
        as_floats<DT>(w, x);
        uint32_t top = 0;
        if constexpr (DT != ENEC_FP16) {
            top = larger_finite(0, x);
#pragma unroll
            for (int d = 1; d < 16; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        }
        if (!mine) continue;
        if (group == 0) inverse[u * pitch + i] = DT == ENEC_FP16 ? 1.f : column_inverse(top);
        const uint32_t at = dst + (u * 4 + (group >> 2)) * columns * 64 + i * 64 + (group & 3) * 16;
        if constexpr (DT == ENEC_FP16) {
            sts128(at, make_uint4(w[0], w[1], w[2], w[3]));
        } else {
            const float factor = column_factor(top);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= factor;
            sts128(at, pack_half8(x));
        }
    }
}

#endif  // __CUDACC__

}  // namespace enec
