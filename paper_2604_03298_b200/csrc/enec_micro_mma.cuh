// tcgen05 in the form the products use it: one CTA per tile, accumulators in tensor memory, operands in shared memory, K-major
// with rows of 128 bytes whose 16-byte chunks are exchanged by the row's number mod 8.
//
// One thread issues. The whole warp runs its loop, waits included, and the issuing instructions are predicated on the elected lane, so
// that control flow and descriptors stay uniform: four small matrix instructions with their scales and waits take 260 clocks to
// issue, 370 with a branch for one lane around them.
#pragma once

#include "enec_micro.cuh"

namespace enec {

// Dynamic shared memory that a kernel takes at least, by its columns of tensor memory: above 256, or up to 256. On an SM's 228 KB two
// CTAs can then only be neighbours if there is room for both their columns, so no allocation ever waits for another CTA. (One that did
// could wait forever: CTAs of two clusters, each holding columns on one SM and waiting for them on another, meet in no barrier.)
constexpr uint32_t kTmemAloneShared = 160 * 1024;
constexpr uint32_t kTmemHalfShared = 77 * 1024;

#ifdef __CUDACC__

__device__ __forceinline__ void tmem_alloc(uint32_t* where, uint32_t columns) {   // by one whole warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns) {      // by the warp that has taken it
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
__device__ __forceinline__ void tcgen05_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// One lane of the warp, the same one at every call.
__device__ __forceinline__ uint32_t elected() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e;
}
// Arrives on `bar` when all tcgen05 operations that this thread has issued are done.
__device__ __forceinline__ void tcgen05_commit(uint32_t leader, uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.u32 e, %1, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)),
        "r"(leader)
        : "memory");
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Whether a phase is complete, without waiting. Shared memory answers after 200 to 300 clocks while other warps keep it busy, so the warp
// that issues asks for the next stage before it issues the present one's instructions: with the question in front of them a
// step of 32 tokens took 900 clocks, most of it two such answers.
__device__ __forceinline__ uint32_t mbar_complete(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(smem_u32(bar)), "r"(parity)
                 : "memory");
    return ok;
}
// Where a wait runs out, suspended_wait() may say so to some lanes of a warp and tell others that the phase is complete. What comes next are
// instructions of the whole warp (votes, loads of tensor memory, barriers), and a warp in two parts would wait in them for good. So a
// warp that leaves its loop then does so together (warp_wait), as it does by the flag by which a CTA gives up (warp_failed); the
// warps that would feel the votes (2048 x 4096 x 4096: 58.2 instead of 56.1 us) set the flag and go on to the end of their loop, each
// further wait two tries long (wait_or_fail; its first try is not among the counted ones, which takes 1.7 us off; as long a try as
// theirs or a mere question there cost 0.3 us). The warps that issue matrix instructions run no instruction of the whole warp but
// behind a __syncwarp(), at the end of a task or of their part, and leave lane by lane.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xFFFFFFFFu, suspended_wait(bar, parity, abort_flag));
}
__device__ __forceinline__ void wait_or_fail(uint64_t* bar, uint32_t parity, volatile int* flag) {
    if (!mbar_try_wait(bar, parity) && !suspended_wait(bar, parity, flag)) *flag = 1;
}
__device__ __forceinline__ bool warp_failed(volatile int* flag) { return __any_sync(0xFFFFFFFFu, *flag); }
// One arrival for a warp, behind what all its lanes have done.
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// Descriptor of an operand: address, 1024 bytes from eight rows to the next eight, 128-byte swizzle.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return uint64_t((addr & 0x3FFFF) >> 4) | uint64_t(1) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// Descriptor of 512 bytes of scales: 32 rows of 16 bytes, eight rows after another, no swizzle.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) {
    return uint64_t((addr & 0x3FFFF) >> 4) | uint64_t(1) << 16 | uint64_t(128 >> 4) << 32 | uint64_t(1) << 46;
}
// Those 512 bytes to four columns of tensor memory, the same for all four groups of 32 lanes.
__device__ __forceinline__ void copy_scales(uint32_t leader, uint32_t tmem, uint64_t desc) {
    asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.u32 e, %2, 0;\n\t@e tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(tmem), "l"(desc),
                 "r"(leader)
                 : "memory");
}

// D (128 rows x n columns) (+)= A B^T over 64 columns of E2M1 with one scale per 32.
__device__ __forceinline__ void mma_scaled(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scale_a, uint32_t scale_b,
                                           bool add) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.u32 p, %6, 0;\n\t"
        "setp.ne.u32 e, %7, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(uint32_t(add)), "r"(leader)
        : "memory");
}
// E2M1 operands (1), E8M0 scales (bit 23), both K-major; the pair of scale bytes in their words goes in at bits 4 (B) and 29 (A).
__device__ __forceinline__ uint32_t scaled_idesc(uint32_t n) { return 1u << 7 | 1u << 10 | (n >> 3) << 17 | 1u << 23 | 1u << 27; }

// D (128 rows x n columns) (+)= A B^T over 16 columns of bf16 or fp16, fp32 sums.
__device__ __forceinline__ void mma_16bit(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "setp.ne.u32 e, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add)), "r"(leader)
        : "memory");
}
// fp32 sums (bit 4), bf16 (1) or fp16 (0) operands, both K-major, 128 rows.
__device__ __forceinline__ uint32_t idesc_16bit(bool bf16, uint32_t n) {
    return 1u << 4 | uint32_t(bf16) << 7 | uint32_t(bf16) << 10 | (n >> 3) << 17 | (128u >> 4) << 24;
}

// 16 columns of this warp's 32 lanes of tensor memory.
__device__ __forceinline__ void tmem_load16(uint32_t tmem, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
          "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(tmem));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Stores a warp's 32 rows (lanes) x 16 tokens (registers) to y[token][row]. Two tokens at a time, neighbouring lanes exchange values
// so that each stores two rows of one token: 4 bytes a lane instead of 2. Where a row of y or the matrix ends unevenly, one by one.
template <int DT>
__device__ __forceinline__ void store_tile16(uint8_t* y, uint64_t ld_y, uint32_t token, uint32_t tokens, uint32_t row, uint32_t rows,
                                             const uint32_t* v, float factor, uint32_t lane) {
    using T = typename MicroType<DT>::T;
    const uint32_t odd = lane & 1, first = row & ~1u;    // the token of two, and the first of the two rows, that this lane stores
    T* at = reinterpret_cast<T*>(y) + uint64_t(token + odd) * ld_y + first;
    const bool whole = (ld_y & 1) == 0 && token + 16 <= tokens && (row | 31) < rows;   // the same for the whole warp
#pragma unroll
    for (int j = 0; j < 16; j += 2) {
        const float a = __uint_as_float(v[j]) * factor, b = __uint_as_float(v[j + 1]) * factor;
        const float theirs = __shfl_xor_sync(0xFFFFFFFFu, odd ? a : b, 1);
        const float low = odd ? theirs : a, high = odd ? b : theirs;
        if (whole) {
            *reinterpret_cast<uint32_t*>(at) = MicroType<DT>::pack(low, high);
        } else if (token + j + odd < tokens) {
            if (first < rows) at[0] = MicroType<DT>::one(low);
            if (first + 1 < rows) at[1] = MicroType<DT>::one(high);
        }
        at += 2 * ld_y;
    }
}

#endif  // __CUDACC__

}  // namespace enec
