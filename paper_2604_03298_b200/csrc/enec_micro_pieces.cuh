// Products of a few columns with microscaled weights: what the product for few tokens and the expert layer share.
//
// Such a product reads every weight once and should be bound by that. Bringing the weights back costs more: two values take a conversion
// and most of an extraction, and with all that belongs to them (mma.m16n8k16, scales, copies) a weight took so many issue slots that 8
// tokens x 4096 x 14336 ran at 1.5 TB/s. So the weights stay as they are, and the columns are brought to the weights' format:
//
//   x = sum over p < 8 of d_p 8^-p 2^s, d_p in -4 .. 3
//
// for 32 neighbouring values with one s: balanced octal digits, all of which E2M1 has exactly, so every digit is a column of its own
// in the 4-bit product with block scales (tcgen05.mma, kind::mxf4), its scale 2^(s - 3p). A column then costs eight columns of an
// instruction that is far from being the bound: a record of 128 x 256 weights arrives every 750 clocks at HBM's rate, and 16 tokens
// (128 columns) take 260. The products of digits and weights are exact; the eight sums are added in fp32, the smallest first.
//
// What x loses: it is rounded to 2^-22 of the largest of its 32 neighbours, whatever weight that one meets (all bits of a bf16 value down to
// 2^-14 of the largest, of an fp16 value down to 2^-11). A NaN or an infinity makes its column NaN.
//
// A CTA takes tasks: 128 rows (a row tile of a matrix) x a range of records of columns. One warp copies records in bulk into a ring, as
// far ahead as the ring is long; one issues the matrix instructions, with two sets of sums in turn; sixteen make the digits and take
// the results of one task while the next one's products run. Not so in lockstep, where the CTAs of a cluster join their sums behind every
// task: there all warps meet, and no record of the next task is asked for before.
#pragma once

#include "enec_micro_mma.cuh"

namespace enec {

constexpr uint32_t kPieces = 8;
constexpr uint32_t kPieceTokens = 16;        // columns of x that a CTA takes: 128 of the accumulator
constexpr uint32_t kPieceMostStages = 8;
constexpr uint32_t kPieceBatches = 16;       // in which a group's digits are announced to the matrix instructions, at most
constexpr uint32_t kPieceWorkers = 16;       // warps
constexpr uint32_t kPieceThreads = (2 + kPieceWorkers) * 32;
constexpr uint32_t kPieceTmem = 512;         // columns: two sets of 128 sums, 16 of scales for each stage

__host__ __device__ constexpr uint32_t piece_columns(uint32_t tokens) { return (tokens * kPieces + 15) / 16 * 16; }
// A record's digits: rows of 128 bytes as a matrix operand, and 1024 bytes of scales.
__host__ __device__ constexpr uint32_t piece_record_bytes(uint32_t tokens) { return piece_columns(tokens) * 128 + 1024; }

#ifdef __CUDACC__

struct PieceShared {
    uint64_t full[kPieceMostStages], empty[kPieceMostStages], staged[kPieceBatches], done[2], drained[2];
    uint32_t tmem;
    volatile int failed;
};

// Rows 128 `row_tile` .. of a matrix whose records begin at `records`, columns in records first .. first + count - 1.
struct PieceTask {
    const uint8_t* records;
    uint32_t first, count;
    uint32_t group;        // tasks of the same group have the same records and use the same digits
    uint32_t n;            // columns of x, a group's
};

__device__ __forceinline__ void piece_setup(PieceShared& sh, uint32_t stages) {
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < stages; ++i) mbar_init(sh.full + i, 1), mbar_init(sh.empty + i, 1);
        for (uint32_t i = 0; i < kPieceBatches; ++i) mbar_init(sh.staged + i, kPieceWorkers);
        for (uint32_t i = 0; i < 2; ++i) mbar_init(sh.done + i, 1), mbar_init(sh.drained + i, kPieceWorkers);
        mbar_fence_init();
        sh.failed = 0;
    }
    if (threadIdx.x >> 5 == 1) tmem_alloc(&sh.tmem, kPieceTmem);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
}

// Eight values of a block (a quarter of it; the quarters are four neighbouring lanes) to eight words of eight digits' codes, digit p of the
// eight in word p; returns the scale byte of digit 0 (digit p's is 3p less), 255 where the block holds a NaN or an infinity.
__device__ __forceinline__ uint32_t make_digits(const float* x, uint32_t* words) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    // the largest magnitude goes to 2^21 .. 2^22 of 8 octal digits, whose largest is 3 (8^8 - 1) / 7 > 2^22; one digit's worth of the first
    // is 8^7 = 2^21, so the first scale is the largest's power of two
    const uint32_t field = min(max(top >> 23, 22u), 254u);            // below: the factor stays, and with it the absolute error
    const float factor = __uint_as_float((127 + 21 + 127 - field) << 23);
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // 1.5 x 2^23 + X, X rounded to a whole number; then X + 4 (8^8 - 1) / 7, whose octal digits are d + 4
        uint32_t o = __float_as_uint(fmaf(x[i], factor, 12582912.f)) - 0x4B400000u + 044444444u;
        // three bits each to four bits each
        o = (o & 0x00000FFFu) | ((o & 0x00FFF000u) << 4);
        o = (o & 0x003F003Fu) | ((o & 0x0FC00FC0u) << 2);
        o = (o & 0x07070707u) | ((o & 0x38383838u) << 1);
        // d + 4 -> the code of d: four nibbles choose among eight bytes
        const uint32_t a = prmt(0x0A0C0D0Eu, 0x05040200u, o), b = prmt(0x0A0C0D0Eu, 0x05040200u, o >> 16);
        v[i] = prmt(a | (a >> 4), b | (b >> 4), 0x6420);
    }
    // 8 x 8 nibbles: from a word per value to a word per digit; digit 0 is the highest nibble
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const uint32_t a = v[i], b = v[i + 1];
        v[i] = select_bits(0x0F0F0F0Fu, a, b << 4);              // nibble 2j: values i, i + 1 of digits 7 - 2j
        v[i + 1] = select_bits(0x0F0F0F0Fu, a >> 4, b);          // of digits 6 - 2j
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        // bytes 0 .. 3 of v[i], v[i + 2], v[i + 4], v[i + 6] are digits 7 - i, 5 - i, 3 - i, 1 - i of two values each
        const uint32_t lo0 = prmt(v[i], v[i + 2], 0x5140), lo1 = prmt(v[i + 4], v[i + 6], 0x5140);
        const uint32_t hi0 = prmt(v[i], v[i + 2], 0x7362), hi1 = prmt(v[i + 4], v[i + 6], 0x7362);
        words[7 - i] = prmt(lo0, lo1, 0x5410);
        words[5 - i] = prmt(lo0, lo1, 0x7632);
        words[3 - i] = prmt(hi0, hi1, 0x5410);
        words[1 - i] = prmt(hi0, hi1, 0x7632);
    }
    return top >= 0x7F800000u ? 255u : field;
}

// One warp: the digits of a column's 256 values of one record (eight a lane) to the operand and its scales.
__device__ __forceinline__ void put_digits(const float* x, uint32_t column, uint32_t record, uint32_t columns16, uint32_t lane) {
    uint32_t words[8];
    const uint32_t byte = make_digits(x, words);
    const uint32_t chunk = lane >> 2, part = lane & 3;
    const uint32_t row = record + column * kPieces * 128 + part * 4;
#pragma unroll
    for (uint32_t p = 0; p < kPieces; ++p) sts32(row + p * 128 + ((chunk ^ p) << 4), byte == 255 ? 0u : words[p]);
    // each lane of a block stores two of the eight scales
    const uint32_t scales = record + columns16 * 128 + (chunk >> 2) * 512 + (chunk & 3);
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t p = 2 * part + i, c = column * kPieces + p;
        const uint32_t scale = byte == 255 ? 255u : byte > 3 * p ? byte - 3 * p : 0u;
        asm volatile("st.shared.u8 [%0], %1;" ::"r"(scales + (c & 31) * 16 + (c >> 5) * 4), "r"(scale) : "memory");
    }
}

// A group's records x columns are staged in sweeps, two by every worker warp (their loads are on the way together), and announced in
// batches of sweeps, so that the products of the first records run while the last ones' digits are made.
struct PieceSweeps {
    uint32_t total, per_batch, batches, reciprocal;
    __device__ __forceinline__ PieceSweeps(uint32_t count, uint32_t n) {
        total = count * n;
        const uint32_t sweeps = (total + 2 * kPieceWorkers - 1) / (2 * kPieceWorkers);
        per_batch = (sweeps + kPieceBatches - 1) / kPieceBatches;
        batches = per_batch ? (sweeps + per_batch - 1) / per_batch : 0;
        reciprocal = 65536 / n + 1;   // i * reciprocal >> 16 = i / n below 65536 / n, far more than shared memory holds
    }
    __device__ __forceinline__ uint32_t batch_of(uint32_t record, uint32_t n) const { return ((record + 1) * n - 1) / (2 * kPieceWorkers) / per_batch; }
};
template <class Values>
__device__ __forceinline__ void stage_digits(PieceShared& sh, uint32_t worker, uint32_t lane, const PieceTask& task, uint32_t at, Values values) {
    const uint32_t n = task.n, columns = piece_columns(n), record_bytes = piece_record_bytes(n);
    const PieceSweeps sweeps(task.count, n);
    for (uint32_t batch = 0; batch < sweeps.batches; ++batch) {
        for (uint32_t s = 0; s < sweeps.per_batch; ++s) {
            const uint32_t first = (batch * sweeps.per_batch + s) * 2 * kPieceWorkers + worker;
            float x[2][8];
            uint32_t record[2], column[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t i = first + j * kPieceWorkers;
                record[j] = i * sweeps.reciprocal >> 16;
                column[j] = i - record[j] * n;
                if (i < sweeps.total) values(column[j], (task.first + record[j]) * kMicroCols + 8 * lane, x[j]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (first + j * kPieceWorkers < sweeps.total) put_digits(x[j], column[j], at + record[j] * record_bytes, columns, lane);
        }
        fence_async_shared();
        warp_arrive(sh.staged + batch);
    }
}

// The sum of a column's eight digits for this lane's row.
__device__ __forceinline__ float take_sum(uint32_t tmem, uint32_t column) {
    uint32_t v[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(tmem + column * kPieces));
    tmem_load_wait();
    float sum = 0.f;
#pragma unroll
    for (int p = kPieces - 1; p >= 0; --p) sum += __uint_as_float(v[p]);
    return sum;
}

// All roles of a CTA over its tasks. tasks: where the first one is, with get() and next(); every role walks a copy. values(c, col, x): by
// the workers, eight values of a group's column c from `col` on. take(i, tmem, ok): by the workers, takes the sums from their lanes of
// tensor memory; where not ok, a wait has run out and they are nothing. after(i, ok): by the workers, once the sums' place is free
// again. meet(i): by all threads behind every task where `lockstep`. smem: the ring, then the digits. cols: of the matrices.
template <class Tasks, class Values, class Take, class After, class Meet>
__device__ __forceinline__ void piece_products(PieceShared& sh, uint8_t* smem, uint32_t stages, uint32_t n_tasks, uint32_t cols, Tasks tasks,
                                               Values values, Take take, After after, bool lockstep, Meet meet) {
    const uint32_t warp = threadIdx.x >> 5;
    const uint32_t ring = smem_u32(smem), digits = ring + stages * kMicroRecordBytes;
    const uint32_t tmem = sh.tmem;
    const uint32_t leader = elected();
    if (warp == 0) {
        uint32_t asked = 0, slot = 0, phase = 0;
        for (uint32_t i = 0; i < n_tasks; ++i, tasks.next()) {
            const PieceTask task = tasks.get();
            for (uint32_t k = 0; k < task.count; ++k) {
                if (asked >= stages && !warp_wait(sh.empty + slot, phase ^ 1, &sh.failed)) {
                    sh.failed = 1;
                    break;
                }
                if (leader) {
                    mbar_expect_tx(sh.full + slot, kMicroRecordBytes);
                    bulk_g2s(smem + slot * kMicroRecordBytes, task.records + uint64_t(task.first + k) * kMicroRecordBytes, kMicroRecordBytes,
                             sh.full + slot);
                }
                ++asked;
                if (++slot == stages) slot = 0, phase ^= 1;
            }
            if (lockstep) meet(i);
        }
        // nothing may be in flight when the CTA ends
        for (uint32_t k = asked > stages ? asked - stages : 0; k < asked; ++k) mbar_wait_bounded(sh.full + k % stages, (k / stages) & 1);
    } else if (warp == 1) {
        const uint64_t ring_desc = operand_desc(ring), ring_scales_desc = scale_desc(ring + kMicroElemBytes);
        const uint64_t digits_desc = operand_desc(digits), digit_scales_desc = scale_desc(digits);
        uint32_t group = 0xFFFFFFFFu, slot = 0, phase = 0;
        uint32_t full_there = mbar_complete(sh.full, 0);
        uint32_t flipped = 0;   // bit b: announcements of batch b so far, mod 2
        volatile int never = 0;
        for (uint32_t i = 0; i < n_tasks; ++i, tasks.next()) {
            const PieceTask task = tasks.get();
            const uint32_t columns = piece_columns(task.n);
            const PieceSweeps sweeps(task.count, task.n);
            const bool begins = task.group != group;
            group = task.group;
            uint32_t known = begins ? 0 : sweeps.batches;   // batches that have been waited for
            const uint32_t set = i & 1, sums = tmem + set * (kPieceTokens * kPieces);
            if (i >= 2 && !suspended_wait(sh.drained + set, ((i >> 1) - 1) & 1, &sh.failed)) sh.failed = 1;
            tcgen05_fence_after();
            const uint32_t idesc = scaled_idesc(columns), record16 = columns * 8 + 64;   // a record's digits in units of 16 bytes
            uint64_t b = digits_desc, bs = digit_scales_desc + columns * 8;
            for (uint32_t k = 0; k < task.count && !sh.failed; ++k) {
                const uint32_t now = slot;
                bool there = full_there || suspended_wait(sh.full + slot, phase, &sh.failed);
                if (++slot == stages) slot = 0, phase ^= 1;
                full_there = mbar_complete(sh.full + slot, phase);
                if (known < sweeps.batches) {
                    const uint32_t batch = sweeps.batch_of(k, task.n);
                    for (; there && known <= batch; ++known) there = suspended_wait(sh.staged + known, flipped >> known & 1, &sh.failed);
                }
                if (!there) {
                    sh.failed = 1;
                    break;
                }
                tcgen05_fence_after();
                const uint64_t a = ring_desc + now * (kMicroRecordBytes / 16), as = ring_scales_desc + now * (kMicroRecordBytes / 16);
                const uint32_t to = tmem + 2 * kPieceTokens * kPieces + now * 16;
                copy_scales(leader, to, as);
                copy_scales(leader, to + 8, bs);
                copy_scales(leader, to + 4, as + 32);
                copy_scales(leader, to + 12, bs + 32);
                const uint32_t steps = (cols - (task.first + k) * kMicroCols + 63) / 64;
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) {
                    const uint32_t h = q >> 1, pair = (q & 1) * 2;
                    mma_scaled(q < steps ? leader : 0, sums, a + q * 2, b + q * 2, idesc | pair << 4 | pair << 29, to + h * 4, to + 8 + h * 4,
                               k > 0 || q > 0);
                }
                tcgen05_commit(leader, sh.empty + now);
                b += record16, bs += record16;
            }
            if (begins) flipped ^= (1u << sweeps.batches) - 1;
            tcgen05_commit(leader, sh.done + set);
            __syncwarp();
            if (lockstep) meet(i);
        }
        // no instruction may be under way when tensor memory is given back
        for (uint32_t i = n_tasks > 2 ? n_tasks - 2 : 0; i < n_tasks; ++i) suspended_wait(sh.done + (i & 1), (i >> 1) & 1, &never);
        __syncwarp();
    } else {
        uint32_t group = 0xFFFFFFFFu;
        for (uint32_t i = 0; i < n_tasks; ++i, tasks.next()) {
            const PieceTask task = tasks.get();
            if (task.group != group) {
                group = task.group;
                stage_digits(sh, warp - 2, threadIdx.x & 31, task, digits, values);
            }
            const uint32_t set = i & 1;
            wait_or_fail(sh.done + set, (i >> 1) & 1, &sh.failed);
            tcgen05_fence_after();
            const bool ok = !sh.failed;   // lane by lane: nothing but stores to global memory may depend on it
            take(i, tmem + set * (kPieceTokens * kPieces) + ((warp & 3) * 32 << 16), ok);
            tcgen05_fence_before();
            warp_arrive(sh.drained + set);
            after(i, ok);
            if (lockstep) meet(i);
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    if (warp == 1) tmem_free(tmem, kPieceTmem);
}

#endif  // __CUDACC__

}  // namespace enec
