// y = x W^T for many tokens, W a microscaled stream, x of 16 bits: tcgen05.mma (kind::f16) on weights that are brought back on the way.
//
// Lanes of the accumulator are rows of W, its columns tokens: 256 (two accumulators) or 128 rows x up to 256 tokens a CTA. Of 64 columns
// (a step) the tensor cores take 1024 clocks at 256 x 256. Meanwhile sixteen warps turn 16384 codes into 16-bit values in shared
// memory (5 instructions a pair, some 370 clocks of the SM's issue slots), and 32 KB of x come by a tensor map, 32 bytes a clock from L2;
// tiles of 128 x 256 would need twice that. Raw records are copied in bulk; a
// thread takes its share of a record to registers at once, so that one record's room is enough.
//
// bf16: a code's value times its scale is exact in bf16 over the whole range of scales. fp16: it would not be, so a row's values are held
// times 2^(13 - largest scale exponent of the row), and the sum is scaled back. fp16 has the values of blocks down to 2^-36 of the
// row's largest so (3 x 2^14 to 2^-24). Blocks that cannot add up to 2^-37, far below fp16's last place, are not counted; rows
// whose other blocks lie further apart take their sums again, in fp32 on the codes themselves (wide_row_sum): 2048 tokens x 4096 x 4096
// take 62 us without such rows, 530 us with one in 128, 20 ms with nothing else.
//
// Where the tiles would not fill the SMs, a cluster of CTAs shares the columns: each leaves its sums in its shared memory and adds
// up a part of the tokens, in the order of the CTAs.
#include "enec_micro_mma.cuh"

#include <cooperative_groups.h>
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>

#include "enec_micro_launch.cuh"

namespace enec {
namespace {

// Stages of x and of raw records at most, as many as fit.
constexpr uint32_t kMostB = 12, kMostRaw = 4;

// Who does what. 256 rows are bound by shared memory and the tensor cores; 128 rows with fewer tokens by how long a step takes one warp from
// its first wait to its last arrival, some 900 clocks both for the warp that issues and for the eight that bring weights back. So
// there two warps issue, each every other step to sums of its own that are added at the end, and four groups of warps bring back
// every fourth step each, a thread a whole row of it. Either alone gains nothing; both: 64 tokens x 14336 x 4096 32.7 -> 23.4 us, four
// issuing warps the same. Where x comes through registers a thread needs 80 of them, which leaves room for two groups: 128
// tokens x 1411 x 2055, 12 steps a CTA, took 20 us so, with four groups 27.
template <int MT, bool MAP>
struct ManyShape {
    static constexpr uint32_t kIssuers = MT == 1 ? 2 : 1;
    static constexpr uint32_t kX = MAP ? 1 : 8;                          // warps for x
    static constexpr uint32_t kParts = MT == 1 ? 1 : 2;                  // threads that share a row of a step
    static constexpr uint32_t kGroups = MT == 2 ? 1 : MAP ? 4 : 2;       // of warps for the weights
    static constexpr uint32_t kWeights = 128 * MT * kParts * kGroups;    // threads
    static constexpr uint32_t kFirstX = 1 + kIssuers, kFirstW = kFirstX + kX, kThreads = kFirstW * 32 + kWeights;
    // Stages of weights. A barrier answers for its last phase alone, and a warp that asks for a stage's next use must not be told of the use
    // before: with several issuers or groups a stage, of weights or of x, always belongs to the same ones. A constant: counted at
    // run time the issuing warp is slower by a tenth of the whole at 256 rows.
    static constexpr uint32_t kStagesA = MT == 1 ? 4 : 5, kLeastB = MT == 1 ? 4 : 3;
    static_assert(MT == 2 || (kStagesA % kIssuers == 0 && kStagesA % kGroups == 0 && kLeastB % kIssuers == 0), "");
};

constexpr uint32_t kManyMostTokens = 256;
constexpr uint32_t kFp16Up = 13, kFp16Span = 36;   // a row's largest scale becomes 2^13; the smallest that fp16 has all values of, below it

struct ManyJob {
    const uint8_t* x;
    uint64_t ld_x;
    const uint8_t* w;
    MicroShape s;
    uint8_t* y;
    uint64_t ld_y;
    uint32_t tokens;
    uint32_t tile_tokens;    // a multiple of 16
    uint32_t row_tiles;      // tiles along the rows
    uint32_t cluster;        // CTAs that share a tile's columns
    uint32_t share;          // records of columns each takes
    uint32_t stages_b, stages_raw;
    CUtensorMap map;         // of x, where its rows begin on 16-byte boundaries
    int* status;
};

template <int MT, bool MAP>
uint32_t many_bytes(const ManyJob& job) {
    return job.stages_raw * MT * kMicroRecordBytes + ManyShape<MT, MAP>::kStagesA * 16384 + job.stages_b * job.tile_tokens * 128 + 1024;
}

// 64 columns x tile_tokens rows of x from (column, token) on; zeros behind the matrix.
__device__ __forceinline__ void tile_g2s(uint32_t dst, const CUtensorMap* map, uint32_t column, uint32_t token, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                 "r"(column), "r"(token), "r"(smem_u32(bar))
                 : "memory");
}

__device__ __forceinline__ uint32_t bf16_times(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmul2(reinterpret_cast<const __nv_bfloat162&>(a), reinterpret_cast<const __nv_bfloat162&>(b));
    return reinterpret_cast<const uint32_t&>(r);
}
__device__ __forceinline__ uint32_t fp16_times(uint32_t a, uint32_t b) {
    const __half2 r = __hmul2(reinterpret_cast<const __half2&>(a), reinterpret_cast<const __half2&>(b));
    return reinterpret_cast<const uint32_t&>(r);
}

// What 32 codes of a scale byte are multiplied with, in both halves of a word. bf16: the values come times 2^-112 (see to_values), so
// 2^(byte - 15); scales above 2^15 need a second factor (bf16_more). fp16: 2^(13 + byte - top), 0 for scales that are not counted. 255 is
// not a number.
__device__ __forceinline__ uint32_t bf16_factor(uint32_t byte) { return (byte == 255 ? 0x7FC0u : (min(byte, 142u) + 112) << 7) * 0x10001u; }
__device__ __forceinline__ uint32_t bf16_more(uint32_t byte) { return (byte > 142 && byte < 255 ? (byte - 142 + 127) << 7 : 0x3F80u) * 0x10001u; }
__device__ __forceinline__ uint32_t fp16_factor(uint32_t byte, uint32_t top) {
    const uint32_t below = top - byte;   // 2^32 less something where the whole row is not counted
    return (byte == 255 ? 0x7E00u : below < 15 + kFp16Up ? (15 + kFp16Up - below) << 10 : below < 25 + kFp16Up ? 0x400u >> (below - 14 - kFp16Up) : 0u) * 0x10001u;
}
// Eight codes times a factor. fp16 holds a code's value with its exponent field in 14 .. 17 and at most one mantissa bit; for bf16 the same
// fields three bits further down are the value times 2^-112.
template <int DT>
__device__ __forceinline__ uint4 to_values(uint32_t codes, uint32_t factor) {
    uint4 h = e2m1_values(codes);
    if constexpr (DT == ENEC_FP16) {
        return make_uint4(fp16_times(h.x, factor), fp16_times(h.y, factor), fp16_times(h.z, factor), fp16_times(h.w, factor));
    } else {
        h.x = select_bits(0x80008000u, h.x, (h.x >> 3) & 0x0FFF0FFFu);
        h.y = select_bits(0x80008000u, h.y, (h.y >> 3) & 0x0FFF0FFFu);
        h.z = select_bits(0x80008000u, h.z, (h.z >> 3) & 0x0FFF0FFFu);
        h.w = select_bits(0x80008000u, h.w, (h.w >> 3) & 0x0FFF0FFFu);
        return make_uint4(bf16_times(h.x, factor), bf16_times(h.y, factor), bf16_times(h.z, factor), bf16_times(h.w, factor));
    }
}

// A warp: sums of one row of weights and 16 tokens, by lanes t and t + 16 that of token t. Every second block a lane: the sum of codes times
// values, then times the block's scale. rec: the first record; row: in it; at: where the first token's values begin; valid_tokens: rows
// of x that exist. Out of line: no ordinary weights come here, and the registers are the main loop's.
__device__ __noinline__ float wide_row_sum(const uint8_t* rec, uint32_t row, uint32_t columns, const uint8_t* at, uint64_t ld_x, uint32_t valid_tokens) {
    const uint32_t lane = threadIdx.x & 31, t = lane & 15;
    const uint8_t* x = at + uint64_t(t) * ld_x * 2;
    float sum = 0.f;
    for (uint32_t c = lane >> 4; c * kMicroBlock < columns; c += 2) {
        const uint8_t* r = rec + uint64_t(c >> 3) * kMicroRecordBytes;
        const uint4 codes = __ldg(reinterpret_cast<const uint4*>(r + row * 128 + (((c & 7) ^ (row & 7)) << 4)));
        const uint32_t scale = __ldg(r + kMicroElemBytes + (c >> 2 & 1) * 512 + (row & 31) * 16 + (row >> 5) * 4 + (c & 3));
        const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
        float part = 0.f;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
            const uint32_t col = c * kMicroBlock + e * 8;
            uint32_t words[4];
            load_eight<ENEC_FP16>(x + uint64_t(col) * 2, t < valid_tokens && col < columns ? int(min(columns - col, 8u)) : 0, words);
            const uint4 h = e2m1_values(w[e]);
            const uint32_t hw[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const float2 a = MicroType<ENEC_FP16>::unpack(hw[i]), b = MicroType<ENEC_FP16>::unpack(words[i]);
                part = fmaf(a.x, b.x, part);
                part = fmaf(a.y, b.y, part);
            }
        }
        sum = fmaf(part, micro_scale(scale), sum);
    }
    return sum + __shfl_xor_sync(0xFFFFFFFFu, sum, 16);
}

template <int DT, int MT, bool MAP>
__global__ void __launch_bounds__(ManyShape<MT, MAP>::kThreads, 1) enec_micro_many_kernel(const __grid_constant__ ManyJob job) {
    using Shape = ManyShape<MT, MAP>;
    constexpr uint32_t kStagesA = Shape::kStagesA;
    extern __shared__ uint8_t raw_shared[];
    __shared__ uint64_t raw_full[kMostRaw], raw_empty[kMostRaw], full_a[kStagesA], empty_a[kStagesA], full_b[kMostB], empty_b[kMostB], done;
    __shared__ uint32_t tmem_at;
    __shared__ volatile int failed;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = raw_shared + ((1024 - (smem_u32(raw_shared) & 1023)) & 1023);
    const uint32_t n = job.tile_tokens;
    constexpr uint32_t kFirstX = Shape::kFirstX, kFirstW = Shape::kFirstW, kGroups = Shape::kGroups, kParts = Shape::kParts, kIssuers = Shape::kIssuers;
    constexpr uint32_t kMine = 4 / kGroups, kEach = 2 / kParts;   // steps of a record, scales of a step's row
    uint32_t tmem_columns = 32;
    while (tmem_columns < 2 * n) tmem_columns *= 2;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < job.stages_raw; ++i) mbar_init(raw_full + i, 1), mbar_init(raw_empty + i, Shape::kWeights / 32);
        for (uint32_t i = 0; i < kStagesA; ++i) mbar_init(full_a + i, 4 * kParts), mbar_init(empty_a + i, 1);
        for (uint32_t i = 0; i < job.stages_b; ++i) mbar_init(full_b + i, Shape::kX), mbar_init(empty_b + i, 1);
        mbar_init(&done, kIssuers);
        mbar_fence_init();
        failed = 0;
    }
    if (warp == 1) tmem_alloc(&tmem_at, tmem_columns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_at;
    pdl_wait();
    pdl_launch_dependents();

    const uint32_t rank = job.cluster > 1 ? blockIdx.x % job.cluster : 0, tile = blockIdx.x / job.cluster;
    const uint32_t row_tile = tile % job.row_tiles * MT, token0 = tile / job.row_tiles * n;
    const uint32_t mt = min(uint32_t(MT), job.s.row_tiles - row_tile);
    const uint32_t k0 = min(rank * job.share, job.s.col_tiles), k1 = min(k0 + job.share, job.s.col_tiles);
    const uint32_t records = k1 - k0;
    const uint32_t columns = min(job.s.cols, k1 * kMicroCols) - min(job.s.cols, k0 * kMicroCols);
    const uint32_t steps = (columns + 63) / 64;
    const uint64_t strip = uint64_t(job.s.col_tiles) * kMicroRecordBytes;
    const uint8_t* wr = job.w + kMicroHeaderBytes + row_tile * strip + uint64_t(k0) * kMicroRecordBytes;
    uint8_t* a_ring = smem;
    uint8_t* b_ring = a_ring + kStagesA * 16384;
    uint8_t* raw = b_ring + job.stages_b * n * 128;
    const bool good = micro_header_ok(job.w, job.s);

    const uint32_t leader = elected();
    if (warp == 0) {
        uint32_t k = 0, s = 0, phase = 1;
        for (; k < records; ++k) {
            if (k >= job.stages_raw && !warp_wait(raw_empty + s, phase, &failed)) {
                failed = 1;
                break;
            }
            if (leader) {
                mbar_expect_tx(raw_full + s, mt * kMicroRecordBytes);
                for (uint32_t i = 0; i < mt; ++i)
                    bulk_g2s(raw + (s * MT + i) * kMicroRecordBytes, wr + i * strip + uint64_t(k) * kMicroRecordBytes, kMicroRecordBytes, raw_full + s);
            }
            if (++s == job.stages_raw) s = 0, phase ^= 1;
        }
        // nothing may be in flight when the CTA ends
        for (uint32_t i = k > job.stages_raw ? k - job.stages_raw : 0; i < k; ++i)
            mbar_wait_bounded(raw_full + i % job.stages_raw, (i / job.stages_raw) & 1);
    } else if (warp < kFirstX) {
        const uint32_t idesc = idesc_16bit(DT == ENEC_BF16, n), me = kIssuers == 1 ? 0 : warp - 1;
        const uint64_t a0 = operand_desc(smem_u32(a_ring)), b0 = operand_desc(smem_u32(b_ring));
        uint32_t slot = me, phase = 0, sb = me, phase_b = 0;
        uint32_t a_there = mbar_complete(full_a + slot, 0), b_there = mbar_complete(full_b + sb, 0);
        bool there = true;
        for (uint32_t j = me; j < steps && there; j += kIssuers) {
            const uint32_t sb_now = sb;
            const uint64_t b = b0 + sb * n * 8;
            there = b_there || suspended_wait(full_b + sb, phase_b, &failed);
            if ((sb += kIssuers) >= job.stages_b) sb -= job.stages_b, phase_b ^= 1;
            b_there = mbar_complete(full_b + sb, phase_b);
            for (uint32_t i = 0; i < mt && there; ++i) {
                const uint32_t now = slot;
                const uint64_t a = a0 + slot * 1024;
                there = a_there || suspended_wait(full_a + slot, phase, &failed);
                if ((slot += kIssuers) >= kStagesA) slot -= kStagesA, phase ^= 1;
                a_there = mbar_complete(full_a + slot, phase);
                if (!there) break;
                tcgen05_fence_after();
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) mma_16bit(leader, tmem + (me + i) * n, a + q * 2, b + q * 2, idesc, j > me || q > 0);
                tcgen05_commit(leader, empty_a + now);
            }
            if (there) tcgen05_commit(leader, empty_b + sb_now);
        }
        if (!there) failed = 1;
        tcgen05_commit(leader, &done);
        mbar_wait_bounded(&done, 0);   // no instruction may be under way when tensor memory is given back
        __syncwarp();
    } else if (warp < kFirstW) {
        // x: eight lanes a row of 64 columns
        const uint32_t me = threadIdx.x - kFirstX * 32, c = me & 7;
        uint32_t asked = 0, sb = 0, phase = 1;
        const uint32_t first_col = min(k0 * kMicroCols, job.s.cols);
        const uint8_t* from = job.x + (uint64_t(token0) * job.ld_x + first_col) * 2;
        if constexpr (MAP) {
            for (uint32_t j = 0; j < steps; ++j) {
                if (j >= job.stages_b && !warp_wait(empty_b + sb, phase, &failed)) {
                    failed = 1;
                    break;
                }
                if (leader) {
                    mbar_expect_tx(full_b + sb, n * 128);
                    tile_g2s(smem_u32(b_ring) + sb * n * 128, &job.map, first_col + j * 64, token0, full_b + sb);
                }
                asked = j + 1;
                if (++sb == job.stages_b) sb = 0, phase ^= 1;
            }
            // nothing may be in flight when the CTA ends
            for (uint32_t j = asked > job.stages_b ? asked - job.stages_b : 0; j < asked; ++j)
                mbar_wait_bounded(full_b + j % job.stages_b, (j / job.stages_b) & 1);
        } else {
            // rows that lie anywhere: through registers, 64 rows of a step at a time, the loads of three such batches on the way together
            constexpr uint32_t kAhead = 3;
            const uint32_t batches = (n + 63) / 64, all = steps * batches;
            EightLoaded<DT> v[kAhead][2];
            auto load = [&](EightLoaded<DT>* to, uint32_t batch) {
                const uint32_t j = batch / batches, col = j * 64 + c * 8, first = (batch - j * batches) * 64;
                const int valid = batch < all && col < columns ? int(min(columns - col, 8u)) : 0;
#pragma unroll
                for (uint32_t i = 0; i < 2; ++i) {
                    const uint32_t r = first + i * 32 + (me >> 3);
                    to[i].load(from + (uint64_t(r) * job.ld_x + col) * 2, r < n && token0 + r < job.tokens ? valid : 0);
                }
            };
#pragma unroll
            for (uint32_t a = 0; a < kAhead; ++a) load(v[a], a);
            for (uint32_t batch0 = 0; batch0 < all; batch0 += kAhead) {
#pragma unroll
                for (uint32_t a = 0; a < kAhead; ++a) {
                    const uint32_t batch = batch0 + a, j = batch / batches, part = batch - j * batches;
                    if (batch >= all) break;
                    if (part == 0 && j >= job.stages_b) wait_or_fail(empty_b + sb, phase, &failed);
#pragma unroll
                    for (uint32_t i = 0; i < 2; ++i) {
                        const uint32_t r = part * 64 + i * 32 + (me >> 3);
                        uint32_t w[4];
                        v[a][i].words(w);
                        if (r < n) sts128(smem_u32(b_ring) + sb * n * 128 + r * 128 + ((c ^ (r & 7)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
                    }
                    load(v[a], batch + kAhead);
                    if (part == batches - 1) {
                        fence_async_shared();
                        warp_arrive(full_b + sb);
                        if (++sb == job.stages_b) sb = 0, phase ^= 1;
                    }
                }
            }
        }
    } else {
        // the weights: thread (tile, half, row) brings back 32 of the 64 columns of a step
        const uint32_t me = threadIdx.x - kFirstW * 32, r = me & 127, half = MT == 2 ? me >> 7 & 1 : 0, i = MT == 2 ? me >> 8 : 0, group = MT == 2 ? 0 : me >> 7;
        const bool mine = i < mt;   // the same for a warp
        uint32_t top = 0;
        bool wide = false;
        if constexpr (DT == ENEC_FP16) {
            // The largest and the smallest of the row's scale bytes. 255 does not count, and neither do bytes up to 71 - log2 of the
            // columns, rounded up: such weights are below 2^2.6 2^(71 - 127) / columns and values of x below 2^16, so all of them
            // together are below 2^-37, where half of fp16's smallest step is 2^-25. (Blocks of zeros have the byte 0.)
            // Two bytes at a time, as (byte + 1) mod 256 + up: those that count become 256 and more, exclusive-or 256 less than the others.
            const uint32_t none = 71 - (32 - __clz(job.s.cols - 1)), up = (254 - none) * 0x10001u;
            const uint8_t* at = wr + i * strip + kMicroElemBytes + (r & 31) * 16 + (r >> 5) * 4;
            uint32_t high = 0, low = 0xFFFFFFFFu;
            if (mine) {
#pragma unroll 8
                for (uint32_t b = 0; b < 2 * records; ++b) {
                    const uint32_t four = __ldg(reinterpret_cast<const uint32_t*>(at + uint64_t(b >> 1) * kMicroRecordBytes + (b & 1) * 512));
#pragma unroll
                    for (uint32_t e = 0; e < 2; ++e) {
                        const uint32_t two = (((four >> (8 * e) & 0x00FF00FFu) + 0x00010001u) & 0x00FF00FFu) + up;
                        high = __vmaxu2(high, two);
                        low = __vminu2(low, two ^ 0x01000100u);
                    }
                }
            }
            high = max(high & 0xFFFF, high >> 16), low = min(low & 0xFFFF, low >> 16);
            if (high >= 256) {
                wide = high - 256 > low + kFp16Span;
                top = high - 255 + none;
            }
            top = max(top, kFp16Up);
        }
        const uint32_t a_base = smem_u32(a_ring) + r * 128;
        uint32_t place[4 * kEach];   // of the four chunks of eight values in the operand's row
#pragma unroll
        for (uint32_t e = 0; e < 4 * kEach; ++e) place[e] = ((4 * half + e) ^ (r & 7)) << 4;
        uint32_t s = 0, phase = 0, sa = MT == 1 ? group : i, phase_a = 1;
        for (uint32_t k = 0; k < records; ++k) {
            wait_or_fail(raw_full + s, phase, &failed);
            uint4 codes[kMine][kEach];
            uint2 scales = {};   // eight bytes
            const uint32_t rec = smem_u32(raw) + (s * MT + i) * kMicroRecordBytes;
            if (mine) {
#pragma unroll
                for (uint32_t p = 0; p < kMine; ++p)
#pragma unroll
                    for (uint32_t h = 0; h < kEach; ++h)
                        codes[p][h] = lds128(rec + r * 128 + (((2 * (p * kGroups + group) + half + h) ^ (r & 7)) << 4));
                const uint32_t at = rec + kMicroElemBytes + (r & 31) * 16 + (r >> 5) * 4;
                scales = make_uint2(lds32(at), lds32(at + 512));
            }
            warp_arrive(raw_empty + s);
            if (++s == job.stages_raw) s = 0, phase ^= 1;
            const uint32_t here = min(4u, steps - 4 * k);
#pragma unroll
            for (uint32_t p = 0; p < kMine; ++p) {
                const uint32_t q = p * kGroups + group;
                if (q >= here) break;
                if (mine) {
                    const uint32_t at = sa;
                    wait_or_fail(empty_a + at, phase_a, &failed);
                    const uint32_t dst = a_base + at * 16384, two = (q < 2 ? scales.x : scales.y) >> (16 * (q & 1));
#pragma unroll
                    for (uint32_t h = 0; h < kEach; ++h) {
                        const uint32_t byte = two >> (8 * (half + h)) & 255;
                        const uint32_t w[4] = {codes[p][h].x, codes[p][h].y, codes[p][h].z, codes[p][h].w};
                        const uint32_t factor = DT == ENEC_BF16 ? bf16_factor(byte) : fp16_factor(byte, top);
                        if (DT == ENEC_BF16 && __any_sync(0xFFFFFFFFu, byte > 142 && byte < 255)) {
                            const uint32_t more = bf16_more(byte);
#pragma unroll
                            for (uint32_t e = 0; e < 4; ++e) {
                                const uint4 v = to_values<DT>(w[e], factor);
                                sts128(dst + place[4 * h + e], make_uint4(bf16_times(v.x, more), bf16_times(v.y, more), bf16_times(v.z, more), bf16_times(v.w, more)));
                            }
                        } else {
#pragma unroll
                            for (uint32_t e = 0; e < 4; ++e) sts128(dst + place[4 * h + e], to_values<DT>(w[e], factor));
                        }
                    }
                    fence_async_shared();
                    warp_arrive(full_a + at);
                    if ((sa += MT == 1 ? kGroups : mt) >= kStagesA) sa -= kStagesA, phase_a ^= 1;
                }
            }
        }
        wait_or_fail(&done, 0, &failed);
        tcgen05_fence_after();
        // results: the warp's quarter of the lanes, every other 16 tokens of its tile
        const uint32_t quarter = warp & 3, row_in = quarter * 32 + lane, row = (row_tile + i) * kMicroRows + row_in;
        float factor = 1.f;
        uint32_t wide_rows = 0;   // of the warp's 32
        if constexpr (DT == ENEC_FP16) {
            // the rows' exponents change hands through shared memory that no operand uses any more
            uint16_t* tops = reinterpret_cast<uint16_t*>(smem);
            asm volatile("bar.sync 1, %0;" ::"n"(Shape::kWeights) : "memory");
            if (half == 0 && group == 0) tops[i * 128 + r] = uint16_t((top - kFp16Up) << 1 | uint32_t(wide));
            asm volatile("bar.sync 1, %0;" ::"n"(Shape::kWeights) : "memory");
            factor = micro_scale(tops[i * 128 + row_in] >> 1);
            wide_rows = __ballot_sync(0xFFFFFFFFu, good && row < job.s.rows && (tops[i * 128 + row_in] & 1));
            asm volatile("bar.sync 1, %0;" ::"n"(Shape::kWeights) : "memory");
        }
        if (!warp_failed(&failed) && steps > 0 && mine) {
            for (uint32_t c = (MT == 2 ? half : group) * 16; c < n; c += 16 * kGroups * kParts) {
                if (token0 + c >= job.tokens) break;
                uint32_t v[16];
                tmem_load16(tmem + (quarter * 32 << 16) + i * n + c, v);
                tmem_load_wait();
                for (uint32_t o = 1; MT == 1 && o < kIssuers && o < steps; ++o) {
                    uint32_t other[16];
                    tmem_load16(tmem + (quarter * 32 << 16) + o * n + c, other);
                    tmem_load_wait();
#pragma unroll
                    for (uint32_t e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) + __uint_as_float(other[e]));
                }
                if (MT == 1 && job.cluster > 1) {
                    float* sums = reinterpret_cast<float*>(smem);   // [token][row]
#pragma unroll
                    for (uint32_t e = 0; e < 16; ++e) sums[(c + e) * kMicroRows + row_in] = __uint_as_float(v[e]) * factor;
                } else if (good) {
                    store_tile16<DT>(job.y, job.ld_y, token0 + c, job.tokens, row, job.s.rows, v, factor, lane);
                }
                if constexpr (DT == ENEC_FP16) {
                    // over what this warp's lanes have just stored
                    if (wide_rows) __syncwarp();
                    for (uint32_t left = wide_rows; left; left &= left - 1) {
                        const uint32_t r_wide = quarter * 32 + __ffs(left) - 1, t = lane & 15;
                        const float sum = wide_row_sum(wr + i * strip, r_wide, columns, job.x + (uint64_t(token0 + c) * job.ld_x + k0 * kMicroCols) * 2,
                                                       job.ld_x, job.tokens - token0 - c);
                        if (lane >= 16) continue;
                        if (MT == 1 && job.cluster > 1) reinterpret_cast<float*>(smem)[(c + t) * kMicroRows + r_wide] = sum;
                        else if (good && token0 + c + t < job.tokens)
                            reinterpret_cast<__half*>(job.y)[uint64_t(token0 + c + t) * job.ld_y + row - row_in + r_wide] = __float2half_rn(sum);
                    }
                }
            }
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    if (threadIdx.x == 0) {
        if (failed) report(job.status, ENEC_ERR_TIMEOUT);
        else if (!good && blockIdx.x == 0) report(job.status, ENEC_ERR_BAD_STREAM);
    }
    if (warp == 1) tmem_free(tmem, tmem_columns);
    if constexpr (MT == 1) {
        if (job.cluster > 1) {
            // CTAs that have columns have left their sums; each adds up every cluster-th group of 4 tokens
            using T = typename MicroType<DT>::T;
            auto cluster = cooperative_groups::this_cluster();
            cluster.sync();
            const uint32_t with = (job.s.col_tiles + job.share - 1) / job.share;
            const uint32_t row_in = threadIdx.x & 127;
            const uint32_t row = row_tile * kMicroRows + row_in;
            if (threadIdx.x < 512 && good && !failed && row < job.s.rows) {
#pragma unroll 2
                for (uint32_t t = (threadIdx.x >> 7) * job.cluster + rank; t < n && token0 + t < job.tokens; t += 4 * job.cluster) {
                    float v = 0.f;
#pragma unroll
                    for (uint32_t k = 0; k < 8; ++k)
                        if (k < with) v += cluster.map_shared_rank(reinterpret_cast<float*>(smem), k)[t * kMicroRows + row_in];
                    reinterpret_cast<T*>(job.y)[uint64_t(token0 + t) * job.ld_y + row] = MicroType<DT>::one(v);
                }
            }
            cluster.sync();   // no CTA ends while its sums are read
        }
    }
}

// The columns of a tile for at most `most` CTAs, two records or more each: 4 tiles x 2 records take 7 us without and 8.5 us with two CTAs.
void share_columns(ManyJob& job, uint32_t most) {
    job.share = (job.s.col_tiles + std::max(most, 1u) - 1) / std::max(most, 1u);
    job.share = std::max(job.share, std::min(job.s.col_tiles, 2u));
    job.cluster = job.share ? (job.s.col_tiles + job.share - 1) / job.share : 1;
}

template <int DT, int MT, bool MAP>
enec_status launch_many(ManyJob job, uint32_t tiles, const MicroDevice& dev, cudaStream_t stream) {
    static std::atomic<uint64_t> allowed{0};
    if (!allow_shared(allowed, dev, enec_micro_many_kernel<DT, MT, MAP>, kFewMostShared)) return ENEC_ERR_CUDA;
    // x first, then raw records: a stage of x comes from L2 a step at a time, a record is taken to registers at once
    using Shape = ManyShape<MT, MAP>;
    job.stages_b = Shape::kLeastB, job.stages_raw = 1;
    const auto grow = [&](uint32_t ManyJob::*stages, uint32_t by, uint32_t most) {
        for (ManyJob more = job; (more.*stages += by) <= most && many_bytes<MT, MAP>(more) <= kFewMostShared;) job = more;
    };
    grow(&ManyJob::stages_raw, 1, 2);
    grow(&ManyJob::stages_b, Shape::kIssuers, 6);
    grow(&ManyJob::stages_raw, 1, 3);
    grow(&ManyJob::stages_b, Shape::kIssuers, kMostB);
    grow(&ManyJob::stages_raw, 1, kMostRaw);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * job.cluster);
    cfg.blockDim = dim3(Shape::kThreads);
    cfg.dynamicSmemBytes = many_bytes<MT, MAP>(job);
    if (job.cluster > 1 && cfg.dynamicSmemBytes < job.tile_tokens * kMicroRows * 4 + 1024) cfg.dynamicSmemBytes = job.tile_tokens * kMicroRows * 4 + 1024;
    const uint32_t least = 2 * job.tile_tokens > 256 ? kTmemAloneShared : kTmemHalfShared;
    if (cfg.dynamicSmemBytes < least) cfg.dynamicSmemBytes = least;
    if (MT == 1 && job.cluster > 1) {
        // clusters that would have to wait for others cost more than larger shares: of 8 CTAs 15 run at the same time, and 17 tokens x 2048 x
        // 4096 (16 tiles) took 16.4 us with 16 of them, 10.2 us with clusters of 4
        uint32_t places = 0;
        do {
            if (places) share_columns(job, job.cluster / 2);
            if (job.cluster > 1 && !resident_clusters(enec_micro_many_kernel<DT, MT, MAP>, dev, job.cluster, Shape::kThreads, uint32_t(cfg.dynamicSmemBytes), places))
                return ENEC_ERR_CUDA;
        } while (job.cluster > 1 && tiles > places);
        cfg.gridDim = dim3(tiles * job.cluster);
    }
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = job.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = job.cluster > 1 ? 2 : 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, enec_micro_many_kernel<DT, MT, MAP>, job);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

}  // namespace

// The driver's encoder of tensor maps, found once; null where there is none.
PFN_cuTensorMapEncodeTiled_v12000 map_encoder() {
    static const PFN_cuTensorMapEncodeTiled_v12000 encode = []() -> PFN_cuTensorMapEncodeTiled_v12000 {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
    }();
    return encode;
}

enec_status micro_many(const MicroProduct& p, const MicroDevice& dev, cudaStream_t stream) {
    ManyJob job;
    job.x = p.x;
    job.ld_x = p.ld_x;
    job.w = p.w;
    job.s = p.s;
    job.y = p.y;
    job.ld_y = p.ld_y;
    job.tokens = p.tokens;
    job.status = p.status;
    const uint64_t token_tiles = (p.tokens + kManyMostTokens - 1) / kManyMostTokens;
    job.tile_tokens = uint32_t(((p.tokens + token_tiles - 1) / token_tiles + 15) / 16 * 16);
    // a map's stride is a multiple of 16 bytes and below 2^40
    const bool aligned = p.ld_x % 8 == 0;
    if (aligned) {
        const cuuint64_t extent[2] = {p.s.cols, p.tokens}, stride[1] = {p.ld_x * 2};
        const cuuint32_t box[2] = {64, job.tile_tokens}, step[2] = {1, 1};
        const auto encode = map_encoder();
        if (!encode || encode(&job.map, p.dt == ENEC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                              const_cast<uint8_t*>(p.x), extent, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return ENEC_ERR_CUDA;
    }
    // 256 rows a tile where that leaves work for most SMs; else 128, and the columns shared out as far as there are SMs
    uint32_t mt = 2;
    uint64_t tiles = (p.s.row_tiles + 1) / 2 * token_tiles;
    if (tiles * 4 < uint64_t(dev.sms) * 3) mt = 1, tiles = p.s.row_tiles * token_tiles;
    if (tiles >> 28) return ENEC_ERR_TOO_LARGE;
    job.row_tiles = (p.s.row_tiles + mt - 1) / mt;
    job.cluster = 1, job.share = p.s.col_tiles;
    if (mt == 1) share_columns(job, uint32_t(std::min<uint64_t>(8, dev.sms / tiles)));
    const auto launch = [&](auto dt, auto tiles_high) {
        constexpr int kDt = decltype(dt)::value, kMt = decltype(tiles_high)::value;
        return aligned ? launch_many<kDt, kMt, true>(job, uint32_t(tiles), dev, stream) : launch_many<kDt, kMt, false>(job, uint32_t(tiles), dev, stream);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    if (p.dt == ENEC_BF16) {
        const std::integral_constant<int, ENEC_BF16> dt;
        return mt == 2 ? launch(dt, two) : launch(dt, one);
    }
    const std::integral_constant<int, ENEC_FP16> dt;
    return mt == 2 ? launch(dt, two) : launch(dt, one);
}

}  // namespace enec
