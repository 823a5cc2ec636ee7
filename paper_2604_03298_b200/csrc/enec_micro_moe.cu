// A mixture-of-experts layer for few tokens over microscaled expert weights, in two launches.
//
//   l = x R^T; of the softmax p of a token's l the `top` largest, w = p or p over their sum (a pair: a token and one of its experts);
//   h[pair] = silu(x G_e^T) * (x U_e^T);   y[token] = sum over its pairs of w (h[pair] D_e^T)
//
// Launch 1: every cluster of CTAs computes the router's products (each CTA a part of the columns; sums are joined through
// distributed shared memory) and every CTA chooses the experts for itself, which costs less than a launch and a wait between.
// Then it takes its share of the tasks: a group of pairs of one expert, a row tile of gate or of up, and all of its columns or, where
// pairs are few, a part of them. Sums go to the workspace. Launch 2 does the same over row tiles of down; it makes the hidden values
// from launch 1's sums as it lays out a group's columns. The CTA that is the last one to finish a row tile adds the pairs of every
// token, in the order of the token's choice and of the parts, so no sum depends on which CTA that was.
// Both are bound by the chosen experts' bytes, which are read once for a group of an expert's pairs: as many as the digits of whole rows
// leave room for, 16 up to 2304 columns, 8 at 4096, 4 at 7168, 1 at 14336 (see enec_micro_pieces.cuh for the products).
#include "enec_micro_pieces.cuh"

#include <cooperative_groups.h>


#include "enec_micro_launch.cuh"

namespace enec {
namespace {

constexpr uint32_t kMoeCluster = 4;
constexpr uint32_t kMoeWarps = kPieceThreads / 32;
constexpr uint32_t kMoeMostTokens = 64;
constexpr uint32_t kMoeMostExperts = 512;
constexpr uint32_t kMoeMostTop = 16;
constexpr uint32_t kMoeMostLogits = 24576;   // tokens x experts: two such arrays of fp32 in shared memory

struct MoeJob {
    const uint8_t* x;
    uint64_t ld_x;
    const uint8_t* router;
    const uint8_t* gate;
    const uint8_t* up;
    const uint8_t* down;
    MicroShape s_in, s_out;          // of gate and up; of down
    uint8_t* y;
    uint64_t ld_y;
    uint32_t tokens, hidden, inter, experts, top, renormalize;
    uint32_t group, stages;          // pairs of a group and stages of the ring, in this launch
    uint32_t most_slices;            // parts of the columns, at most
    uint32_t ld_h;
    uint32_t* slices;                // the parts that launch 1 has chosen
    uint8_t* tables;                 // launch 1's routing tables
    uint32_t* tickets;               // one per row tile of down
    float* in_sums;                  // [part][gate, up][pair][ld_h]
    float* out_sums;                 // [part][pair][hidden]
    int* status;
};

// Shared memory: [routing tables | ring | digits]; the router's sums use what lies behind the tables.
__host__ __device__ inline uint32_t routing_bytes(uint32_t pairs, uint32_t experts) {
    return (pairs * 8 + (experts + 1) * 10 + 1023) / 1024 * 1024;
}
struct Routing {
    float* weight;            // [pairs]
    uint16_t* expert;         // [pairs]
    uint16_t* list;           // [pairs]: pairs by expert, then by number
    uint32_t* count;          // [experts + 1]
    uint16_t* first;          // [experts + 1]: into list
    uint16_t* next;           // [experts + 1]
    uint16_t* group_first;    // [experts + 1]
    uint32_t pairs, experts;
};
__device__ __forceinline__ Routing routing_at(uint8_t* smem, uint32_t pairs, uint32_t experts) {
    Routing r;
    r.weight = reinterpret_cast<float*>(smem);
    r.count = reinterpret_cast<uint32_t*>(r.weight + pairs);
    r.expert = reinterpret_cast<uint16_t*>(r.count + experts + 1);
    r.list = r.expert + pairs;
    r.first = r.list + pairs;
    r.next = r.first + experts + 1;
    r.group_first = r.next + experts + 1;
    r.pairs = pairs;
    r.experts = experts;
    return r;
}

// From every pair's expert: the pairs of each expert in order, cut into groups. Called by the whole CTA; every CTA of both launches has
// to come to the same groups, so a pair's place goes by its number, not by which thread was faster.
__device__ __forceinline__ void build_lists(const Routing& r, uint32_t group) {
    for (uint32_t e = threadIdx.x; e <= r.experts; e += blockDim.x) r.count[e] = 0;
    __syncthreads();
    for (uint32_t p = threadIdx.x; p < r.pairs; p += blockDim.x) atomicAdd(r.count + r.expert[p], 1u);
    __syncthreads();
    if (threadIdx.x < 32) {
        const uint32_t lane = threadIdx.x;
        uint32_t pairs = 0, groups = 0;
        for (uint32_t e0 = 0; e0 < r.experts; e0 += 32) {
            const uint32_t e = e0 + lane;
            const uint32_t n = e < r.experts ? r.count[e] : 0, g = (n + group - 1) / group;
            uint32_t sum_n = n, sum_g = g;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const uint32_t a = __shfl_up_sync(0xFFFFFFFFu, sum_n, d), b = __shfl_up_sync(0xFFFFFFFFu, sum_g, d);
                if (int(lane) >= d) sum_n += a, sum_g += b;
            }
            if (e < r.experts) {
                r.first[e] = uint16_t(pairs + sum_n - n);
                r.next[e] = uint16_t(pairs + sum_n - n);
                r.group_first[e] = uint16_t(groups + sum_g - g);
            }
            pairs += __shfl_sync(0xFFFFFFFFu, sum_n, 31);
            groups += __shfl_sync(0xFFFFFFFFu, sum_g, 31);
        }
        if (lane == 0) r.first[r.experts] = uint16_t(pairs), r.group_first[r.experts] = uint16_t(groups);
        __syncwarp();
        for (uint32_t p0 = 0; p0 < r.pairs; p0 += 32) {
            const uint32_t p = p0 + lane, e = p < r.pairs ? r.expert[p] : 0xFFFFu;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, e);
            const uint32_t before = __popc(same & ((1u << lane) - 1));
            if (p < r.pairs) r.list[r.next[e] + before] = uint16_t(p);
            __syncwarp();
            if (p < r.pairs && before == 0) r.next[e] += uint16_t(__popc(same));
            __syncwarp();
        }
    }
    __syncthreads();
}

struct Group {
    uint32_t expert, first, n;   // pairs list[first .. first + n - 1]
};
__device__ __forceinline__ Group group_of(const Routing& r, uint32_t index, uint32_t group) {
    uint32_t low = 0, high = r.experts;   // the last expert whose first group is not behind `index`
    while (high - low > 1) {
        const uint32_t mid = (low + high) / 2;
        if (r.group_first[mid] <= index) low = mid;
        else high = mid;
    }
    Group g;
    g.expert = low;
    const uint32_t begin = (index - r.group_first[low]) * group;
    g.first = r.first[low] + begin;
    g.n = min(group, r.count[low] - begin);
    return g;
}

template <int DT>
__device__ __forceinline__ void mma_native(float* c, const uint32_t* a0, const uint32_t* a1, const uint32_t* b) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        if constexpr (DT == ENEC_FP16) {
            asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                : "r"(a0[i]), "r"(a1[i]), "r"(a0[i + 1]), "r"(a1[i + 1]), "r"(b[i]), "r"(b[i + 1]));
        } else {
            asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                : "r"(a0[i]), "r"(a1[i]), "r"(a0[i + 1]), "r"(a1[i + 1]), "r"(b[i]), "r"(b[i + 1]));
        }
    }
}

// The order of logits as numbers without sign, from 1 on; NaN comes last. (-infinity is 0x007FFFFF.) 0 is free for what cannot be chosen.
__device__ __forceinline__ uint32_t logit_key(float v) {
    const uint32_t b = __float_as_uint(v == 0.f ? 0.f : v);   // the two zeros are equal
    if (v != v) return 1;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Parts of a CTA's columns that warps share in the router's products; and the bytes of its sums.
__host__ __device__ inline uint32_t router_splits(uint32_t tokens, uint32_t experts) {
    const uint32_t tiles = (experts + 15) / 16 * ((tokens + 7) / 8);
    return tiles >= 16 ? 1 : 16 / tiles;
}
__host__ __device__ inline uint32_t router_bytes(uint32_t tokens, uint32_t experts) {
    return (1 + router_splits(tokens, experts)) * tokens * experts * 4;
}

// A warp: the `top` largest of `experts` logits, ties to the lower number; lane j gets the j-th. N: experts a lane looks after.
template <uint32_t N>
__device__ __forceinline__ uint32_t choose_experts(const float* l, uint32_t experts, uint32_t top, uint32_t lane) {
    uint32_t keys[N];   // of experts lane, lane + 32, ..; 0 for those that do not exist or have been chosen
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) keys[i] = lane + 32 * i < experts ? logit_key(l[lane + 32 * i]) : 0u;
    uint32_t mine = 0;
    for (uint32_t j = 0; j < top; ++j) {
        uint32_t key = 0, at = 0;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            at = keys[i] > key ? i : at;
            key = max(keys[i], key);
        }
        const uint32_t best = __reduce_max_sync(0xFFFFFFFFu, key);
        const uint32_t chosen = __reduce_min_sync(0xFFFFFFFFu, key == best ? lane + 32 * at : 0xFFFFFFFFu);
        const uint32_t gone = (chosen & 31) == lane ? chosen >> 5 : N;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) keys[i] = i == gone ? 0u : keys[i];
        mine = lane == j ? chosen : mine;
    }
    return mine;
}

// The router: logits of all tokens to every CTA of the cluster, then every warp chooses for its tokens.
template <int DT>
__device__ __forceinline__ void route(const MoeJob& job, const Routing& r, float* scratch) {
    auto cluster = cooperative_groups::this_cluster();
    const uint32_t rank = cluster.block_rank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t total = job.tokens * job.experts;
    const uint32_t blocks = (job.hidden + 31) / 32, share = (blocks + kMoeCluster - 1) / kMoeCluster;
    const uint32_t b0 = min(rank * share, blocks), b1 = min(b0 + share, blocks);
    const uint32_t expert_tiles = (job.experts + 15) / 16, token_tiles = (job.tokens + 7) / 8, tiles = expert_tiles * token_tiles;
    // where tiles are few, warps share a tile's columns too
    const uint32_t splits = router_splits(job.tokens, job.experts), split_blocks = (share + splits - 1) / splits;
    float* logits = scratch;
    float* part = scratch + total;   // [split][token][expert]
    const bool whole = job.hidden % 32 == 0 && job.ld_x % 8 == 0;   // every load is of 16 aligned bytes
    for (uint32_t unit = warp; unit < tiles * splits; unit += kMoeWarps) {
        const uint32_t tile = unit % tiles, split = unit / tiles;
        const uint32_t e = tile % expert_tiles * 16 + g, token = tile / expert_tiles * 8 + g;
        // rows that do not exist are read from the last one's place and not written
        const uint8_t* r0 = job.router + uint64_t(min(e, job.experts - 1)) * job.hidden * 2;
        const uint8_t* r1 = job.router + uint64_t(min(e + 8, job.experts - 1)) * job.hidden * 2;
        const uint8_t* xr = job.x + uint64_t(min(token, job.tokens - 1)) * job.ld_x * 2;
        const uint32_t first = min(b0 + split * split_blocks, b1), last = min(first + split_blocks, b1);
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        constexpr uint32_t kBatch = 4;
        for (uint32_t b = first; b < last; b += kBatch) {
            uint32_t a0[kBatch][4], a1[kBatch][4], bx[kBatch][4];
            if (whole && b + kBatch <= last) {
#pragma unroll
                for (uint32_t i = 0; i < kBatch; ++i) {
                    const uint64_t at = uint64_t(32 * (b + i) + 8 * t) * 2;
                    const uint4 v0 = __ldg(reinterpret_cast<const uint4*>(r0 + at)), v1 = __ldg(reinterpret_cast<const uint4*>(r1 + at)),
                                v2 = __ldg(reinterpret_cast<const uint4*>(xr + at));
                    a0[i][0] = v0.x, a0[i][1] = v0.y, a0[i][2] = v0.z, a0[i][3] = v0.w;
                    a1[i][0] = v1.x, a1[i][1] = v1.y, a1[i][2] = v1.z, a1[i][3] = v1.w;
                    bx[i][0] = v2.x, bx[i][1] = v2.y, bx[i][2] = v2.z, bx[i][3] = v2.w;
                }
            } else {
#pragma unroll
                for (uint32_t i = 0; i < kBatch; ++i) {
                    const uint32_t col = 32 * (b + i) + 8 * t;
                    const int valid = b + i < last && col < job.hidden ? int(min(job.hidden - col, 8u)) : 0;
                    load_eight<DT>(r0 + uint64_t(col) * 2, valid, a0[i]);
                    load_eight<DT>(r1 + uint64_t(col) * 2, valid, a1[i]);
                    load_eight<DT>(xr + uint64_t(col) * 2, valid, bx[i]);
                }
            }
#pragma unroll
            for (uint32_t i = 0; i < kBatch; ++i) mma_native<DT>(c, a0[i], a1[i], bx[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t ee = tile % expert_tiles * 16 + g + (i >> 1) * 8, tt = tile / expert_tiles * 8 + 2 * t + (i & 1);
            if (ee < job.experts && tt < job.tokens) part[split * total + tt * job.experts + ee] = c[i];
        }
    }
    if (splits > 1) {
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < total; i += blockDim.x) {
            float v = part[i];
            for (uint32_t s = 1; s < splits; ++s) v += part[s * total + i];
            part[i] = v;
        }
    }
    cluster.sync();
    const uint32_t per = (total + kMoeCluster - 1) / kMoeCluster;
    for (uint32_t i = rank * per + threadIdx.x; i < min(total, (rank + 1) * per); i += blockDim.x) {
        float v = 0.f;
#pragma unroll
        for (uint32_t k = 0; k < kMoeCluster; ++k) v += cluster.map_shared_rank(part, k)[i];
#pragma unroll
        for (uint32_t k = 0; k < kMoeCluster; ++k) cluster.map_shared_rank(logits, k)[i] = v;
    }
    cluster.sync();
    for (uint32_t token = warp; token < job.tokens; token += kMoeWarps) {
        const float* l = logits + token * job.experts;
        const uint32_t my_expert = job.experts <= 64    ? choose_experts<2>(l, job.experts, job.top, lane)
                                   : job.experts <= 128 ? choose_experts<4>(l, job.experts, job.top, lane)
                                                        : choose_experts<kMoeMostExperts / 32>(l, job.experts, job.top, lane);
        float my_logit = 0.f;
        if (lane < job.top) my_logit = l[my_expert];
        const float highest = __shfl_sync(0xFFFFFFFFu, my_logit, 0);
        const float mine = lane < job.top ? expf(my_logit - highest) : 0.f;
        float sum = job.renormalize ? mine : 0.f;
        if (!job.renormalize)
            for (uint32_t e = lane; e < job.experts; e += 32) sum += expf(l[e] - highest);
#pragma unroll
        for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (lane < job.top) {
            r.weight[token * job.top + lane] = mine / sum;
            r.expert[token * job.top + lane] = uint16_t(my_expert);
        }
    }
    __syncthreads();
}

// How many parts a matrix's columns are cut into: what gives the CTA with most tasks the least to do, a task counted as its records and
// two more for taking its sums.
__device__ __forceinline__ uint32_t choose_slices(uint32_t tasks, uint32_t records, uint32_t most) {
    if (most == 1) return 1;
    const uint32_t lane = threadIdx.x & 31, n = 1u << (lane & 3);   // by whole warps: lanes 0 to 3 look at 1, 2, 4 and 8 parts
    uint32_t cost = 0xFFFFFFFFu;
    if (n <= most && n <= records) cost = (tasks * n + gridDim.x - 1) / gridDim.x * ((records + n - 1) / n + 2);
    const uint32_t least = __reduce_min_sync(0xFFFFFFFFu, cost);
    return 1u << __reduce_min_sync(0xFFFFFFFFu, cost == least ? lane & 3 : 3u);
}

// The tasks of a launch, in the order group, part of the columns, matrix, row tile; and a CTA's share of them.
struct Tasks {
    uint32_t matrices, tiles, slices, records, share;
    uint32_t begin, end;
    __device__ __forceinline__ Tasks(uint32_t groups, uint32_t matrices_, const MicroShape& s, uint32_t slices_)
        : matrices(matrices_), tiles(s.row_tiles), slices(slices_), records(s.col_tiles), share((s.col_tiles + slices_ - 1) / slices_) {
        // below 2^32: 1024 groups, two matrices, 2^17 row tiles, eight parts where groups are at most eight
        const uint32_t all = groups * matrices * tiles * slices, each = all / gridDim.x, more = all % gridDim.x;
        begin = blockIdx.x * each + min(blockIdx.x, more);
        end = begin + each + (blockIdx.x < more ? 1 : 0);
    }
};
// A walk over a CTA's tasks: divisions once, then counting.
struct Walk {
    const Tasks& tasks;
    const Routing& r;
    uint32_t group_size;
    const uint8_t* m0;
    const uint8_t* m1;
    uint32_t group, matrix, tile, slice;
    Group now;
    __device__ __forceinline__ Walk(const Tasks& tasks_, const Routing& r_, uint32_t group_size_, const uint8_t* m0_, const uint8_t* m1_)
        : tasks(tasks_), r(r_), group_size(group_size_), m0(m0_), m1(m1_) {
        tile = tasks.begin % tasks.tiles;
        uint32_t rest = tasks.begin / tasks.tiles;
        matrix = rest % tasks.matrices, rest /= tasks.matrices;
        slice = rest % tasks.slices;
        group = rest / tasks.slices;
        if (tasks.begin < tasks.end) now = group_of(r, group, group_size);
    }
    __device__ __forceinline__ PieceTask get() const {
        const uint32_t first = min(slice * tasks.share, tasks.records);
        const uint64_t strip = uint64_t(now.expert) * tasks.tiles + tile;
        return {(matrix ? m1 : m0) + kMicroHeaderBytes + strip * tasks.records * kMicroRecordBytes, first, min(tasks.share, tasks.records - first),
                group * tasks.slices + slice, now.n};
    }
    __device__ __forceinline__ void next() {
        if (++tile < tasks.tiles) return;
        tile = 0;
        if (++matrix < tasks.matrices) return;
        matrix = 0;
        if (++slice < tasks.slices) return;
        slice = 0;
        if (++group < r.group_first[r.experts]) now = group_of(r, group, group_size);
    }
};

template <int DT>
__global__ void __launch_bounds__(kPieceThreads, 1) enec_moe_in_kernel(const __grid_constant__ MoeJob job) {
    extern __shared__ uint8_t raw[];
    __shared__ PieceShared sh;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    const uint32_t pairs = job.tokens * job.top, tables = routing_bytes(pairs, job.experts);
    const Routing r = routing_at(smem, pairs, job.experts);
    piece_setup(sh, job.stages);
    pdl_wait();
    pdl_launch_dependents();
    const MicroProbe gate_header(job.gate), up_header(job.up);
    route<DT>(job, r, reinterpret_cast<float*>(smem + tables));
    build_lists(r, job.group);
    fence_async_shared();   // the ring's bulk copies go where the router's sums were
    __syncthreads();
    const uint32_t groups = r.group_first[job.experts];
    const uint32_t slices = choose_slices(groups * 2 * job.s_in.row_tiles, job.s_in.col_tiles, job.most_slices);
    if (blockIdx.x == 0) {
        for (uint32_t i = threadIdx.x; i < tables / 16; i += kPieceThreads)
            reinterpret_cast<uint4*>(job.tables)[i] = reinterpret_cast<const uint4*>(smem)[i];
        for (uint32_t i = threadIdx.x; i < job.s_out.row_tiles; i += kPieceThreads) job.tickets[i] = 0;
        if (threadIdx.x == 0) *job.slices = slices;
    }
    const bool good = gate_header.fits(job.s_in) && up_header.fits(job.s_in);
    const Tasks tasks(groups, 2, job.s_in, slices);
    const uint32_t worker = warp - 2, row_in = (warp & 3) * 32 + lane;
    Walk walk(tasks, r, job.group, job.gate, job.up), here = walk;
    piece_products(
        sh, smem + tables, job.stages, tasks.end - tasks.begin, job.hidden, walk,
        [&](uint32_t c, uint32_t col, float* x) {
            uint32_t w[4];
            load_eight<DT>(job.x + (uint64_t(r.list[here.now.first + c] / job.top) * job.ld_x + col) * 2,
                           col < job.hidden ? int(min(job.hidden - col, 8u)) : 0, w);
            as_floats<DT>(w, x);
        },
        [&](uint32_t, uint32_t tmem, bool ok) {
            const uint32_t row = here.tile * kMicroRows + row_in;
            const bool any = here.slice * tasks.share < tasks.records;
            for (uint32_t c = worker >> 2; c < here.now.n; c += kPieceWorkers / 4) {
                const float v = any ? take_sum(tmem, c) : 0.f;
                if (good && ok && row < job.inter)
                    job.in_sums[(uint64_t(here.slice * 2 + here.matrix) * pairs + r.list[here.now.first + c]) * job.ld_h + row] = v;
            }
        },
        [&](uint32_t, bool) { here.next(); }, false, [](uint32_t) {});
    if (threadIdx.x == 0) {
        if (sh.failed) report(job.status, ENEC_ERR_TIMEOUT);
        else if (!good && blockIdx.x == 0) report(job.status, ENEC_ERR_BAD_STREAM);
    }
}

template <int DT>
__global__ void __launch_bounds__(kPieceThreads, 1) enec_moe_out_kernel(const __grid_constant__ MoeJob job) {
    extern __shared__ uint8_t raw[];
    __shared__ PieceShared sh;
    __shared__ uint32_t last;
    using T = typename MicroType<DT>::T;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    const uint32_t pairs = job.tokens * job.top, tables = routing_bytes(pairs, job.experts);
    const Routing r = routing_at(smem, pairs, job.experts);
    piece_setup(sh, job.stages);
    pdl_wait();
    pdl_launch_dependents();
    // the tables of launch 1: the groups are the same
    for (uint32_t i = threadIdx.x; i < tables / 16; i += kPieceThreads) reinterpret_cast<uint4*>(smem)[i] = __ldcg(reinterpret_cast<const uint4*>(job.tables) + i);
    const uint32_t in_slices = *job.slices;
    const MicroProbe gate_header(job.gate), up_header(job.up), down_header(job.down);
    __syncthreads();
    const uint32_t groups = r.group_first[job.experts];
    const uint32_t slices = choose_slices(groups * job.s_out.row_tiles, job.s_out.col_tiles, job.most_slices);
    const bool good = gate_header.fits(job.s_in) && up_header.fits(job.s_in) && down_header.fits(job.s_out);
    const Tasks tasks(groups, 1, job.s_out, slices);
    const uint32_t worker = warp - 2, row_in = (warp & 3) * 32 + lane;
    Walk walk(tasks, r, job.group, job.down, nullptr), here = walk;
    piece_products(
        sh, smem + tables, job.stages, tasks.end - tasks.begin, job.inter, walk,
        [&](uint32_t c, uint32_t col, float* x) {
            const int valid = col < job.inter ? int(min(job.inter - col, 8u)) : 0;
            const float* from = job.in_sums + uint64_t(r.list[here.now.first + c]) * job.ld_h + col;
            const uint64_t matrix = uint64_t(pairs) * job.ld_h;
            float u[8] = {};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
            for (uint32_t s = 0; s < in_slices; ++s, from += 2 * matrix) {
                uint32_t wa[8], wu[8];
                load_eight<ENEC_FP32>(reinterpret_cast<const uint8_t*>(from), valid, wa);
                load_eight<ENEC_FP32>(reinterpret_cast<const uint8_t*>(from + matrix), valid, wu);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += __uint_as_float(wa[e]), u[e] += __uint_as_float(wu[e]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] / (1.f + expf(-x[e])) * u[e];
        },
        [&](uint32_t, uint32_t tmem, bool) {
            const uint32_t row = here.tile * kMicroRows + row_in;
            const bool any = here.slice * tasks.share < tasks.records;
            for (uint32_t c = worker >> 2; c < here.now.n; c += kPieceWorkers / 4) {
                const float v = any ? take_sum(tmem, c) : 0.f;
                const uint32_t pair = r.list[here.now.first + c];
                if (row < job.hidden) __stcg(job.out_sums + (uint64_t(here.slice) * pairs + pair) * job.hidden + row, v * r.weight[pair]);
            }
        },
        [&](uint32_t, bool ok) {
            const uint32_t tile = here.tile, row = tile * kMicroRows + row_in;
            here.next();
            // every worker's values are visible to all before the ticket counts the task
            __threadfence();
            asm volatile("bar.sync 1, %0;" ::"n"(kPieceWorkers * 32) : "memory");
            if (worker == 0 && lane == 0) last = atomicAdd(job.tickets + tile, 1u) == groups * slices - 1;
            asm volatile("bar.sync 1, %0;" ::"n"(kPieceWorkers * 32) : "memory");
            if (!last || !good || !ok) return;
            __threadfence();
            if (row >= job.hidden) return;
            // a token's pairs in the order of its choice, each part by part; loads of eight pairs are on the way together
#pragma unroll 2
            for (uint32_t token = worker >> 2; token < job.tokens; token += kPieceWorkers / 4) {
                const float* from = job.out_sums + uint64_t(token) * job.top * job.hidden + row;
                float v = 0.f;
                for (uint32_t j0 = 0; j0 < job.top; j0 += 8) {
                    float term[8];
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) term[j] = j0 + j < job.top ? __ldcg(from + uint64_t(j0 + j) * job.hidden) : 0.f;
                    for (uint32_t s = 1; s < slices; ++s) {
#pragma unroll
                        for (uint32_t j = 0; j < 8; ++j)
                            if (j0 + j < job.top) term[j] += __ldcg(from + (uint64_t(s) * pairs + j0 + j) * job.hidden);
                    }
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) v += term[j];
                }
                reinterpret_cast<T*>(job.y)[uint64_t(token) * job.ld_y + row] = MicroType<DT>::one(v);
            }
        },
        false, [](uint32_t) {});
    if (threadIdx.x == 0) {
        if (sh.failed) report(job.status, ENEC_ERR_TIMEOUT);
        else if (!good && blockIdx.x == 0) report(job.status, ENEC_ERR_BAD_STREAM);
    }
}

// Pairs per group, stages of the ring and with them the shared memory: as many pairs as there may be with four stages; where there is no room
// for one pair so, with three or two.
bool choose_group(uint32_t fixed, uint32_t records, uint32_t most, uint32_t least_bytes, uint32_t& group, uint32_t& stages, uint32_t& bytes) {
    const auto fits = [&](uint32_t pairs, uint32_t ring) {
        const uint64_t others = 1024 + fixed + uint64_t(records) * piece_record_bytes(pairs);
        if (others + ring * kMicroRecordBytes > kFewMostShared) return false;
        const uint64_t fit = (kFewMostShared - others) / kMicroRecordBytes;
        group = pairs;
        stages = fit < kPieceMostStages ? uint32_t(fit) : kPieceMostStages;
        bytes = uint32_t(others + stages * kMicroRecordBytes);
        if (bytes < 1024 + fixed + least_bytes) bytes = 1024 + fixed + least_bytes;
        if (bytes < kTmemAloneShared) bytes = kTmemAloneShared;
        return bytes <= kFewMostShared;
    };
    for (uint32_t pairs = most; pairs > 0; --pairs)
        if (fits(pairs, 4)) return true;
    return fits(1, 2);
}

template <int DT>
enec_status launch_moe(MoeJob job, const MicroDevice& dev, cudaStream_t stream) {
    const uint32_t pairs = job.tokens * job.top, tables = routing_bytes(pairs, job.experts);
    const uint32_t most = kPieceTokens < job.tokens ? kPieceTokens : job.tokens;   // an expert has at most one pair of a token
    uint32_t bytes = 0, clusters = 0;
    static std::atomic<uint64_t> allowed_in{0}, allowed_out{0};
    MoeJob second = job;
    uint32_t bytes2 = 0;
    if (!choose_group(tables, job.s_in.col_tiles, most, router_bytes(job.tokens, job.experts), job.group, job.stages, bytes) ||
        !choose_group(tables, job.s_out.col_tiles, most, 0, second.group, second.stages, bytes2))
        return ENEC_ERR_TOO_LARGE;
    // one size of group for both launches: the larger rows' decides
    const uint32_t group = job.group < second.group ? job.group : second.group;
    if (!choose_group(tables, job.s_in.col_tiles, group, router_bytes(job.tokens, job.experts), job.group, job.stages, bytes) ||
        !choose_group(tables, job.s_out.col_tiles, group, 0, second.group, second.stages, bytes2) || job.group != second.group)
        return ENEC_ERR_TOO_LARGE;
    if (!allow_shared(allowed_in, dev, enec_moe_in_kernel<DT>, kFewMostShared) ||
        !allow_shared(allowed_out, dev, enec_moe_out_kernel<DT>, kFewMostShared) ||
        !resident_clusters(enec_moe_in_kernel<DT>, dev, kMoeCluster, kPieceThreads, bytes, clusters))
        return ENEC_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(clusters * kMoeCluster);
    cfg.blockDim = dim3(kPieceThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kMoeCluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t err = cudaLaunchKernelEx(&cfg, enec_moe_in_kernel<DT>, job);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (err != cudaSuccess) return ENEC_ERR_CUDA;
    err = launch_pdl(enec_moe_out_kernel<DT>, uint32_t(dev.sms), kPieceThreads, bytes2, stream, second);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

struct MoeLayout {
    uint64_t tickets, in_sums, out_sums, total;
    uint32_t ld_h, most_slices;
};
bool moe_layout(uint64_t tokens, uint64_t hidden, uint64_t inter, uint64_t experts, uint64_t top, MoeLayout& l) {
    if (tokens > kMoeMostTokens || experts > kMoeMostExperts || top > kMoeMostTop || tokens * experts > kMoeMostLogits || (hidden >> 24) ||
        (inter >> 24))
        return false;
    const uint64_t pairs = tokens * top;
    // parts of the columns only while pairs are few: with 64 pairs and more there are tasks enough
    l.most_slices = pairs >= 64 ? 1 : pairs > 8 ? uint32_t(64 / pairs) : 8;
    l.ld_h = uint32_t((inter + 3) & ~uint64_t(3));
    l.tickets = 16 + routing_bytes(uint32_t(pairs), uint32_t(experts));
    l.in_sums = l.tickets + align16((hidden + kMicroRows) / kMicroRows * 4);
    l.out_sums = l.in_sums + l.most_slices * 2 * pairs * l.ld_h * 4;
    l.total = l.out_sums + align16(l.most_slices * pairs * hidden * 4);
    return true;
}

}  // namespace
}  // namespace enec

using namespace enec;

extern "C" size_t enec_moe_microscaled_workspace(size_t tokens, size_t hidden, size_t inter, size_t experts, size_t top_k) {
    MoeLayout l;
    return moe_layout(tokens, hidden, inter, experts, top_k, l) ? size_t(l.total) : 0;
}

extern "C" enec_status enec_moe_microscaled(const void* d_x, enec_dtype dt, size_t tokens, size_t hidden, size_t ld_x, const void* d_router,
                                            size_t experts, size_t top_k, int renormalize, const void* d_gate, size_t gate_size, const void* d_up,
                                            size_t up_size, const void* d_down, size_t down_size, size_t inter, void* d_y, size_t ld_y,
                                            void* d_workspace, size_t workspace_bytes, int* d_status, enec_stream_t stream) {
    if (dt != ENEC_BF16 && dt != ENEC_FP16) return ENEC_ERR_UNSUPPORTED_DTYPE;
    MoeLayout l;
    MoeJob job;
    if (!moe_layout(tokens, hidden, inter, experts, top_k, l) || !make_micro_shape(experts, inter, hidden, job.s_in) ||
        !make_micro_shape(experts, hidden, inter, job.s_out))
        return ENEC_ERR_TOO_LARGE;
    if (tokens == 0) return ENEC_OK;
    if (hidden == 0 || inter == 0 || experts == 0 || top_k == 0 || top_k > experts || ld_x < hidden || ld_y < hidden || (uint64_t(ld_x) >> 36) ||
        (uint64_t(ld_y) >> 36))
        return ENEC_ERR_INVALID_ARG;
    for (const void* p : {d_x, d_router, d_gate, d_up, d_down, static_cast<const void*>(d_y), static_cast<const void*>(d_workspace)})
        if (!p || !micro_aligned16(p)) return ENEC_ERR_INVALID_ARG;
    if (gate_size < job.s_in.total || up_size < job.s_in.total || down_size < job.s_out.total || workspace_bytes < l.total)
        return ENEC_ERR_BUFFER_TOO_SMALL;
    MicroDevice dev;
    if (!micro_device(dev)) return ENEC_ERR_CUDA;
    uint8_t* ws = static_cast<uint8_t*>(d_workspace);
    job.x = static_cast<const uint8_t*>(d_x);
    job.ld_x = ld_x;
    job.router = static_cast<const uint8_t*>(d_router);
    job.gate = static_cast<const uint8_t*>(d_gate);
    job.up = static_cast<const uint8_t*>(d_up);
    job.down = static_cast<const uint8_t*>(d_down);
    job.y = static_cast<uint8_t*>(d_y);
    job.ld_y = ld_y;
    job.tokens = uint32_t(tokens);
    job.hidden = uint32_t(hidden);
    job.inter = uint32_t(inter);
    job.experts = uint32_t(experts);
    job.top = uint32_t(top_k);
    job.renormalize = renormalize != 0;
    job.group = job.stages = 0;
    job.most_slices = l.most_slices;
    job.ld_h = l.ld_h;
    job.slices = reinterpret_cast<uint32_t*>(ws);
    job.tables = ws + 16;
    job.tickets = reinterpret_cast<uint32_t*>(ws + l.tickets);
    job.in_sums = reinterpret_cast<float*>(ws + l.in_sums);
    job.out_sums = reinterpret_cast<float*>(ws + l.out_sums);
    job.status = d_status;
    return dt == ENEC_BF16 ? launch_moe<ENEC_BF16>(job, dev, stream) : launch_moe<ENEC_FP16>(job, dev, stream);
}
