// A mixture-of-experts layer for few tokens over microscaled expert weights, in two launches.
//
//   l = x R^T; of the softmax p of a token's l the `top` largest, w = p or p over their sum (a pair: a token and one of its experts);
//   h[pair] = silu(x G_e^T) * (x U_e^T);   y[token] = sum over its pairs of w (h[pair] D_e^T)
//
// Launch 1: every cluster of eight CTAs computes the router's products (each CTA an eighth of the columns; sums are joined through
// distributed shared memory) and every CTA chooses the experts for itself, which costs less than a launch and a wait between.
// Then it takes its share of the items (a group of pairs of one expert x a strip of 16 rows of gate and up) and writes h in fp32.
// Launch 2 does the same over strips of down. A pair's sums go to the workspace; the CTA that is the last one to finish a strip
// adds the pairs of every token, in the order of the token's choice, so no sum depends on which CTA that was.
// Both are bound by the chosen experts' bytes, which are read once per group (8 or 16 pairs; see enec_micro_few.cuh for the products).
#include "enec_micro_few.cuh"

#include <cooperative_groups.h>

#include <map>
#include <mutex>

#include "enec_micro_launch.cuh"

namespace enec {
namespace {

constexpr uint32_t kMoeCluster = 8;
constexpr uint32_t kMoeMostTokens = 64;
constexpr uint32_t kMoeMostExperts = 512;
constexpr uint32_t kMoeMostTop = 16;
constexpr uint32_t kMoeMostShared = kFewMostShared - 1024;   // the kernels have a little static shared memory too
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
    uint32_t strips_in, strips_out;
    uint32_t group;                  // pairs of a group, in this launch
    uint32_t team;                   // warps of a team, in this launch
    uint32_t ld_h;
    uint32_t* pair_expert;
    float* pair_weight;
    uint32_t* tickets;               // one per strip of down
    float* h;
    float* partial;
    int* status;
};

// Shared memory: [routing tables | sums | inverses | ring | columns]; the router's sums use what lies behind the tables.
__host__ __device__ inline uint32_t routing_bytes(uint32_t pairs, uint32_t experts) {
    return (pairs * 8 + (3 * experts + 4) * 2 + 127) / 128 * 128;
}
struct Routing {
    float* weight;            // [pairs]
    uint16_t* expert;         // [pairs]
    uint16_t* list;           // [pairs]: pairs by expert, then by number
    uint16_t* count;          // [experts]
    uint16_t* first;          // [experts + 1]: into list
    uint16_t* group_first;    // [experts + 1]
    uint32_t pairs, experts;
};
__device__ __forceinline__ Routing routing_at(uint8_t* smem, uint32_t pairs, uint32_t experts) {
    Routing r;
    r.weight = reinterpret_cast<float*>(smem);
    r.expert = reinterpret_cast<uint16_t*>(r.weight + pairs);
    r.list = r.expert + pairs;
    r.count = r.list + pairs;
    r.first = r.count + experts;
    r.group_first = r.first + experts + 1;
    r.pairs = pairs;
    r.experts = experts;
    return r;
}

// From every pair's expert: the pairs of each expert in order, cut into groups. Called by the whole CTA.
__device__ __forceinline__ void build_lists(const Routing& r, uint32_t group) {
    for (uint32_t e = threadIdx.x; e < r.experts; e += blockDim.x) {
        uint32_t n = 0;
        for (uint32_t p = 0; p < r.pairs; ++p) n += r.expert[p] == e;
        r.count[e] = uint16_t(n);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        uint32_t pairs = 0, groups = 0;
        for (uint32_t e0 = 0; e0 < r.experts; e0 += 32) {
            const uint32_t e = e0 + threadIdx.x;
            const uint32_t n = e < r.experts ? r.count[e] : 0, g = (n + group - 1) / group;
            uint32_t sum_n = n, sum_g = g;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const uint32_t a = __shfl_up_sync(0xFFFFFFFFu, sum_n, d), b = __shfl_up_sync(0xFFFFFFFFu, sum_g, d);
                if (int(threadIdx.x) >= d) sum_n += a, sum_g += b;
            }
            if (e < r.experts) {
                r.first[e] = uint16_t(pairs + sum_n - n);
                r.group_first[e] = uint16_t(groups + sum_g - g);
            }
            pairs += __shfl_sync(0xFFFFFFFFu, sum_n, 31);
            groups += __shfl_sync(0xFFFFFFFFu, sum_g, 31);
        }
        if (threadIdx.x == 0) r.first[r.experts] = uint16_t(pairs), r.group_first[r.experts] = uint16_t(groups);
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < r.experts; e += blockDim.x) {
        if (r.count[e] == 0) continue;
        uint32_t at = r.first[e];
        for (uint32_t p = 0; p < r.pairs; ++p)
            if (r.expert[p] == e) r.list[at++] = uint16_t(p);
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
    g.n = min(group, uint32_t(r.count[low]) - begin);
    return g;
}

template <int DT>
__device__ __forceinline__ void mma_native(float* c, const uint32_t* a0, const uint32_t* a1, const uint32_t* b) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        if constexpr (DT == ENEC_FP16) {
            mma_f16(c, a0[i], a1[i], a0[i + 1], a1[i + 1], b[i], b[i + 1]);
        } else {
            asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                : "r"(a0[i]), "r"(a1[i]), "r"(a0[i + 1]), "r"(a1[i + 1]), "r"(b[i]), "r"(b[i + 1]));
        }
    }
}

// The order of logits as numbers without sign; NaN comes last.
__device__ __forceinline__ uint32_t logit_key(float v) {
    const uint32_t b = __float_as_uint(v);
    if (v != v) return 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The router: logits of all tokens to every CTA of the cluster, then every warp chooses for its tokens.
template <int DT>
__device__ __forceinline__ void route(const MoeJob& job, const Routing& r, float* scratch) {
    auto cluster = cooperative_groups::this_cluster();
    const uint32_t rank = cluster.block_rank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t total = job.tokens * job.experts;
    float* part = scratch;
    float* logits = scratch + total;
    const uint32_t blocks = (job.hidden + 31) / 32, share = (blocks + kMoeCluster - 1) / kMoeCluster;
    const uint32_t b0 = min(rank * share, blocks), b1 = min(b0 + share, blocks);
    const uint32_t expert_tiles = (job.experts + 15) / 16, token_tiles = (job.tokens + 7) / 8;
    for (uint32_t unit = warp; unit < expert_tiles * token_tiles; unit += kFewWarps) {
        const uint32_t e = unit % expert_tiles * 16 + g, token = unit / expert_tiles * 8 + g;
        const uint8_t* r0 = job.router + uint64_t(e) * job.hidden * 2;
        const uint8_t* r1 = r0 + uint64_t(8) * job.hidden * 2;
        const uint8_t* xr = job.x + uint64_t(token) * job.ld_x * 2;
        float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (uint32_t b = b0; b < b1; ++b) {
            const uint32_t col = 32 * b + 8 * t;
            const int valid = col < job.hidden ? int(min(job.hidden - col, 8u)) : 0;
            uint32_t a0[4], a1[4], bx[4];
            load_eight<DT>(r0 + uint64_t(col) * 2, e < job.experts ? valid : 0, a0);
            load_eight<DT>(r1 + uint64_t(col) * 2, e + 8 < job.experts ? valid : 0, a1);
            load_eight<DT>(xr + uint64_t(col) * 2, token < job.tokens ? valid : 0, bx);
            mma_native<DT>(c, a0, a1, bx);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t ee = unit % expert_tiles * 16 + g + (i >> 1) * 8, tt = unit / expert_tiles * 8 + 2 * t + (i & 1);
            if (ee < job.experts && tt < job.tokens) part[tt * job.experts + ee] = c[i];
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
    for (uint32_t token = warp; token < job.tokens; token += kFewWarps) {
        const float* l = logits + token * job.experts;
        uint32_t taken = 0;   // bit i: expert lane + 32 i
        float highest = 0.f, sum = 0.f, mine = 0.f;
        uint32_t my_expert = 0;
        for (uint32_t j = 0; j < job.top; ++j) {
            uint32_t key = 0, at = 0xFFFFFFFFu;
            for (uint32_t i = 0; lane + 32 * i < job.experts; ++i) {
                const uint32_t k = logit_key(l[lane + 32 * i]);
                if (!(taken >> i & 1) && (at == 0xFFFFFFFFu || k > key)) key = k, at = lane + 32 * i;
            }
            const uint32_t best = __reduce_max_sync(0xFFFFFFFFu, at == 0xFFFFFFFFu ? 0u : key);
            const uint32_t chosen = __reduce_min_sync(0xFFFFFFFFu, key == best ? at : 0xFFFFFFFFu);
            if ((chosen & 31) == lane) taken |= 1u << (chosen >> 5);
            const float v = l[chosen];
            if (j == 0) highest = v;
            const float p = expf(v - highest);
            if (job.renormalize) sum += p;
            if (lane == j) mine = p, my_expert = chosen;
        }
        if (!job.renormalize) {
            for (uint32_t e = lane; e < job.experts; e += 32) sum += expf(l[e] - highest);
#pragma unroll
            for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        }
        if (lane < job.top) {
            r.weight[token * job.top + lane] = mine / sum;
            r.expert[token * job.top + lane] = uint16_t(my_expert);
        }
    }
    __syncthreads();
}

// The items of a CTA: [begin, end) of groups x strips, the strips of a group one after another.
struct Share {
    uint32_t begin, end;
};
__device__ __forceinline__ Share share_of(uint64_t items) {
    return {uint32_t(items * blockIdx.x / gridDim.x), uint32_t(items * (blockIdx.x + 1) / gridDim.x)};
}

// A team's walk over its CTA's items: of every group's the team's own, every teams-th one.
struct Walk {
    uint32_t item, end, stop;        // the next item; where the CTA's items of its group end, and all of them
    uint32_t strips, team, teams;
    __device__ __forceinline__ void enter(uint32_t begin) {   // the group of item `begin`
        const uint32_t group_end = (begin / strips + 1) * strips;
        end = min(group_end, stop);
        item = begin + team;
    }
    __device__ __forceinline__ void settle() {                // on to the next group that has an item for the team
        while (item >= end && end < stop) enter(end);
    }
    __device__ __forceinline__ bool more() const { return item < end; }
};

// What both kernels do: the strips of `mats` matrices (gate and up, or down) of the CTA's groups times the groups' staged columns. `rows_of`
// gives the values of a column, `finish` takes an item's sums (of the team's warps) between two barriers of the team.
template <int DT, int NT, int MATS, class RowOf, class Finish>
__device__ __forceinline__ void expert_products(const Routing& r, uint32_t group, uint32_t team_warps, const uint8_t* m0, const uint8_t* m1, const MicroShape& s,
                                                uint32_t strips, uint8_t* smem, RowOf row_of, Finish finish) {
    constexpr uint32_t kStages = few_stages(MATS), kSums = few_sum_words(NT, MATS);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t units = (s.cols + kUnitCols - 1) / kUnitCols;
    const uint32_t team = warp / team_warps, in_team = warp % team_warps, teams = kFewWarps / team_warps;
    float* sums = reinterpret_cast<float*>(smem + few_ring_bytes(MATS)) + team * team_warps * kSums;
    float* inverse = reinterpret_cast<float*>(smem + few_fixed_bytes(NT, MATS));
    const uint32_t ring = smem_u32(smem) + warp * kStages * few_stage_bytes(MATS);
    const uint32_t staged = smem_u32(inverse + units * 8 * NT);
    const Share mine = share_of(uint64_t(r.group_first[r.experts]) * strips);
    if (mine.begin == mine.end) return;
    Walk asked{0, 0, mine.end, strips, team, teams};
    asked.enter(mine.begin);
    asked.settle();
    uint32_t ask_u = in_team, slot = 0, ask_group = 0xFFFFFFFFu;
    uint64_t ask_matrix = 0;
    auto ask = [&]() {
        if (asked.more() && ask_u < units) {
            const uint32_t index = asked.item / strips, strip = asked.item % strips;
            if (index != ask_group) {
                ask_group = index;
                ask_matrix = uint64_t(group_of(r, index, group).expert) * s.row_tiles;
            }
            const uint64_t at = kMicroHeaderBytes + (ask_matrix + (strip >> 3)) * s.col_tiles * kMicroRecordBytes;
            const uint32_t stage = ring + slot * few_stage_bytes(MATS);
            ask_unit(m0 + at, strip & 7, ask_u, stage, lane);
            if (MATS == 2) ask_unit(m1 + at, strip & 7, ask_u, stage + few_stage_bytes(1), lane);
            ask_u += team_warps;
            if (ask_u >= units) {
                ask_u = in_team;
                asked.item += teams;
                asked.settle();
            }
        }
        cp_async_commit();
        slot = slot + 1 == kStages ? 0 : slot + 1;
    };
#pragma unroll
    for (uint32_t i = 0; i < kStages - 1; ++i) ask();
    const uint32_t values = staged + g * 64 + t * 16;
    uint32_t from = 0;
    Walk walk{0, 0, mine.end, strips, team, teams};
    for (uint32_t begin = mine.begin; begin < mine.end; begin = walk.end) {
        walk.enter(begin);
        const Group now = group_of(r, begin / strips, group);
        __syncthreads();   // the columns of the group before have been used
        stage_columns<DT>([&](uint32_t i) { return row_of(r.list[now.first + i]); }, now.n, units, 0, s.cols, staged, inverse, 8 * NT);
        __syncthreads();
        bool exists[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) exists[nt] = nt * 8 + g < now.n;
        for (; walk.more(); walk.item += teams) {
            float acc[MATS][NT][4] = {};
            for (uint32_t u = in_team; u < units; u += team_warps) {
                cp_async_wait<kStages - 2>();
                __syncwarp();
                ask();   // into the slot that the unit before was read from, by all lanes
#pragma unroll
                for (int i = 0; i < MATS; ++i)
                    add_unit<NT>(acc[i], ring + from * few_stage_bytes(MATS) + i * few_stage_bytes(1), values + u * 4 * now.n * 64,
                                 inverse + u * 8 * NT + 2 * t, now.n, exists, lane);
                from = from + 1 == kStages ? 0 : from + 1;
            }
#pragma unroll
            for (int i = 0; i < MATS; ++i) put_sums<NT>(sums + in_team * kSums + i * few_sum_words(NT, 1), acc[i], lane);
            team_sync(team, team_warps * 32);
            finish(now, walk.item % strips, sums, in_team * 32 + lane, team);
            team_sync(team, team_warps * 32);   // the sums have been read before they are written again
        }
    }
    cp_async_wait<0>();
}

template <int DT, int NT>
__global__ void __launch_bounds__(kFewThreads, 1) enec_moe_in_kernel(const __grid_constant__ MoeJob job) {
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t pairs = job.tokens * job.top, tables = routing_bytes(pairs, job.experts);
    const Routing r = routing_at(smem, pairs, job.experts);
    pdl_wait();
    pdl_launch_dependents();
    route<DT>(job, r, reinterpret_cast<float*>(smem + tables));
    build_lists(r, job.group);
    if (blockIdx.x == 0) {
        for (uint32_t p = threadIdx.x; p < pairs; p += kFewThreads) job.pair_expert[p] = r.expert[p], job.pair_weight[p] = r.weight[p];
        for (uint32_t i = threadIdx.x; i < job.strips_out; i += kFewThreads) job.tickets[i] = 0;
    }
    if (!micro_header_ok(job.gate, job.s_in) || !micro_header_ok(job.up, job.s_in)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(job.status, ENEC_ERR_BAD_STREAM);
        return;
    }
    expert_products<DT, NT, 2>(
        r, job.group, job.team, job.gate, job.up, job.s_in, job.strips_in, smem + tables,
        [&](uint32_t pair) { return job.x + uint64_t(pair / job.top) * job.ld_x * 2; },
        [&](const Group& now, uint32_t strip, const float* sums, uint32_t thread, uint32_t) {
            for (uint32_t i = thread; i < 16 * now.n; i += job.team * 32) {
                const uint32_t m = i & 15, column = i >> 4;
                const uint32_t row = (strip >> 3) * kMicroRows + strip_row(strip & 7, m);
                float u = 0.f, v = 0.f;
                for (uint32_t k = 0; k < job.team; ++k) {
                    const float* theirs = sums + k * few_sum_words(NT, 2) + m * few_sum_row(NT) + column;
                    u += theirs[0];
                    v += theirs[few_sum_words(NT, 1)];
                }
                if (row < job.inter) job.h[uint64_t(r.list[now.first + column]) * job.ld_h + row] = u / (1.f + expf(-u)) * v;
            }
        });
}

template <int DT, int NT>
__global__ void __launch_bounds__(kFewThreads, 1) enec_moe_out_kernel(const __grid_constant__ MoeJob job) {
    extern __shared__ __align__(128) uint8_t smem[];
    using T = typename MicroType<DT>::T;
    __shared__ uint32_t last[kFewWarps / 4];   // of each team
    const uint32_t pairs = job.tokens * job.top, tables = routing_bytes(pairs, job.experts);
    const Routing r = routing_at(smem, pairs, job.experts);
    pdl_wait();
    pdl_launch_dependents();
    for (uint32_t p = threadIdx.x; p < pairs; p += kFewThreads) r.expert[p] = uint16_t(job.pair_expert[p]), r.weight[p] = job.pair_weight[p];
    if (!micro_header_ok(job.gate, job.s_in) || !micro_header_ok(job.up, job.s_in) || !micro_header_ok(job.down, job.s_out)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(job.status, ENEC_ERR_BAD_STREAM);
        return;
    }
    __syncthreads();
    build_lists(r, job.group);
    const uint32_t groups = r.group_first[job.experts];
    expert_products<ENEC_FP32, NT, 1>(
        r, job.group, job.team, job.down, nullptr, job.s_out, job.strips_out, smem + tables,
        [&](uint32_t pair) { return reinterpret_cast<const uint8_t*>(job.h + uint64_t(pair) * job.ld_h); },
        [&](const Group& now, uint32_t strip, const float* sums, uint32_t thread, uint32_t team) {
            for (uint32_t i = thread; i < 16 * now.n; i += job.team * 32) {
                const uint32_t m = i & 15, column = i >> 4, pair = r.list[now.first + column];
                const uint32_t row = (strip >> 3) * kMicroRows + strip_row(strip & 7, m);
                float v = 0.f;
                for (uint32_t k = 0; k < job.team; ++k) v += sums[k * few_sum_words(NT, 1) + m * few_sum_row(NT) + column];
                if (row < job.hidden) __stcg(job.partial + uint64_t(pair) * job.hidden + row, v * r.weight[pair]);
            }
            // every thread's values are visible to all before the ticket counts the item
            __threadfence();
            team_sync(team, job.team * 32);
            if (thread == 0) last[team] = atomicAdd(job.tickets + strip, 1u) == groups - 1;
            team_sync(team, job.team * 32);
            if (!last[team]) return;
            __threadfence();
            for (uint32_t i = thread; i < 16 * job.tokens; i += job.team * 32) {
                const uint32_t m = i & 15, token = i >> 4;
                const uint32_t row = (strip >> 3) * kMicroRows + strip_row(strip & 7, m);
                if (row >= job.hidden) continue;
                float v = 0.f;
                for (uint32_t j = 0; j < job.top; ++j) v += __ldcg(job.partial + uint64_t(token * job.top + j) * job.hidden + row);
                reinterpret_cast<T*>(job.y)[uint64_t(token) * job.ld_y + row] = MicroType<DT>::one(v);
            }
        });
}

uint32_t strips_of(const MicroShape& s) {
    const uint32_t last = s.rows - (s.row_tiles - 1) * kMicroRows;
    return (s.row_tiles - 1) * 8 + (last >= 32 ? 8 : (last + 3) / 4);
}

// Pairs per group, and with them the shared memory: as many as there may be.
bool choose_group(uint32_t fixed, uint32_t units, int nt, uint32_t most, uint32_t least_bytes, uint32_t& group, uint32_t& bytes) {
    for (group = most; group > 0; --group) {
        const uint64_t need = fixed + uint64_t(units) * few_unit_bytes(nt, group);
        if (need > kMoeMostShared) continue;
        bytes = need > least_bytes ? uint32_t(need) : least_bytes;
        return bytes <= kMoeMostShared;
    }
    return false;
}

// Clusters of a kernel that run at the same time, asked once per kernel, device and size.
template <class Kernel>
bool resident_clusters(Kernel* kernel, const MicroDevice& dev, uint32_t bytes, uint32_t& out) {
    static std::mutex mu;
    static std::map<std::pair<const void*, std::pair<int, uint32_t>>, int> known;
    std::lock_guard<std::mutex> lock(mu);
    int& n = known[std::make_pair(reinterpret_cast<const void*>(kernel), std::make_pair(dev.ordinal, bytes))];
    if (n == 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(kMoeCluster);
        cfg.blockDim = dim3(kFewThreads);
        cfg.dynamicSmemBytes = bytes;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = kMoeCluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
            n = 0;
            return false;
        }
    }
    out = uint32_t(n);
    return true;
}

template <int DT, int NT>
enec_status launch_moe(MoeJob job, const MicroDevice& dev, cudaStream_t stream) {
    const uint32_t pairs = job.tokens * job.top, tables = routing_bytes(pairs, job.experts);
    const uint32_t most = 8 * NT < job.tokens ? 8 * NT : job.tokens;   // an expert has at most one pair of a token
    uint32_t bytes = 0, clusters = 0;
    static std::atomic<uint64_t> allowed_in{0}, allowed_out{0};
    const uint32_t units_in = (job.hidden + kUnitCols - 1) / kUnitCols, units_out = (job.inter + kUnitCols - 1) / kUnitCols;
    MoeJob second = job;
    uint32_t bytes2 = 0;
    if (!choose_group(tables + few_fixed_bytes(NT, 2), units_in, NT, most, tables + 8 * job.tokens * job.experts, job.group, bytes) ||
        !choose_group(tables + few_fixed_bytes(NT, 1), units_out, NT, most, 0, second.group, bytes2))
        return ENEC_ERR_TOO_LARGE;
    if (!allow_shared(allowed_in, dev, enec_moe_in_kernel<DT, NT>, kMoeMostShared) ||
        !allow_shared(allowed_out, dev, enec_moe_out_kernel<DT, NT>, kMoeMostShared) ||
        !resident_clusters(enec_moe_in_kernel<DT, NT>, dev, bytes, clusters))
        return ENEC_ERR_CUDA;
    const uint64_t used = pairs < job.experts ? pairs : job.experts;   // experts with work, at most
    job.team = few_team(used * job.strips_in, units_in, clusters * kMoeCluster);
    second.team = few_team(used * job.strips_out, units_out, uint32_t(dev.sms));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(clusters * kMoeCluster);
    cfg.blockDim = dim3(kFewThreads);
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
    cudaError_t err = cudaLaunchKernelEx(&cfg, enec_moe_in_kernel<DT, NT>, job);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (err != cudaSuccess) return ENEC_ERR_CUDA;
    err = launch_pdl(enec_moe_out_kernel<DT, NT>, uint32_t(dev.sms), kFewThreads, bytes2, stream, second);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return err == cudaSuccess ? ENEC_OK : ENEC_ERR_CUDA;
}

struct MoeLayout {
    uint64_t weight, tickets, h, partial, total;
    uint32_t ld_h;
};
bool moe_layout(uint64_t tokens, uint64_t hidden, uint64_t inter, uint64_t experts, uint64_t top, MoeLayout& l) {
    if (tokens > kMoeMostTokens || experts > kMoeMostExperts || top > kMoeMostTop || tokens * experts > kMoeMostLogits || (hidden >> 24) ||
        (inter >> 24))
        return false;
    const uint64_t pairs = tokens * top;
    l.ld_h = uint32_t((inter + 3) & ~uint64_t(3));
    l.weight = align16(pairs * 4);
    l.tickets = l.weight + align16(pairs * 4);
    l.h = l.tickets + align16((hidden + kMicroRows) / kMicroRows * 8 * 4);
    l.partial = l.h + pairs * l.ld_h * 4;
    l.total = l.partial + align16(pairs * hidden * 4);
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
    job.strips_in = strips_of(job.s_in);
    job.strips_out = strips_of(job.s_out);
    job.group = job.team = 0;
    job.ld_h = l.ld_h;
    job.pair_expert = reinterpret_cast<uint32_t*>(ws);
    job.pair_weight = reinterpret_cast<float*>(ws + l.weight);
    job.tickets = reinterpret_cast<uint32_t*>(ws + l.tickets);
    job.h = reinterpret_cast<float*>(ws + l.h);
    job.partial = reinterpret_cast<float*>(ws + l.partial);
    job.status = d_status;
    if (dt == ENEC_BF16) return tokens <= 8 ? launch_moe<ENEC_BF16, 1>(job, dev, stream) : launch_moe<ENEC_BF16, 2>(job, dev, stream);
    return tokens <= 8 ? launch_moe<ENEC_FP16, 1>(job, dev, stream) : launch_moe<ENEC_FP16, 2>(job, dev, stream);
}
