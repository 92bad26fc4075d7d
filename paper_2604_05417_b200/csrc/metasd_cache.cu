// metasd_cache_plan / metasd_cache_release: where the next entries of paged caches go.
//
// A sequence adds new = max(0, length - cached) entries to the cache of the model (pool) it runs on.  Sequences are ordered by
// pool, in sequence order within each; with token_start the running sum of `new` in that order, entry t of the packed step belongs
// to the place at with token_start[at] <= t < token_start[at + 1], has position cached + t - token_start[at] and the slot
//     block_table[pool][sequence][position / page] * page + position % page.
// A sequence whose table is too short takes need = ceil(length / page) - held blocks from the end of its pool's free list, behind
// what the sequences before it take: running sums again.
//
// Two kernels.  The sums are one block's work: it reads some 20 bytes a sequence, and what it costs is the latency of its steps (4 us
// for 1024 sequences: two dependent loads 1.1, the sums and what is written for them 2).  The entries are spread over the whole
// GPU: 16 bytes are written for each, 100 MB for 6.3 M entries in 20 us (5 TB/s; a fill of that size takes 15), and what is
// left is latency, not instructions: the same walk in two thirds of them takes as long.  A step whose buffers have room for few entries is
// done by the first kernel alone.
//
// A release gives back what lies beyond the entries that stay, to the end of the free list, in the order that lets the next plan
// take the same blocks for the same places: one cluster per pool, bound by latency too (2.1 us for one sequence, 3.3 for 1024 with
// nothing to give back, 7 for 98 304 blocks).
#include <algorithm>

#include "metasd_staged.cuh"

namespace metasd {

namespace {

constexpr int MOST_THREADS = 1024, MOST_WARPS = 32;
constexpr int KEYS = METASD_MAX_POOLS + 1;      // the pools, and who takes no part
constexpr int FILL_THREADS = 256, FILL_BLOCKS = 6;     // of the second kernel; blocks to an SM
constexpr int STARTS = 2048;                    // places whose first entries a block keeps in shared memory
constexpr unsigned FULL = 0xFFFFFFFFu;

// What the plan knows of the sequence at a place (workspace).  `first` is its position in the free list of the first block it
// takes (the next ones lie in front of it) or -1: it is not served.
struct __align__(16) PlanEntry {
    int32_t sequence, pool, cached, held;
    int32_t fresh, need, first, leads;      // leads: the pool's first place
};
template <typename T> __device__ __forceinline__ T warp_sum_up_to(T x)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T t = __shfl_up_sync(FULL, x, o);
        if (lane >= o) x += t;
    }
    return x;
}
// Running sums that stop at 2^31 - 1: entries behind that have no place in any output.
__device__ __forceinline__ uint32_t add_up(uint32_t a, uint32_t b) { return min(a + b, 0x7FFFFFFFu); }
__device__ __forceinline__ uint32_t warp_add_up_to(uint32_t x)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(FULL, x, o);
        if (lane >= o) x = add_up(x, t);
    }
    return x;
}
__device__ __forceinline__ long long warp_total(long long x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
    return x;
}

// Sequence b's pool, or n_pools: it takes no part.
__device__ __forceinline__ int pool_of(const CachePlanParams &p, int b, uint32_t &flags)
{
    if (!p.pool) return 0;
    const int g = __ldg(p.pool + b);
    if (g >= p.c.n_pools) flags |= METASD_STATUS_BAD_INDEX;
    return g < 0 || g >= p.c.n_pools ? p.c.n_pools : g;
}

// First entries by place, in shared memory where they fit.
struct InShared {
    const int32_t *at;
    __device__ __forceinline__ int operator[](int i) const { return at[i]; }
};
struct InGlobal {
    const int32_t *at;
    __device__ __forceinline__ int operator[](int i) const { return __ldcg(at + i); }
};
// The last place from lo on (token_start[lo] <= t) that starts at or in front of entry t: entry t is its.
template <typename Starts> __device__ __forceinline__ int place_of(const Starts &token_start, int lo, int batch, int t)
{
    int hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (token_start[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The entries of one place.  The first entry of a block that is taken writes the block table.
struct Place {
    int sequence, cached, held;
    bool planned;
    int32_t *table;             // the sequence's row of the block table
    const int32_t *taken;       // taken[-block]: block `block` of the row, where it is taken from the free list

    __device__ __forceinline__ void at(const CachePlanParams &p, const PlanEntry &e)
    {
        sequence = e.sequence;
        cached = e.cached;
        held = e.held;
        planned = e.first != -1;
        table = p.c.block_table + ((int64_t)e.pool * p.c.max_batch + e.sequence) * p.c.max_blocks;
        taken = p.c.free_blocks + (int64_t)e.pool * p.c.n_blocks + ((int64_t)e.held + e.first);
    }
    __device__ __forceinline__ int id(int block) const { return planned ? *(block >= held ? taken - block : table + block) : 0; }
    __device__ __forceinline__ void note(int block, int id) const
    {
        if (planned && block >= held) table[block] = id;
    }
    __device__ __forceinline__ long long slot(const CachePlanParams &p, int id, int in) const
    {
        return planned ? (long long)id * p.c.page_size + in : -1;
    }
};

// Two entries that lie next to each other.
struct Two {
    long long slot, slot1;
    int position, position1, sequence, sequence1;
};
__device__ __forceinline__ void put(const CachePlanParams &p, int t, int end, const Two &e)
{
    if (p.wide && t + 1 < end) {
        *reinterpret_cast<longlong2 *>(p.slot_map + t) = make_longlong2(e.slot, e.slot1);
        if (p.position) *reinterpret_cast<int2 *>(p.position + t) = make_int2(e.position, e.position1);
        if (p.sequence) *reinterpret_cast<int2 *>(p.sequence + t) = make_int2(e.sequence, e.sequence1);
        return;
    }
    p.slot_map[t] = e.slot;
    if (p.position) p.position[t] = e.position;
    if (p.sequence) p.sequence[t] = e.sequence;
    if (t + 1 >= end) return;
    p.slot_map[t + 1] = e.slot1;
    if (p.position) p.position[t + 1] = e.position1;
    if (p.sequence) p.sequence[t + 1] = e.sequence1;
}

// Entries begin .. end - 1, by one block, two to a thread at a time; a thread's next two are often of the same sequence.
template <int THREADS, typename Starts>
__device__ __forceinline__ void fill(const CachePlanParams &p, const PlanEntry *entries, const Starts &token_start, int begin, int end)
{
    Place x;
    int from = 0, to = 0, at = 0;       // the entries of the place
    const int page = p.c.page_size;
    auto find = [&](int t) {
        at = place_of(token_start, at, p.batch, t);
        from = token_start[at];
        to = token_start[at + 1];
        x.at(p, entries[at]);
    };
    auto split = [&](int position, int &block, int &in) {
        block = divide(position, page, p.page_inverse);
        in = position - block * page;
    };
    for (long long next = begin + 2 * (int)threadIdx.x; next < end; next += 2 * THREADS) {
        const int t = (int)next;
        if (t >= to) find(t);
        Two e;
        int block, in;
        e.position = x.cached + (t - from);
        e.sequence = x.sequence;
        split(e.position, block, in);
        int id = x.id(block);
        if (in == 0) x.note(block, id);
        e.slot = x.slot(p, id, in);
        e.slot1 = 0;
        e.position1 = e.sequence1 = 0;
        if (t + 1 < end) {
            if (t + 1 >= to) {
                find(t + 1);
                e.position1 = x.cached;
                split(e.position1, block, in);
                id = x.id(block);
            } else {
                e.position1 = e.position + 1;
                if (++in == page) {
                    ++block;
                    in = 0;
                    id = x.id(block);
                }
            }
            if (in == 0) x.note(block, id);
            e.sequence1 = x.sequence;
            e.slot1 = x.slot(p, id, in);
        }
        put(p, t, end, e);
    }
}

// The same, an entry to a thread, where there are enough of them: a second entry of another sequence is a second chain of loads.
template <int THREADS, typename Starts>
__device__ __forceinline__ void fill_singly(const CachePlanParams &p, const PlanEntry *entries, const Starts &token_start, int begin, int end)
{
    for (int t = begin + (int)threadIdx.x; t < end; t += THREADS) {
        const int at = place_of(token_start, 0, p.batch, t);
        Place x;
        x.at(p, entries[at]);
        const int position = x.cached + (t - token_start[at]), block = divide(position, p.c.page_size, p.page_inverse);
        const int in = position - block * p.c.page_size, id = x.id(block);
        if (in == 0) x.note(block, id);
        p.slot_map[t] = x.slot(p, id, in);
        if (p.position) p.position[t] = position;
        if (p.sequence) p.sequence[t] = x.sequence;
    }
}

// Shared memory of the first kernel.
template <int THREADS> struct PlanShared {
    int tally[KEYS][MOST_WARPS];        // sequences of a pool in front of a warp's, then the places behind them
    int total[KEYS];
    int start[KEYS + 1];
    long long need[MOST_WARPS];
    uint32_t tokens[MOST_WARPS];
    long long base[KEYS];               // running sum of the blocks at a pool's first place
    int free[KEYS], taken[KEYS];
    int token_start[STARTS + 1];
    PlanEntry entries[THREADS];         // by place, where a thread has one sequence
};

// The sequence's entry of the plan, as far as it is known without the others.
__device__ __forceinline__ PlanEntry plan_entry(const CachePlanParams &p, int b, int g, uint32_t &flags)
{
    const metasd_cache &c = p.c;
    PlanEntry e = {b, g, 0, 0, 0, 0, -1, 0};
    if (g >= c.n_pools) return e;
    const int cached = __ldg(p.cached + g * p.cached_pool + b), length = __ldg(p.length + b), held = c.held[(int64_t)g * c.max_batch + b];
    const int kept = min(max(held, 0), c.max_blocks);
    if (kept != held) flags |= METASD_STATUS_BAD_STATE;
    // a cache that the table does not cover, or a length that it cannot: nothing is planned
    const bool bad = cached < 0 || length < 0 || (int64_t)cached > (int64_t)kept * c.page_size || (int64_t)length > (int64_t)c.max_blocks * c.page_size;
    if (bad) {
        flags |= METASD_STATUS_BAD_LENGTH;
        return e;
    }
    e.cached = cached;
    e.held = kept;
    e.fresh = max(length - cached, 0);
    if (e.fresh) e.need = max(divide(length - 1, c.page_size, p.page_inverse) + 1 - kept, 0);
    return e;
}

// What the sums say about the place: whether it is planned, and from where in the free list it takes its blocks.
template <int THREADS>
__device__ __forceinline__ void serve(const CachePlanParams &p, PlanShared<THREADS> &sh, PlanEntry &e, int at, uint32_t start, long long before, uint32_t &flags)
{
    const metasd_cache &c = p.c;
    const uint32_t end = add_up(start, (uint32_t)e.fresh);
    p.token_start[at] = (int32_t)start;
    if (at == p.batch - 1) p.token_start[p.batch] = (int32_t)end;
    if (at <= STARTS) sh.token_start[at] = (int32_t)start;
    if (at == p.batch - 1 && at < STARTS) sh.token_start[p.batch] = (int32_t)end;
    if (e.fresh) {
        const bool room = (long long)start + e.fresh <= p.max_tokens, enough = e.need == 0 || before + e.need <= sh.free[e.pool];
        if (!room) flags |= METASD_STATUS_TRUNCATED;
        if (!enough) flags |= METASD_STATUS_NO_BLOCKS;
        if (room && enough) {
            e.first = e.need ? sh.free[e.pool] - 1 - (int)before : 0;
            if (e.need) {
                atomicMax(sh.taken + e.pool, (int)(before + e.need));
                c.held[(int64_t)e.pool * c.max_batch + e.sequence] = e.held + e.need;
            }
        }
    }
}

// The free lists' lengths, and none taken yet.
template <int THREADS> __device__ __forceinline__ void look_at_pools(const CachePlanParams &p, PlanShared<THREADS> &sh, uint32_t &flags)
{
    for (int i = threadIdx.x; i < p.c.n_pools; i += THREADS) {
        const int free = p.c.free_count[i];
        sh.free[i] = min(max(free, 0), p.c.n_blocks);
        sh.taken[i] = 0;
        if (sh.free[i] != free) flags |= METASD_STATUS_BAD_STATE;
    }
}

// Order, running sums and the block tables' growth of a step, by one block with a sequence (then a place) per thread, in registers
// and shared memory; the blocks of all tables together are fewer than 2^31.
template <int THREADS> __device__ __forceinline__ void plan_step(const CachePlanParams &p, PlanShared<THREADS> &sh)
{
    constexpr int WARPS = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batch = p.batch, P = p.c.n_pools;
    const bool in = tid < batch;
    uint32_t flags = 0;
    PlanEntry e = {tid, P, 0, 0, 0, 0, -1, 0};
    if (in) e = plan_entry(p, tid, pool_of(p, tid, flags), flags);
    look_at_pools<THREADS>(p, sh, flags);
    if (p.pool) {       // order by pool: a counting sort
        for (int g = lane; g <= P; g += 32) sh.tally[g][warp] = 0;
        __syncwarp();
        const unsigned same = __match_any_sync(FULL, in ? e.pool : -1);
        const int rank = __popc(same & ((1u << lane) - 1u));
        if (in && rank == 0) sh.tally[e.pool][warp] = __popc(same);
        __syncthreads();
        for (int g = warp; g <= P; g += WARPS) {
            const int x = lane < WARPS ? sh.tally[g][lane] : 0, upto = warp_sum_up_to(x);
            if (lane < WARPS) sh.tally[g][lane] = upto - x;
            if (lane == 31) sh.total[g] = upto;
        }
        __syncthreads();
        const int x = lane < P ? sh.total[lane] : 0, upto = warp_sum_up_to(x);
        const int start = __shfl_sync(FULL, upto - x, e.pool & 31), behind = __shfl_sync(FULL, upto, 31);
        if (in) {
            const int at = (e.pool < P ? start : behind) + sh.tally[e.pool][warp] + rank;
            e.leads = e.pool < P && at == start;
            sh.entries[at] = e;
            if (p.order) p.order[at] = tid;
            if (p.place) p.place[tid] = at;
        }
        if (p.pool_start && warp == 0) {
            if (lane < P) p.pool_start[lane] = upto - x;
            if (lane == 0) p.pool_start[P] = behind;
        }
        __syncthreads();
        if (in) e = sh.entries[tid];
    } else {
        if (in && p.order) p.order[tid] = tid;
        if (in && p.place) p.place[tid] = tid;
        if (p.pool_start && tid <= P) p.pool_start[tid] = tid == 0 ? 0 : batch;
    }
    // running sums of the entries and of the blocks
    const uint32_t tokens = in ? (uint32_t)e.fresh : 0u, upto_tokens = warp_add_up_to(tokens);
    const int need = in ? e.need : 0, upto_need = warp_sum_up_to(need);      // p.narrow: they fit
    if (lane == 31) { sh.tokens[warp] = upto_tokens; sh.need[warp] = upto_need; }
    __syncthreads();
    const uint32_t tokens_w = warp_add_up_to(lane < WARPS ? sh.tokens[lane] : 0u);
    const int need_w = warp_sum_up_to(lane < WARPS ? (int)sh.need[lane] : 0);
    uint32_t tokens0 = __shfl_sync(FULL, tokens_w, (warp + 31) & 31), before_lane = __shfl_up_sync(FULL, upto_tokens, 1);
    int need0 = __shfl_sync(FULL, need_w, (warp + 31) & 31);
    if (warp == 0) { tokens0 = 0u; need0 = 0; }
    if (lane == 0) before_lane = 0u;
    const int blocks = need0 + upto_need - need;
    if (p.pool) {
        if (in && e.leads) sh.base[e.pool] = blocks;
        __syncthreads();
    }
    if (in) {
        serve(p, sh, e, tid, add_up(tokens0, before_lane), p.pool && e.fresh ? blocks - (int)sh.base[e.pool] : blocks, flags);
        sh.entries[tid] = e;
        ((PlanEntry *)p.c.workspace)[tid] = e;
    }
    flags = __reduce_or_sync(FULL, flags);
    if (flags && lane == 0 && p.c.status) atomicOr(p.c.status, flags);
    __syncthreads();
    for (int i = tid; i < P; i += THREADS) p.c.free_count[i] = sh.free[i] - sh.taken[i];
}

// The same for any number of sequences and blocks: a warp takes rows of 32, one behind the other, through the workspace.
__device__ __forceinline__ void plan_rows(const CachePlanParams &p, PlanShared<MOST_THREADS> &sh)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batch = p.batch, P = p.c.n_pools;
    PlanEntry *entries = (PlanEntry *)p.c.workspace;
    uint32_t flags = 0;
    for (int i = tid; i < (P + 1) * MOST_WARPS; i += MOST_THREADS) (&sh.tally[0][0])[i] = 0;
    look_at_pools<MOST_THREADS>(p, sh, flags);
    __syncthreads();
    const int rows = (batch + 31) / 32, row0 = rows * warp / MOST_WARPS, row1 = rows * (warp + 1) / MOST_WARPS;
    for (int row = row0; row < row1; ++row) {
        const int b = row * 32 + lane, g = b < batch ? pool_of(p, b, flags) : -1;
        const unsigned same = __match_any_sync(FULL, g);
        if (b < batch && lane == __ffs(same) - 1) sh.tally[g][warp] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    for (int g = warp; g <= P; g += MOST_WARPS) {
        const int x = sh.tally[g][lane], upto = warp_sum_up_to(x);
        sh.tally[g][lane] = upto - x;
        if (lane == 31) sh.total[g] = upto;
    }
    __syncthreads();
    if (warp == 0) {
        const int x = lane < P ? sh.total[lane] : 0, upto = warp_sum_up_to(x);
        if (lane < P) sh.start[lane] = upto - x;
        if (lane == 31) sh.start[P] = upto;
        if (p.pool_start && lane < P) p.pool_start[lane] = upto - x;
        if (p.pool_start && lane == 31) p.pool_start[P] = upto;
    }
    __syncthreads();
    for (int row = row0; row < row1; ++row) {
        const int b = row * 32 + lane;
        uint32_t seen = 0;
        const int g = b < batch ? pool_of(p, b, seen) : -1;
        const unsigned same = __match_any_sync(FULL, g);
        int at = 0;
        if (b < batch) at = sh.start[g] + sh.tally[g][warp] + __popc(same & ((1u << lane) - 1u));
        __syncwarp();
        if (b < batch) {
            if (lane == __ffs(same) - 1) sh.tally[g][warp] += __popc(same);
            entries[at] = plan_entry(p, b, g, flags);
            if (p.order) p.order[at] = b;
            if (p.place) p.place[b] = at;
        }
        __syncwarp();
    }
    __syncthreads();
    uint32_t tokens = 0;
    long long need = 0;
    for (int row = row0; row < row1; ++row) {
        const int at = row * 32 + lane;
        if (at < batch) {
            tokens = add_up(tokens, (uint32_t)entries[at].fresh);
            need += entries[at].need;
        }
    }
    tokens = warp_add_up_to(tokens);
    need = warp_sum_up_to(need);
    if (lane == 31) { sh.tokens[warp] = tokens; sh.need[warp] = need; }
    __syncthreads();
    const uint32_t tokens_w = warp_add_up_to(sh.tokens[lane]);
    const long long need_w = warp_sum_up_to(sh.need[lane]);
    tokens = __shfl_sync(FULL, tokens_w, (warp + 31) & 31);
    need = __shfl_sync(FULL, need_w, (warp + 31) & 31);
    if (warp == 0) { tokens = 0u; need = 0; }
    long long run = need;
    for (int row = row0; row < row1; ++row) {
        const int at = row * 32 + lane;
        const int n = at < batch ? entries[at].need : 0;
        const long long upto = warp_sum_up_to((long long)n);
        if (at < batch) {
            const int g = entries[at].pool;
            if (g < P && at == sh.start[g]) sh.base[g] = run + upto - n;
        }
        run += __shfl_sync(FULL, upto, 31);
    }
    __syncthreads();
    for (int row = row0; row < row1; ++row) {
        const int at = row * 32 + lane;
        PlanEntry e = {0, P, 0, 0, 0, 0, -1, 0};
        if (at < batch) e = entries[at];
        const uint32_t upto_t = warp_add_up_to((uint32_t)e.fresh);
        const long long upto_n = warp_sum_up_to((long long)e.need);
        uint32_t before_lane = __shfl_up_sync(FULL, upto_t, 1);
        if (lane == 0) before_lane = 0u;
        if (at < batch) {
            serve(p, sh, e, at, add_up(tokens, before_lane), e.fresh ? need + upto_n - e.need - sh.base[e.pool] : 0, flags);
            entries[at].first = e.first;
        }
        tokens = add_up(tokens, __shfl_sync(FULL, upto_t, 31));
        need += __shfl_sync(FULL, upto_n, 31);
    }
    flags = __reduce_or_sync(FULL, flags);
    if (flags && lane == 0 && p.c.status) atomicOr(p.c.status, flags);
    __syncthreads();
    for (int i = tid; i < P; i += MOST_THREADS) p.c.free_count[i] = sh.free[i] - sh.taken[i];
}

// FILLS: a cluster; its first block plans, then all of them write the entries.
template <int THREADS, bool FILLS> __global__ void __launch_bounds__(THREADS) plan_kernel(const CachePlanParams p)
{
    __shared__ PlanShared<THREADS> sh;
    launch_dependents();
    grid_dependency_wait();
    const int rank = FILLS ? (int)cluster_rank() : 0, batch = p.batch;
    if (rank == 0) {
        if constexpr (THREADS == MOST_THREADS) {
            if (p.narrow && batch <= THREADS) plan_step<THREADS>(p, sh);
            else plan_rows(p, sh);
        } else {
            plan_step<THREADS>(p, sh);
        }
    }
    if constexpr (FILLS) {
        const int ranks = (int)cluster_size();
        if (ranks > 1) cluster_sync_all();
        const bool near = batch <= STARTS;
        if (near && rank != 0) {
            for (int i = threadIdx.x; i <= batch; i += THREADS) sh.token_start[i] = __ldcg(p.token_start + i);
            __syncthreads();
        }
        const PlanEntry *entries = rank == 0 && p.narrow && batch <= THREADS ? sh.entries : (const PlanEntry *)p.c.workspace;
        // a stretch each, of the entries that there are
        const int total = min(near ? sh.token_start[batch] : __ldcg(p.token_start + batch), p.max_tokens);
        const int each = (total / ranks / 32 + 1) * 32;
        const long long begin = (long long)each * rank;
        const int end = (int)min(begin + each, (long long)total);
        if (begin >= total) return;
        if (near) fill_singly<THREADS>(p, entries, InShared{sh.token_start}, (int)begin, end);
        else fill_singly<THREADS>(p, entries, InGlobal{p.token_start}, (int)begin, end);
    }
}

// Each block a stretch of its own, of the entries that there are: one search and a walk.
__global__ void __launch_bounds__(FILL_THREADS, FILL_BLOCKS) fill_kernel(const CachePlanParams p)
{
    __shared__ int32_t sh_start[STARTS + 1];
    launch_dependents();
    grid_dependency_wait();
    const PlanEntry *entries = (const PlanEntry *)p.c.workspace;
    const bool near = p.batch <= STARTS;
    const int total = min(__ldcg(p.token_start + p.batch), p.max_tokens);
    const bool few = total <= (long long)gridDim.x * FILL_THREADS;      // an entry to a thread
    const long long turn = few ? 32 : 2 * FILL_THREADS, turns = (total + turn - 1) / turn, each = (turns + gridDim.x - 1) / gridDim.x * turn;
    const long long begin = each * blockIdx.x;
    if (begin >= total) return;
    if (near) {
        for (int i = threadIdx.x; i <= p.batch; i += FILL_THREADS) sh_start[i] = __ldcg(p.token_start + i);
        __syncthreads();
    }
    const int end = (int)min(begin + each, (long long)total);
    auto write = [&](const auto &starts) {
        if (few) fill_singly<FILL_THREADS>(p, entries, starts, (int)begin, end);
        else fill<FILL_THREADS>(p, entries, starts, (int)begin, end);
    };
    if (near) write(InShared{sh_start});
    else write(InGlobal{p.token_start});
}

// A cluster per pool.  A warp takes a row of 32 sequences, or several, one behind the other; where there are more warps than rows,
// several share a row's blocks.  A few blocks are copied over all lanes at once, whatever sequence they come from; many one sequence after
// the other, with less to do for each.
constexpr int RELEASE_CLUSTER = 8, RELEASE_GROUPS = RELEASE_CLUSTER * MOST_WARPS, AT_ONCE = 4;
constexpr int LONG = 1024;      // blocks of a table from which a release takes all the warps there are
constexpr int MANY = 256;       // blocks that a row of sequences gives back: 1024 x 96 37.4 -> 35.2 us a plan and release; 64 .. 1024 as good

template <int THREADS> __global__ void __launch_bounds__(THREADS) release_kernel(const CacheReleaseParams p)
{
    __shared__ long long sh_drop[RELEASE_GROUPS];       // the warps' sums, of the whole cluster
    launch_dependents();
    grid_dependency_wait();
    const metasd_cache &c = p.c;
    const int ranks = (int)cluster_size(), rank = (int)cluster_rank();
    const int g = (int)blockIdx.x / ranks, lane = threadIdx.x & 31, batch = p.batch;
    const int warps = ranks * (THREADS / 32), w = rank * (THREADS / 32) + (int)(threadIdx.x >> 5);
    // p.share warps to a row, or p.share == 0 and several rows to a warp
    const int rows = (batch + 31) / 32, share = max(p.share, 1), group = p.share > 1 ? divide(w, share, p.share_inverse) : w, sub = w - group * share;
    const int groups = p.share ? min(rows, warps) : warps, each = p.share ? 1 : (rows + warps - 1) / warps;
    const int row0 = min(group * each, rows), row1 = min(row0 + each, rows);
    const int32_t *keep = p.keep + g * p.keep_pool;
    int32_t *held = c.held + (int64_t)g * c.max_batch;
    const int32_t *tables = c.block_table + (int64_t)g * c.max_batch * c.max_blocks;
    int32_t *list = c.free_blocks + (int64_t)g * c.n_blocks;
    const int count = c.free_count[g], free = min(max(count, 0), c.n_blocks);
    uint32_t flags = free != count ? METASD_STATUS_BAD_STATE : 0u;
    // blocks that the row's sequences give back, a lane each, and the first of them
    auto look = [&](int row, int &from) {
        const int b = row * 32 + lane;
        from = 0;
        if (b >= batch) return 0;
        const int has = held[b], kept = min(max(has, 0), c.max_blocks), length = __ldg(keep + b);
        if (kept != has) flags |= METASD_STATUS_BAD_STATE;
        if (length < 0) flags |= METASD_STATUS_BAD_LENGTH;
        if (length > 0) from = divide(length - 1, c.page_size, p.page_inverse) + 1;
        return length < 0 ? 0 : max(kept - from, 0);
    };
    int from = 0, drop = 0;
    long long mine = 0;
    for (int row = row0; row < row1; ++row) {
        drop = look(row, from);
        mine += drop;
    }
    mine = warp_total(mine);
    cluster_arrive_relaxed();
    cluster_wait();             // every block of the cluster runs
    if (sub == 0 && lane < ranks && group < groups) {
        const uint32_t to = map_to_rank(smem_addr(sh_drop + group), (uint32_t)lane);
        asm volatile("st.shared::cluster.s64 [%0], %1;" ::"r"(to), "l"(mine) : "memory");
    }
    cluster_sync_all();         // the sums are there, and everyone has read what is changed below
    long long before = 0, total = 0;
    for (int i = lane; i < groups; i += 32) {
        total += sh_drop[i];
        if (i < group) before += sh_drop[i];
    }
    total = warp_total(total);
    before = warp_total(before);
    const bool fits = free + total <= c.n_blocks;       // else the tables hold what was not taken from here: nothing is given back
    if (!fits) flags |= METASD_STATUS_BAD_STATE;
    if (fits && group < groups) {
        for (int row = row0; row < row1; ++row) {
            if (row1 - row0 > 1) drop = look(row, from);
            const int upto = warp_sum_up_to(drop), n = __shfl_sync(FULL, upto, 31);
            const long long top = free + total - 1 - before;
            for (int e0 = 32 * sub; e0 < n && n < MANY; e0 += 32 * share * AT_ONCE) {
                int id[AT_ONCE];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    const int e = e0 + 32 * share * i + lane;
                    int owner = 0;          // the lane whose blocks hold entry e: the first that ends behind it
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1)
                        if (__shfl_sync(FULL, upto, owner + o - 1) <= e) owner += o;
                    owner = min(owner, 31);
                    const int place = __shfl_sync(FULL, from - (upto - drop), owner) + e;
                    id[i] = e < n ? tables[(int64_t)(row * 32 + owner) * c.max_blocks + place] : 0;
                }
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    const int e = e0 + 32 * share * i + lane;
                    if (e < n) list[top - e] = id[i];
                }
            }
            if (n >= MANY) {
                // Much to give back: the row's warps take a sequence each, and share those that are more than twice a warp's part.
                auto give = [&](int s, uint32_t begin, uint32_t by) {      // unsigned: four steps beyond 2^31 - 1 blocks are below 2^32
                    const uint32_t d = __shfl_sync(FULL, drop, s);
                    const int ahead = __shfl_sync(FULL, upto - drop, s), first = __shfl_sync(FULL, from, s);
                    const int32_t *source = tables + (int64_t)(row * 32 + s) * c.max_blocks + first;
                    int32_t *to = list + (top - ahead);
                    for (uint32_t e0 = begin; e0 < d; e0 += by * AT_ONCE) {
                        int id[AT_ONCE];
#pragma unroll
                        for (int i = 0; i < AT_ONCE; ++i) id[i] = e0 + by * i < d ? source[e0 + by * i] : 0;
#pragma unroll
                        for (int i = 0; i < AT_ONCE; ++i)
                            if (e0 + by * i < d) to[-(int64_t)(e0 + by * i)] = id[i];
                    }
                };
                unsigned shared = __ballot_sync(FULL, (long long)drop * share > 2ll * n);
                for (int s = sub; s < 32; s += share)
                    if (!(shared >> s & 1u)) give(s, lane, 32);
                for (; shared; shared &= shared - 1u) give(__ffs(shared) - 1, lane + 32 * sub, 32 * share);
            }
            before += n;
            __syncwarp();
            if (sub == 0 && drop > 0) held[row * 32 + lane] = from;
        }
    }
    flags = __reduce_or_sync(FULL, flags);
    if (flags && lane == 0 && c.status) atomicOr(c.status, flags);
    if (w == 0 && lane == 0 && (fits || free != count)) c.free_count[g] = fits ? free + (int)total : free;
}

}  // namespace

size_t cache_workspace_bytes(int max_batch, int n_pools) { return (size_t)max_batch * sizeof(PlanEntry); }

// Up to so many entries (that the outputs have room for) the planning cluster writes them too.  Us a plan and release on the device with one
// launch and with two, and the entries there is room for and there are: 1024 sequences, 9216 and 5 k, 11.1 and 11.2 (a launch takes the host
// 2.2 us besides); 333 sequences, 62 k and 16 k, 12.6 and 10.5; 256 sequences, 87 k and 26 k, 18.6 and 10.2.
constexpr int ALONE_ENTRIES = 16384, PLAN_CLUSTER = 8;
// Releases of so many sequences take blocks of 256 threads, of more 1024: fewer warps are quicker where little comes back (1024
// sequences, 10.4 us a plan and release instead of 11.1), more where much does (1024 x 96 blocks: 35.4 us instead of 41.5), or may: tables
// of more than LONG blocks take all there is (45 sequences, tables of 10 k blocks, of which 70 k come back: 14.3 us instead of 48).
constexpr int SMALL_RELEASE = 512;

cudaError_t launch_cache_plan(const CachePlanParams &params, int n_sm, cudaStream_t stream)
{
    CachePlanParams p = params;
    p.narrow = (long long)p.batch * p.c.max_blocks < (1ll << 31);
    const bool small = p.narrow && p.batch <= 256;
    if (p.max_tokens <= ALONE_ENTRIES) {
        const int threads = small ? 256 : MOST_THREADS;
        int cluster = 1;
        while (cluster < PLAN_CLUSTER && cluster * threads < p.max_tokens) cluster *= 2;
        return small ? launch_kernel(plan_kernel<256, true>, (unsigned)cluster, 256, 0, cluster, true, stream, p)
                     : launch_kernel(plan_kernel<MOST_THREADS, true>, (unsigned)cluster, MOST_THREADS, 0, cluster, true, stream, p);
    }
    cudaError_t e = small ? launch_kernel(plan_kernel<256, false>, 1, 256, 0, 1, true, stream, p)
                          : launch_kernel(plan_kernel<MOST_THREADS, false>, 1, MOST_THREADS, 0, 1, true, stream, p);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)std::min<long long>(((long long)p.max_tokens + FILL_THREADS - 1) / FILL_THREADS, (long long)FILL_BLOCKS * n_sm);
    return launch_kernel(fill_kernel, grid, FILL_THREADS, 0, 1, true, stream, p);
}

cudaError_t launch_cache_release(const CacheReleaseParams &params, cudaStream_t stream)
{
    CacheReleaseParams p = params;
    const int rows = (p.batch + 31) / 32;
    const bool small = p.batch <= SMALL_RELEASE && p.c.max_blocks <= LONG;
    int cluster = p.c.max_blocks <= LONG ? 1 : RELEASE_CLUSTER;
    while (cluster < RELEASE_CLUSTER && cluster * (small ? 32 : 128) < p.batch) cluster *= 2;
    p.share = cluster * (small ? 8 : MOST_WARPS) / rows;
    p.share_inverse = inverse_of((uint32_t)std::max(p.share, 1));
    return small ? launch_kernel(release_kernel<256>, (unsigned)(p.c.n_pools * cluster), 256, 0, cluster, true, stream, p)
                 : launch_kernel(release_kernel<MOST_THREADS>, (unsigned)(p.c.n_pools * cluster), MOST_THREADS, 0, cluster, true, stream, p);
}

}  // namespace metasd
