// metasd_cache_plan / metasd_cache_release: where the next entries of paged caches go.
//
// A sequence adds new = max(0, length - cached) entries to the cache of the model (pool) it runs on.  Sequences are ordered by
// pool, in sequence order within each; with token_start the running sum of `new` in that order, entry t of the packed step belongs
// to the place at with token_start[at] <= t < token_start[at + 1], has position cached + t - token_start[at] and the slot
//     block_table[pool][sequence][position / page] * page + position % page.
// A sequence whose table is too short takes need = ceil(length / page) - held blocks from the end of its pool's free list, behind
// what the sequences before it take: running sums again.
//
// Two kernels.  The sums are one block's work: it reads some 20 bytes a sequence, and what it costs is the latency of its steps.
// The entries are spread over the whole GPU and bound by the 16 bytes that are written for each.  A step whose buffers have room
// for few entries is done by the first kernel alone.
#include <algorithm>

#include "metasd_staged.cuh"

namespace metasd {

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_WARPS = PLAN_THREADS / 32;
constexpr int KEYS = METASD_MAX_POOLS + 1;      // the pools, and who takes no part
constexpr int FILL_THREADS = 256;
constexpr int SPAN = 2048;                      // entries that a block deals with at once
constexpr int RELEASE_THREADS = 1024, RELEASE_WARPS = RELEASE_THREADS / 32;
constexpr unsigned FULL = 0xFFFFFFFFu;

// What the plan knows of the sequence at a place (workspace).  `first` is its position in the free list of the first block it
// takes (the next ones lie in front of it) or -1: it is not served.
struct __align__(16) PlanEntry {
    int32_t sequence, pool, cached, held;
    int32_t fresh, need, first, unused;
};
// A sequence's part of a release (workspace): `drop` blocks from `from` on go to `to`, `to - 1`, .. of the pool's free list.
struct __align__(16) ReleaseEntry {
    int32_t from, drop, to, unused;
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

// The places of a span's entries, by one block: sh_at[i] = place of entry `begin + i`.
template <int THREADS>
__device__ __forceinline__ void places_of_span(const int32_t *token_start, int batch, int begin, int end, int *sh_at, int *sh_warp)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int PER = SPAN / THREADS;
    // the last place that starts at or in front of `begin` (every warp looks for itself): 32 probes a step
    int lo = 0, hi = batch;     // token_start[lo] <= begin, and < token_start[hi] or hi == batch
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int at = min(lo + lane * step, hi);
        const unsigned below = __ballot_sync(FULL, at < hi && __ldcg(token_start + at) <= begin);
        const int last = 31 - __clz(below);     // lane 0 always is
        hi = min(lo + (last + 1) * step, hi);
        lo = lo + last * step;
    }
    for (int i = tid; i < SPAN; i += THREADS) sh_at[i] = 0;
    __syncthreads();
    if (tid == 0) sh_at[0] = lo;
    __syncthreads();
    // every place that starts inside the span marks its first entry; the largest of those that start together has entries
    for (int at = lo + 1 + tid; at < batch; at += THREADS) {
        const int start = __ldcg(token_start + at);
        if (start >= end) break;
        atomicMax(sh_at + (start - begin), at);
    }
    __syncthreads();
    // running maximum
    int mine[PER], top = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        top = max(top, sh_at[tid * PER + i]);
        mine[i] = top;
    }
    int upto = top;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(FULL, upto, o);
        if (lane >= o) upto = max(upto, t);
    }
    if (lane == 31) sh_warp[warp] = upto;
    int before = __shfl_up_sync(FULL, upto, 1);
    if (lane == 0) before = 0;
    __syncthreads();
    for (int w = 0; w < warp; ++w) before = max(before, sh_warp[w]);
#pragma unroll
    for (int i = 0; i < PER; ++i) sh_at[tid * PER + i] = max(mine[i], before);
    __syncthreads();
}

// Entry t: its slot, position and sequence.  The first entry of a block that is taken writes the block table.
struct Entry {
    long long slot;
    int position, sequence;
};
__device__ __forceinline__ Entry entry_at(const CachePlanParams &p, const PlanEntry *entries, const int32_t *token_start, int at, int t)
{
    const metasd_cache &c = p.c;
    const PlanEntry e = entries[at];
    Entry r;
    r.sequence = e.sequence;
    r.position = e.cached + (t - token_start[at]);
    r.slot = -1;
    if (e.first != -1) {
        const int block = divide(r.position, c.page_size, p.page_inverse), in = r.position - block * c.page_size;
        int32_t *table = c.block_table + ((int64_t)e.pool * c.max_batch + e.sequence) * c.max_blocks;
        int id;
        if (block >= e.held) {
            id = c.free_blocks[(int64_t)e.pool * c.n_blocks + (e.first - (block - e.held))];
            if (in == 0) table[block] = id;
        } else {
            id = table[block];
        }
        r.slot = (long long)id * c.page_size + in;
    }
    return r;
}

template <int THREADS>
__device__ __forceinline__ void fill_span(const CachePlanParams &p, int begin, int end, int *sh_at, int *sh_warp)
{
    const PlanEntry *entries = (const PlanEntry *)p.c.workspace;
    places_of_span<THREADS>(p.token_start, p.batch, begin, end, sh_at, sh_warp);
    for (int i = 2 * threadIdx.x; begin + i < end; i += 2 * THREADS) {
        const int t = begin + i;
        const Entry a = entry_at(p, entries, p.token_start, sh_at[i], t);
        if (t + 1 < end && p.wide) {
            const Entry b = entry_at(p, entries, p.token_start, sh_at[i + 1], t + 1);
            *reinterpret_cast<longlong2 *>(p.slot_map + t) = make_longlong2(a.slot, b.slot);
            if (p.position) *reinterpret_cast<int2 *>(p.position + t) = make_int2(a.position, b.position);
            if (p.sequence) *reinterpret_cast<int2 *>(p.sequence + t) = make_int2(a.sequence, b.sequence);
        } else {
            p.slot_map[t] = a.slot;
            if (p.position) p.position[t] = a.position;
            if (p.sequence) p.sequence[t] = a.sequence;
            if (t + 1 < end) {
                const Entry b = entry_at(p, entries, p.token_start, sh_at[i + 1], t + 1);
                p.slot_map[t + 1] = b.slot;
                if (p.position) p.position[t + 1] = b.position;
                if (p.sequence) p.sequence[t + 1] = b.sequence;
            }
        }
    }
}

template <bool ALONE> __global__ void __launch_bounds__(PLAN_THREADS) plan_kernel(const CachePlanParams p)
{
    __shared__ int sh_tally[KEYS][PLAN_WARPS];      // sequences of a pool in front of a warp's, then the places behind them
    __shared__ int sh_start[KEYS + 1];
    __shared__ long long sh_tokens[PLAN_WARPS], sh_need[PLAN_WARPS];
    __shared__ long long sh_base[KEYS];             // running sum of the blocks at a pool's first place
    __shared__ int sh_free[KEYS], sh_taken[KEYS];
    __shared__ int sh_at[ALONE ? SPAN : 1], sh_warp[PLAN_WARPS];
    __shared__ int sh_total;

    launch_dependents();
    grid_dependency_wait();
    const metasd_cache &c = p.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batch = p.batch, P = c.n_pools;
    PlanEntry *entries = (PlanEntry *)c.workspace;
    uint32_t flags = 0;
    for (int i = tid; i < KEYS * PLAN_WARPS; i += PLAN_THREADS) (&sh_tally[0][0])[i] = 0;
    for (int i = tid; i < P; i += PLAN_THREADS) {
        sh_free[i] = min(max(c.free_count[i], 0), c.n_blocks);
        sh_taken[i] = 0;
        if (sh_free[i] != c.free_count[i]) flags |= METASD_STATUS_BAD_STATE;
    }
    __syncthreads();

    // ---- order by pool: a warp takes rows of 32 sequences, one behind the other
    const int rows = (batch + 31) / 32, row0 = (int)((long long)rows * warp / PLAN_WARPS), row1 = (int)((long long)rows * (warp + 1) / PLAN_WARPS);
    for (int row = row0; row < row1; ++row) {
        const int b = row * 32 + lane;
        const unsigned here = __ballot_sync(FULL, b < batch);
        if (b < batch) {
            const int g = pool_of(p, b, flags);
            const unsigned same = __match_any_sync(here, g);
            if (lane == __ffs(same) - 1) sh_tally[g][warp] += __popc(same);
        }
        __syncwarp();
    }
    __syncthreads();
    for (int g = warp; g <= P; g += PLAN_WARPS) {
        const int x = sh_tally[g][lane], upto = warp_sum_up_to(x);
        sh_tally[g][lane] = upto - x;
        if (lane == 31) sh_start[g + 1] = upto;
    }
    __syncthreads();
    if (tid == 0) {
        sh_start[0] = 0;
        for (int g = 0; g <= P; ++g) sh_start[g + 1] += sh_start[g];
        if (p.pool_start)
            for (int g = 0; g <= P; ++g) p.pool_start[g] = sh_start[g];
    }
    __syncthreads();
    for (int row = row0; row < row1; ++row) {
        const int b = row * 32 + lane;
        const unsigned here = __ballot_sync(FULL, b < batch);
        int g = 0, at = 0;
        unsigned same = 0;
        if (b < batch) {
            uint32_t seen = 0;
            g = pool_of(p, b, seen);
            same = __match_any_sync(here, g);
            at = sh_start[g] + sh_tally[g][warp] + __popc(same & ((1u << lane) - 1u));
        }
        __syncwarp();
        if (b < batch) {
            if (lane == __ffs(same) - 1) sh_tally[g][warp] += __popc(same);
            PlanEntry e = {b, g, 0, 0, 0, 0, -1, 0};
            if (g < P) {
                const int64_t row_of = (int64_t)g * c.max_batch + b;
                const int cached = __ldg(p.cached + g * p.cached_pool + b), length = __ldg(p.length + b), held = c.held[row_of];
                const int kept = min(max(held, 0), c.max_blocks);
                if (kept != held) flags |= METASD_STATUS_BAD_STATE;
                // a cache that the table does not cover, or a length that it cannot: nothing is planned
                const bool bad = cached < 0 || length < 0 || (int64_t)cached > (int64_t)kept * c.page_size || (int64_t)length > (int64_t)c.max_blocks * c.page_size;
                if (bad) {
                    flags |= METASD_STATUS_BAD_LENGTH;
                } else {
                    e.cached = cached;
                    e.held = kept;
                    e.fresh = max(length - cached, 0);
                    if (e.fresh) e.need = max(divide(length - 1, c.page_size, p.page_inverse) + 1 - kept, 0);
                }
            }
            entries[at] = e;
            if (p.order) p.order[at] = b;
            if (p.place) p.place[b] = at;
        }
        __syncwarp();
    }
    __syncthreads();

    // ---- running sums of the entries and of the blocks, in that order
    long long tokens = 0, need = 0;
    for (int row = row0; row < row1; ++row) {
        const int at = row * 32 + lane;
        if (at < batch) {
            tokens += entries[at].fresh;
            need += entries[at].need;
        }
    }
    tokens = warp_total(tokens);
    need = warp_total(need);
    if (lane == 0) { sh_tokens[warp] = tokens; sh_need[warp] = need; }
    __syncthreads();
    {
        const long long t = sh_tokens[lane], n = sh_need[lane];
        const long long before_t = warp_sum_up_to(t) - t, before_n = warp_sum_up_to(n) - n;
        tokens = __shfl_sync(FULL, before_t, warp);
        need = __shfl_sync(FULL, before_n, warp);
    }
    const long long tokens0 = tokens, need0 = need;
    for (int row = row0; row < row1; ++row) {
        const int at = row * 32 + lane;
        const int n = at < batch ? entries[at].need : 0;
        const long long upto = warp_sum_up_to((long long)n);
        if (at < batch) {
            const int g = entries[at].pool;
            if (g < P && at == sh_start[g]) sh_base[g] = need + upto - n;
        }
        need += __shfl_sync(FULL, upto, 31);
    }
    __syncthreads();
    need = need0;
    tokens = tokens0;
    for (int row = row0; row < row1; ++row) {
        const int at = row * 32 + lane;
        const int fresh = at < batch ? entries[at].fresh : 0, n = at < batch ? entries[at].need : 0;
        const long long upto_t = warp_sum_up_to((long long)fresh), upto_n = warp_sum_up_to((long long)n);
        if (at < batch) {
            const int g = entries[at].pool;
            const long long start = tokens + upto_t - fresh;
            p.token_start[at] = (int32_t)min(start, 0x7FFFFFFFll);
            if (at == batch - 1) p.token_start[batch] = sh_total = (int32_t)min(start + fresh, 0x7FFFFFFFll);
            if (fresh) {
                const long long before = need + upto_n - n - sh_base[g];
                const bool room = start + fresh <= p.max_tokens, enough = n == 0 || before + n <= sh_free[g];
                if (!room) flags |= METASD_STATUS_TRUNCATED;
                if (!enough) flags |= METASD_STATUS_NO_BLOCKS;
                if (room && enough) {
                    entries[at].first = n ? sh_free[g] - 1 - (int)before : 0;
                    if (n) {
                        atomicMax(sh_taken + g, (int)(before + n));
                        c.held[(int64_t)g * c.max_batch + entries[at].sequence] = entries[at].held + n;
                    }
                }
            }
        }
        tokens += __shfl_sync(FULL, upto_t, 31);
        need += __shfl_sync(FULL, upto_n, 31);
    }
    flags = __reduce_or_sync(FULL, flags);
    if (flags && lane == 0 && c.status) atomicOr(c.status, flags);
    __syncthreads();
    for (int i = tid; i < P; i += PLAN_THREADS) c.free_count[i] = sh_free[i] - sh_taken[i];
    if constexpr (ALONE) {
        const int total = min(sh_total, p.max_tokens);
        for (int begin = 0; begin < total; begin += SPAN) {
            fill_span<PLAN_THREADS>(p, begin, min(begin + SPAN, total), sh_at, sh_warp);
            __syncthreads();
        }
    }
}

__global__ void __launch_bounds__(FILL_THREADS) fill_kernel(const CachePlanParams p)
{
    __shared__ int sh_at[SPAN], sh_warp[FILL_THREADS / 32];
    launch_dependents();
    grid_dependency_wait();
    const int total = min(p.token_start[p.batch], p.max_tokens);
    for (long long begin = (long long)blockIdx.x * SPAN; begin < total; begin += (long long)gridDim.x * SPAN) {
        fill_span<FILL_THREADS>(p, (int)begin, (int)min(begin + SPAN, (long long)total), sh_at, sh_warp);
        __syncthreads();
    }
}

// A block per pool: how many blocks each sequence gives back, and where to.
__global__ void __launch_bounds__(RELEASE_THREADS) release_kernel(const CacheReleaseParams p)
{
    __shared__ long long sh_drop[RELEASE_WARPS];
    __shared__ int sh_total;
    launch_dependents();
    grid_dependency_wait();
    const metasd_cache &c = p.c;
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batch = p.batch;
    ReleaseEntry *entries = (ReleaseEntry *)c.workspace + (int64_t)g * c.max_batch;
    const int32_t *keep = p.keep + g * p.keep_pool;
    int32_t *held = c.held + (int64_t)g * c.max_batch;
    const int free = min(max(c.free_count[g], 0), c.n_blocks);
    uint32_t flags = free != c.free_count[g] ? METASD_STATUS_BAD_STATE : 0u;
    auto look = [&](int b, int &from) {
        const int has = held[b], kept = min(max(has, 0), c.max_blocks), length = __ldg(keep + b);
        if (kept != has) flags |= METASD_STATUS_BAD_STATE;
        if (length < 0) flags |= METASD_STATUS_BAD_LENGTH;
        from = length <= 0 ? 0 : divide(length - 1, c.page_size, p.page_inverse) + 1;
        return length < 0 ? 0 : max(kept - from, 0);
    };
    const int rows = (batch + 31) / 32, row0 = (int)((long long)rows * warp / RELEASE_WARPS), row1 = (int)((long long)rows * (warp + 1) / RELEASE_WARPS);
    long long drop = 0;
    int from;
    for (int row = row0; row < row1; ++row) {
        const int b = row * 32 + lane;
        if (b < batch) drop += look(b, from);
    }
    drop = warp_total(drop);
    if (lane == 0) sh_drop[warp] = drop;
    if (tid == 0) sh_total = 0;
    __syncthreads();
    {
        const long long d = sh_drop[lane], before = warp_sum_up_to(d) - d;
        drop = __shfl_sync(FULL, before, warp);
    }
    const long long drop0 = drop;
    // the sequences whose blocks fit behind the free ones: all, unless the tables hold what was not taken from here
    for (int row = row0; row < row1; ++row) {
        const int b = row * 32 + lane, n = b < batch ? look(b, from) : 0;
        const long long upto = warp_sum_up_to((long long)n);
        if (n && free + drop + upto <= c.n_blocks) atomicMax(&sh_total, (int)(drop + upto));
        drop += __shfl_sync(FULL, upto, 31);
    }
    __syncthreads();
    drop = drop0;
    for (int row = row0; row < row1; ++row) {
        const int b = row * 32 + lane, n = b < batch ? look(b, from) : 0;
        const long long upto = warp_sum_up_to((long long)n);
        if (b < batch) {
            ReleaseEntry e = {0, 0, 0, 0};
            if (n) {
                if (drop + upto <= sh_total) {
                    e = ReleaseEntry{from, n, free + sh_total - 1 - (int)(drop + upto - n), 0};
                    held[b] = from;
                } else {
                    flags |= METASD_STATUS_BAD_STATE;
                }
            }
            entries[b] = e;
        }
        drop += __shfl_sync(FULL, upto, 31);
    }
    flags = __reduce_or_sync(FULL, flags);
    if (flags && lane == 0 && c.status) atomicOr(c.status, flags);
    if (tid == 0) c.free_count[g] = free + sh_total;
}

// A warp per sequence and pool.
__global__ void __launch_bounds__(FILL_THREADS) give_back_kernel(const CacheReleaseParams p)
{
    launch_dependents();
    grid_dependency_wait();
    const metasd_cache &c = p.c;
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * (FILL_THREADS / 32) + (threadIdx.x >> 5);
    const int g = (int)(unit / p.batch), b = (int)(unit - (int64_t)g * p.batch);
    if (g >= c.n_pools) return;
    const ReleaseEntry e = ((const ReleaseEntry *)c.workspace)[(int64_t)g * c.max_batch + b];
    const int32_t *table = c.block_table + ((int64_t)g * c.max_batch + b) * c.max_blocks + e.from;
    int32_t *free = c.free_blocks + (int64_t)g * c.n_blocks + e.to;
    for (int i = lane; i < e.drop; i += 32) free[-i] = table[i];
}

}  // namespace

size_t cache_workspace_bytes(int max_batch, int n_pools)
{
    return std::max((size_t)max_batch * sizeof(PlanEntry), (size_t)max_batch * n_pools * sizeof(ReleaseEntry));
}

constexpr int ALONE_TOKENS = 4096;

cudaError_t launch_cache_plan(const CachePlanParams &p, int n_sm, cudaStream_t stream)
{
    if (p.max_tokens <= ALONE_TOKENS) return launch_kernel(plan_kernel<true>, 1, PLAN_THREADS, 0, 1, true, stream, p);
    cudaError_t e = launch_kernel(plan_kernel<false>, 1, PLAN_THREADS, 0, 1, true, stream, p);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)std::min<long long>(((long long)p.max_tokens + SPAN - 1) / SPAN, 8ll * n_sm);
    return launch_kernel(fill_kernel, grid, FILL_THREADS, 0, 1, true, stream, p);
}

cudaError_t launch_cache_release(const CacheReleaseParams &p, cudaStream_t stream)
{
    cudaError_t e = launch_kernel(release_kernel, (unsigned)p.c.n_pools, RELEASE_THREADS, 0, 1, true, stream, p);
    if (e != cudaSuccess) return e;
    const long long units = (long long)p.batch * p.c.n_pools, per = FILL_THREADS / 32;
    return launch_kernel(give_back_kernel, (unsigned)((units + per - 1) / per), FILL_THREADS, 0, 1, true, stream, p);
}

}  // namespace metasd
