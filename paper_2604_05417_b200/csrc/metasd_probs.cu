// metasd_verify_probs: verification of drafted tokens from probabilities and given random numbers.
//
//   accept x_j            iff  u_j q_j(x_j) < p_j(x_j)                       (u < min(1, p/q) without the division)
//   n = first rejection   (k_b if there is none)
//   next token            first v with  sum_{i<=v} w_i > u S,  w = max(0, p_n - q_n),  S = sum_i w_i   (all accepted: w = p_n)
//   d_TV(p_j, q_j)        1/2 sum_v |p_j(v) - q_j(v)|                        (only where it is asked for)
//
// Whole numbers come out of sums over a row, so the sums are made as if in real numbers: with d = fl(p - q) the rounding error
// (p - d) - q of a difference that is above zero is a float, exactly (p >= q >= 0), and so is the rounding error of an addition
// (Knuth's two-sum, six operations on a packed pair).  The errors, 2^-24 of what they belong to, are added up apart; what is lost
// is theirs.  Of n additions that come to S the errors' sum is at most (i + 1) 2^-24 S after the i-th, which rounds it twice: all in all
// less than (n^2 + 3n) 2^-48 S.  No chain is longer than n = 32, which bounds the loss by 2^-37 of the sum, and next to no draw is that near
// to an edge.  Chains and lanes join in fp64.
//
// Bound by memory: without distances one row pair per sequence is read (the one that the token is drawn from), with them every
// pair.  512 sequences of 152064 fp32 entries without: 94 us, 6.5 TB/s; 256 x 7 pairs of 128256 bf16 entries with: 149 us, 6.2 TB/s
// (a copy makes 6.5).  Small calls are a chain: the accept tests' two dependent loads 1.0 us, a part 1.1, the blocks' meeting 0.6, the
// parts' sums and the draw 1.5; one sequence of 32000 entries 5.1 us.
// A row is cut into parts by its length alone, a warp sums a part, and the parts' sums are put together in one order:
// results do not depend on the launch's shape, and the draw re-reads one part (of 80 to 160 of a long row) and not the row.
#include <algorithm>
#include <cfloat>

#include "metasd_staged.cuh"

namespace metasd {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int MAX_PARTS = 160;      // of a row; 5 per lane of the warp that looks for the crossing.  With 256 (8 a lane) that takes longer: 128256 fp32
                                    // lookups 13.1 us instead of 12.2, 512 rows of 152064 the same; with 128, 4 x 8 pairs of 152064 bf16 12.5 instead of 11.7
constexpr int BATCH = 4;            // vectors of a row that a lane has in flight
constexpr int CHAIN = 32;           // additions of a lane to one sum, at most (V up to 327680).  Longer parts add every batch's sums up in fp64, which costs
                                    // registers: in all rows 256 x 7 pairs of 128256 bf16 took 150.1 us instead of 148.7, 256 draws of 32001 9.9 instead
                                    // of 9.6, 64 lookups in 128256 fp32 12.15 instead of 11.75
constexpr unsigned FULL = 0xFFFFFFFFu;

// A pair of rows as 16-byte vectors: vector g of the row holds entries g VEC .. g VEC + VEC - 1.
template <typename LT> struct PairOfRows {
    const uint4 *a, *d;     // from the 16-byte boundary at or in front of the row's start
    int lead_a, lead_d;     // entries between that boundary and the row
    int V, n_vec;
    int certain;            // no draft row: the token that q = 1 for, or -1
};

template <typename LT> __device__ __forceinline__ const uint4 *vectors_of(const LT *row, int &lead)
{
    lead = row_lead(row);
    return reinterpret_cast<const uint4 *>(row - lead);
}

// Entries from tok0 + n on are not the row's.
template <typename LT> __device__ __forceinline__ uint4 cut(uint4 v, int n)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(LT) == 2) {
            if (2 * i >= n) w[i] = 0u;
            else if (2 * i + 1 >= n) w[i] &= 0xFFFFu;
        } else {
            if (i >= n) w[i] = 0u;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Vector g of a row that starts `lead` entries behind a 16-byte boundary.  No 16 bytes are read that hold nothing of the row.
template <typename LT, bool SHIFTED> __device__ __forceinline__ uint4 vector_at(const uint4 *row, int lead, int g, int V)
{
    constexpr int VEC = Logit<LT>::VEC;
    const int n = V - g * VEC;      // entries from here to the row's end
    uint4 v;
    if (!SHIFTED) {
        v = ld_stream(row + g);
    } else {
        v = __ldg(row + g);
        if (lead) {
            uint4 next = make_uint4(0u, 0u, 0u, 0u);
            if (lead + min(n, VEC) > VEC) next = __ldg(row + g + 1);
            v = Logit<LT>::shifted(v, next, lead);
        }
    }
    return n < VEC ? cut<LT>(v, n) : v;
}

__device__ __forceinline__ bool is_probability(float x) { return x >= 0.f && x < INFINITY; }   // -0 is one

// Sums of a lane.  NaN and infinite entries make those they come into NaN; what has its sign set is looked for apart.
struct Sums {
    uint64_t over;          // of max(0, p - q), the differences as rounded, rounded again at every addition; a packed pair
    uint64_t rest;          // what these roundings left out
    float apart, apart1;    // of |p - q|
    bool bad;               // an entry below zero
    __device__ __forceinline__ Sums() : over(0ull), rest(0ull), apart(0.f), apart1(0.f), bad(false) {}
};

__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) { return fma2(b, pack2(-1.f), a); }
// The larger of both, half by half; NaN where either is.
__device__ __forceinline__ uint64_t max2(uint64_t a, uint64_t b)
{
    float al, ah, bl, bh;
    unpack2(a, al, ah);
    unpack2(b, bl, bh);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(al) : "f"(bl));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(ah) : "f"(bh));
    return pack2(al, ah);
}
// sum += x, and what the rounding takes away goes to rest (x and the sum in any order of size).
__device__ __forceinline__ void add_exactly(uint64_t &sum, uint64_t &rest, uint64_t x)
{
    const uint64_t s = add2(sum, x), part = sub2(s, sum);
    rest = add2(rest, add2(sub2(sum, sub2(s, part)), sub2(x, part)));
    sum = s;
}
template <typename LT> __device__ __forceinline__ uint64_t pair_at(const uint4 &v, int i)   // entries 2 i, 2 i + 1
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(LT) == 2) return pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    else return pack2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
}

// A pair of entries of both rows.  With m = max(p, q), m - q is max(0, p - q) with no comparison of its own.  WEIGHT: the row may be drawn
// from; TV: its distance is wanted.  Neither changes the other.
template <bool WEIGHT, bool TV> __device__ __forceinline__ void add_pair(Sums &s, uint64_t p, uint64_t q)
{
    if (WEIGHT) {
        const uint64_t m = max2(p, q), d = sub2(m, q);
        s.rest = add2(s.rest, sub2(sub2(m, d), q));
        add_exactly(s.over, s.rest, d);
    }
    if (TV) {
        float lo, hi;
        unpack2(sub2(p, q), lo, hi);
        s.apart += fabsf(lo);
        s.apart1 += fabsf(hi);
    }
}

template <typename LT, bool PAIR, bool WEIGHT, bool TV>
__device__ __forceinline__ void add_vectors(Sums &s, const uint4 &ra, const uint4 &rd, int tok0, int certain)
{
    constexpr int VEC = Logit<LT>::VEC;
    uint32_t signs = ra.x | ra.y | ra.z | ra.w;
    if (PAIR) signs |= rd.x | rd.y | rd.z | rd.w;
    if (signs & (sizeof(LT) == 2 ? 0x80008000u : 0x80000000u)) {
        float p[VEC], q[VEC];
        Logit<LT>::unpack(ra, p);
        Logit<LT>::unpack(rd, q);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (p[e] < 0.f || (PAIR && q[e] < 0.f)) s.bad = true;
    }
    if (PAIR) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) add_pair<WEIGHT, TV>(s, pair_at<LT>(ra, i), pair_at<LT>(rd, i));
    } else if (certain < tok0 || certain >= tok0 + VEC) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const uint64_t p = pair_at<LT>(ra, i);
            if (WEIGHT) add_exactly(s.over, s.rest, p);
            if (TV) {
                float lo, hi;
                unpack2(p, lo, hi);
                s.apart += lo;
                s.apart1 += hi;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i)
            add_pair<WEIGHT, TV>(s, pair_at<LT>(ra, i), pack2(certain == tok0 + 2 * i ? 1.f : 0.f, certain == tok0 + 2 * i + 1 ? 1.f : 0.f));
    }
}

// The lane's sum of max(0, p - q) in fp64.
__device__ __forceinline__ double weight_of(const Sums &s)
{
    float lo, hi;
    unpack2(s.over, lo, hi);
    const float sum = lo + hi, part = sum - lo;
    return (double)sum + (double)(((lo - (sum - part)) + (hi - part)) + sum2(s.rest));
}

// A warp's BATCH vectors of 32 lanes, read from 16-byte boundaries LEAD entries in front of the row's, become the row's: what a
// lane lacks, the next one has (the last lane: the first, of the next vector; `behind` follows the last vector).
template <typename LT, int LEAD> __device__ __forceinline__ void realign(uint4 (&v)[BATCH], const uint4 &behind)
{
    constexpr bool HALF = sizeof(LT) == 2 && LEAD % 2 != 0;
    constexpr int WORDS = sizeof(LT) == 2 ? LEAD / 2 : LEAD, MORE = WORDS + HALF;   // whole words to skip; words of the next lane
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
        const uint4 n = i + 1 < BATCH ? v[i + 1 < BATCH ? i + 1 : 0] : behind;
        uint32_t w[8] = {v[i].x, v[i].y, v[i].z, v[i].w, n.x, n.y, n.z, n.w};
#pragma unroll
        for (int j = 0; j < MORE; ++j) w[4 + j] = __shfl_sync(FULL, lane == 0 ? w[4 + j] : w[j], (lane + 1) & 31);
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = HALF ? __byte_perm(w[j + WORDS], w[(j + WORDS + 1) & 7], 0x5432) : w[j + WORDS];
        v[i] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}
template <typename LT> __device__ __forceinline__ void realign(uint4 (&v)[BATCH], const uint4 &behind, int lead)
{
    switch (lead) {
    case 1: realign<LT, 1>(v, behind); break;
    case 2: realign<LT, 2>(v, behind); break;
    case 3: realign<LT, 3>(v, behind); break;
    default:
        if constexpr (sizeof(LT) == 2) {
            switch (lead) {
            case 4: realign<LT, 4>(v, behind); break;
            case 5: realign<LT, 5>(v, behind); break;
            case 6: realign<LT, 6>(v, behind); break;
            case 7: realign<LT, 7>(v, behind); break;
            }
        }
    }
}

// 32 BATCH vectors of a row from vector c on, all of them whole.
template <typename LT, bool SHIFTED> __device__ __forceinline__ void load_batch(uint4 (&v)[BATCH], const uint4 *row, int lead, int c)
{
    const uint4 *at = row + c + (threadIdx.x & 31);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) v[i] = ld_stream(at + 32 * i);
}
template <typename LT, bool SHIFTED> __device__ __forceinline__ uint4 load_behind(const uint4 *row, int lead, int c)
{
    return SHIFTED && lead ? ld_stream(row + c + 32 * BATCH) : make_uint4(0u, 0u, 0u, 0u);
}

template <typename LT, bool PAIR, bool WEIGHT, bool TV>
__device__ __forceinline__ void add_batch(Sums &s, const uint4 (&ra)[BATCH], const uint4 (&rd)[BATCH], int c, int certain)
{
    constexpr int VEC = Logit<LT>::VEC;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) add_vectors<LT, PAIR, WEIGHT, TV>(s, ra[i], rd[i], (c + 32 * i + (int)(threadIdx.x & 31)) * VEC, certain);
}

// A warp's sums of a part, put where the sequence's sums are collected.
template <bool WEIGHT, bool TV>
__device__ __forceinline__ void publish(bool lane_bad, double lane_weight, double lane_apart, int s, uint32_t weights_at, uint32_t apart_at)
{
    const double w = WEIGHT ? warp_sum(lane_weight) : 0.0;
    const float apart = TV ? warp_sum_f((float)lane_apart) : 0.f;
    const bool bad = __any_sync(FULL, lane_bad);
    if ((threadIdx.x & 31) == 0) {
        st_cluster(weights_at + 8u * s, bad ? (double)NAN : w);
        if (TV) st_cluster(apart_at + 4u * s, __float_as_int(bad ? NAN : apart));
    }
}

// Asks L2 for a batch: 2 KB of each row, a line per lane.
template <typename LT> __device__ __forceinline__ void prefetch_batch(const PairOfRows<LT> &r, bool pair, int c)
{
    const int lane = threadIdx.x & 31, g = c + 8 * (lane & 15);
    const uint4 *row = lane < 16 ? r.a : r.d;
    if ((lane < 16 || pair) && g < r.n_vec) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + g));
}

// The parts s0, s0 + step, .. below s1 of a row (pair), by one warp.  The order of additions does not depend on where the rows
// start, and the sums that a draw needs (WEIGHT) do not change those of the distance.  LONG: parts of chains above CHAIN.
template <typename LT, bool PAIR, bool WEIGHT, bool TV, bool LONG, bool SHIFTED>
__device__ __forceinline__ void sum_parts(const PairOfRows<LT> r, int part_vecs, int s0, int s1, int step, uint32_t weights_at, uint32_t apart_at)
{
    constexpr int VEC = Logit<LT>::VEC;
    const int whole = r.V / VEC;
    for (int s = s0; s < s1; s += step) {
        const int g0 = s * part_vecs, g1 = min(g0 + part_vecs, r.n_vec);
        Sums x;
        double weight = 0.0, apart = 0.0;
        auto fold = [&] {       // no chain of fp32 additions is longer than a batch
            if (TV) {
                apart += (double)(x.apart + x.apart1);
                x.apart = x.apart1 = 0.f;
            }
        };
        auto fold_weight = [&] {
            if (WEIGHT && LONG) {
                weight += weight_of(x);
                x.over = x.rest = 0ull;
            }
        };
        int c = g0;
        // whole vectors, whole batches: nothing but loads and sums
        for (; c + 32 * BATCH <= min(g1, whole); c += 32 * BATCH) {
            uint4 ra[BATCH], rd[BATCH];
            load_batch<LT, SHIFTED>(ra, r.a, r.lead_a, c);
            const uint4 behind_a = load_behind<LT, SHIFTED>(r.a, r.lead_a, c);
            if (PAIR) {
                load_batch<LT, SHIFTED>(rd, r.d, r.lead_d, c);
                const uint4 behind_d = load_behind<LT, SHIFTED>(r.d, r.lead_d, c);
                if (SHIFTED) realign<LT>(rd, behind_d, r.lead_d);
            }
            if (SHIFTED) realign<LT>(ra, behind_a, r.lead_a);
            add_batch<LT, PAIR, WEIGHT, TV>(x, ra, PAIR ? rd : ra, c, r.certain);
            fold();
            fold_weight();
        }
        // the row's end
#pragma unroll 1
        for (int g = c + (threadIdx.x & 31); g < g1; g += 32) {
            const uint4 ra = vector_at<LT, SHIFTED>(r.a, r.lead_a, g, r.V);
            const uint4 rd = PAIR ? vector_at<LT, SHIFTED>(r.d, r.lead_d, g, r.V) : ra;
            add_vectors<LT, PAIR, WEIGHT, TV>(x, ra, rd, g * VEC, r.certain);
        }
        fold();
        publish<WEIGHT, TV>(x.bad, WEIGHT ? weight + weight_of(x) : 0.0, apart, s, weights_at, apart_at);
    }
}

template <typename LT, bool WEIGHT, bool TV, bool LONG>
__device__ __forceinline__ void sum_parts(const PairOfRows<LT> &r, bool pair, int part_vecs, int s0, int s1, int step, uint32_t weights_at, uint32_t apart_at)
{
    if (pair) {
        if ((r.lead_a | r.lead_d) == 0) sum_parts<LT, true, WEIGHT, TV, LONG, false>(r, part_vecs, s0, s1, step, weights_at, apart_at);
        else sum_parts<LT, true, WEIGHT, TV, LONG, true>(r, part_vecs, s0, s1, step, weights_at, apart_at);
    } else {
        if (r.lead_a == 0) sum_parts<LT, false, WEIGHT, TV, LONG, false>(r, part_vecs, s0, s1, step, weights_at, apart_at);
        else sum_parts<LT, false, WEIGHT, TV, LONG, true>(r, part_vecs, s0, s1, step, weights_at, apart_at);
    }
}

// Inclusive sums over the lanes.
__device__ __forceinline__ double lanes_up_to(double x)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double t = __shfl_up_sync(FULL, x, o);
        if (lane >= o) x += t;
    }
    return x;
}
// The lane in whose x, laid end to end (upto: their inclusive sums), the threshold lies: the first that ends beyond it; rounding
// may leave none, then the last with weight; -1: no weight.
__device__ __forceinline__ int crossing_lane(double x, double upto, double threshold, bool &beyond)
{
    const unsigned mass = __ballot_sync(FULL, x > 0.0), hits = __ballot_sync(FULL, upto > threshold) & mass;
    beyond = hits != 0;
    return hits ? __ffs(hits) - 1 : 31 - __clz(mass);
}

// What the block looks for in a part of a row: the token at which the sums from `base` on pass the threshold.
struct Crossing {
    double base, threshold;
    int g0, g1;         // the part's vectors
    int found;          // the first token whose sum is beyond the threshold
    int last;           // the last token with weight so far, for sums that rounding leaves below the threshold
    bool again;         // nothing is left over of the target's row: it is drawn from as it stands
};

// By all threads, a vector each and a stretch of THREADS vectors at a time; thread 0 has the token.  Every warp offers its first candidate and the
// smallest is taken: sums of different lanes are rounded differently and need not rise from lane to lane by the last bit.
template <typename LT>
__device__ __forceinline__ int find_token(const PairOfRows<LT> &r, bool pair, Crossing &sh, double (&sh_warp)[WARPS])
{
    constexpr int VEC = Logit<LT>::VEC;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    double base = sh.base;
    const double threshold = sh.threshold;
    for (int c = sh.g0; c < sh.g1; c += THREADS) {
        const int g = c + tid;
        uint4 ra = make_uint4(0u, 0u, 0u, 0u), rd = ra;
        if (g < sh.g1) {
            ra = vector_at<LT, true>(r.a, r.lead_a, g, r.V);
            if (pair) rd = vector_at<LT, true>(r.d, r.lead_d, g, r.V);
        }
        float p[VEC], q[VEC];
        Logit<LT>::unpack(ra, p);
        Logit<LT>::unpack(rd, q);
        Sums x;
        int last = -1;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (!pair) q[e] = g * VEC + e == r.certain ? 1.f : 0.f;
            if (p[e] > q[e]) last = g * VEC + e;
        }
#pragma unroll
        for (int e = 0; e < VEC; e += 2) add_pair<true, false>(x, pack2(p[e], p[e + 1]), pack2(q[e], q[e + 1]));
        const double mine = weight_of(x);
        const double upto = lanes_up_to(mine);
        if (lane == 31) sh_warp[warp] = upto;
        last = __reduce_max_sync(FULL, last);
        if (lane == 0 && last >= 0) atomicMax(&sh.last, last);
        __syncthreads();
        double offset = base;
        for (int i = 0; i < warp; ++i) offset += sh_warp[i];
        double end = offset;
        for (int i = warp; i < WARPS; ++i) end += sh_warp[i];
        const unsigned hits = __ballot_sync(FULL, mine > 0.0 && offset + upto > threshold);
        if (hits && lane == __ffs(hits) - 1) {
            double run = offset + (upto - mine);
            int token = -1;
            bool done = false;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const bool some = p[e] > q[e];
                run += some ? (double)p[e] - (double)q[e] : 0.0;
                if (!done && some) {
                    token = g * VEC + e;
                    done = run > threshold;
                }
            }
            atomicMin(&sh.found, token);
        }
        if (__syncthreads_or(hits != 0)) return tid == 0 ? sh.found : -1;
        base = end;
    }
    return tid == 0 ? sh.last : -1;
}

template <typename LT, bool TV, bool LONG>
__global__ void __launch_bounds__(THREADS, 4) probs_kernel(const ProbsParams p)
{
    constexpr int VEC = Logit<LT>::VEC;
    __shared__ double sh_weight[MAX_PARTS];     // the parts' sums; NaN: the part holds what is no probability
    __shared__ float sh_apart[TV ? MAX_PARTS : 1];
    __shared__ int sh_n, sh_token;
    __shared__ Crossing sh_crossing;
    __shared__ double sh_warp[WARPS];

    launch_dependents();
    grid_dependency_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = (int)cluster_size(), rank = (int)cluster_rank();
    const int job = (int)blockIdx.x / C, k = p.k, V = p.V;
    const int b = TV ? job / (k + 1) : job;
    int j = TV ? job - b * (k + 1) : 0;

    uint32_t flags = 0;
    int kb = k;
    if (p.draft_len) {
        kb = __ldg(p.draft_len + b);
        const int as_given = kb;
        kb = min(max(kb, p.min_draft), k);
        if (kb != as_given) flags |= METASD_STATUS_BAD_LENGTH;
    }
    if (TV && j > kb) return;
    const LT *target = reinterpret_cast<const LT *>(p.target) + (int64_t)b * p.target_seq;
    const LT *draft = nullptr;
    bool lost = false;       // the sequence's draft rows are not where the caller says
    if (p.draft && kb > 0) {
        const int place = p.place ? __ldg(p.place + b) : b;
        lost = place < 0 || place >= p.batch;
        if (lost) flags |= METASD_STATUS_BAD_INDEX;
        else draft = reinterpret_cast<const LT *>(p.draft) + (int64_t)place * p.draft_seq;
    }
    if (lost) {     // nothing is accepted, nothing can be drawn
        if (TV && j < kb && rank == 0 && tid == 0) p.d_tv[(int64_t)b * k + j] = 1.f;
        if (j == 0 && rank == 0 && tid == 0) {
            p.accepted_len[b] = 0;
            p.next_token[b] = -1;
            if (p.status) atomicOr(p.status, flags);
        }
        return;
    }

    const int parts = p.parts, part_vecs = p.part_vecs, s0 = parts * rank / C + warp, s1 = parts * (rank + 1) / C;
    const int32_t *tokens = p.tokens + (int64_t)b * k;
    PairOfRows<LT> r;
    bool pair = false;
    auto rows_of = [&](int position) {
        r.a = vectors_of(target + position * p.target_row, r.lead_a);
        pair = draft && position < kb;
        r.d = r.a;
        r.lead_d = 0;
        if (pair) r.d = vectors_of(draft + position * p.draft_row, r.lead_d);
    };
    r.V = V;
    r.n_vec = (V + VEC - 1) / VEC;
    r.certain = -1;
    const float u_draw = rank == 0 && warp == 0 ? __ldg(p.u_draw + b) : 0.f;
    // The accept tests, a lane each, by one warp.
    int x = -1;
    float u = 0.f;
    if (warp == 0 && lane < kb) {
        x = __ldg(tokens + lane);
        u = __ldg(p.u_accept + (int64_t)b * k + lane);
    }
    if (TV && j < kb) {     // this row is read whatever the tests say: its first lines come meanwhile
        rows_of(j);
        if (!draft) r.certain = __ldg(tokens + j);
        if (s0 < s1) prefetch_batch(r, pair, s0 * part_vecs);
    }
    if (warp == 0) {
        bool accepted = false;
        uint32_t f = 0;
        if (lane < kb) {
            if (x < 0 || x >= V) {
                f |= METASD_STATUS_TOKEN_OOR;
            } else {
                const float px = Logit<LT>::scalar(target + lane * p.target_row, x);
                const float qx = draft ? Logit<LT>::scalar(draft + lane * p.draft_row, x) : 1.f;
                if (!is_probability(px) || !is_probability(qx)) {
                    f |= METASD_STATUS_NONFINITE;
                } else {
                    if (qx == 0.f) f |= METASD_STATUS_Q_ZERO;
                    accepted = (double)u * (double)qx < (double)px;     // the product of two floats: exact
                }
            }
        }
        flags |= __reduce_or_sync(FULL, f);
        const int stop = __ffs(__ballot_sync(FULL, !accepted)) - 1;     // lanes from kb on never accept
        if (lane == stop) { sh_n = stop; sh_token = x; }
    }
    __syncthreads();
    const int n = sh_n;
    if (TV && j == kb && n < kb) return;       // no bonus token
    if (!TV || j == kb) {
        j = n;
        rows_of(j);
        if (!TV && !draft && j < kb) r.certain = sh_token;
    }
    cluster_arrive_relaxed();           // every CTA of the cluster runs: its shared memory may be written

    const uint32_t weights_at = map_to_rank(smem_addr(sh_weight), 0), apart_at = map_to_rank(smem_addr(sh_apart), 0);
    cluster_wait();
    if (!TV || n == j) sum_parts<LT, true, TV, LONG>(r, pair, part_vecs, s0, s1, WARPS, weights_at, apart_at);
    else if constexpr (TV) sum_parts<LT, false, true, LONG>(r, pair, part_vecs, s0, s1, WARPS, weights_at, apart_at);
    cluster_sync_all();
    if (rank != 0) return;

    // One warp puts the parts together: lane l holds parts l per .. l per + per - 1.
    constexpr int PER = MAX_PARTS / 32;
    const int per = (parts + 31) / 32;
    for (bool first = true;; first = false) {
        if (warp == 0) {
            double w[PER], mine = 0.0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                w[i] = 0.0;
                if (i < per && lane * per + i < parts) w[i] = sh_weight[lane * per + i];
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) mine += w[i];
            const double upto = lanes_up_to(mine), total = __shfl_sync(FULL, upto, 31);
            const bool bad = !(total <= (double)FLT_MAX);
            Crossing x = {0.0, 0.0, 0, 0, 0x7FFFFFFF, -1, false};      // nothing to look for
            if (n == j) {       // the row that the token is drawn from
                if (total > 0.0 && !bad) {
                    x.threshold = (double)u_draw * total;
                    if (x.threshold < 0.0) x.threshold = 0.0;
                    bool beyond;
                    const int src = crossing_lane(mine, upto, x.threshold, beyond);
                    int part = -1;      // of the lane's: the first that ends beyond the threshold, else the last with weight
                    double run = upto - mine;
                    bool done = false;
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        if (!done && w[i] > 0.0) {
                            part = lane * per + i;
                            x.base = run;
                        }
                        run += w[i];
                        done = done || (w[i] > 0.0 && run > x.threshold);
                    }
                    part = __shfl_sync(FULL, part, src);
                    x.base = fmin(__shfl_sync(FULL, x.base, src), x.threshold);
                    x.g0 = part * part_vecs;
                    x.g1 = min(x.g0 + part_vecs, r.n_vec);
                } else if (!bad && (pair || r.certain >= 0)) {
                    x.again = true;
                } else {
                    flags |= METASD_STATUS_NONFINITE;       // or a row of zeros
                }
            }
            if (lane == 0) sh_crossing = x;
            if (TV && first && j < kb) {
                double apart = 0.0;
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (i < per && lane * per + i < parts) apart += (double)sh_apart[lane * per + i];
                apart = warp_sum(apart);
                // a token outside the vocabulary has no place in the row
                const bool nowhere = !pair && (r.certain < 0 || r.certain >= V);
                const bool finite = apart <= (double)FLT_MAX;
                if (!finite) flags |= METASD_STATUS_NONFINITE;
                if (lane == 0) p.d_tv[(int64_t)b * k + j] = !finite || nowhere ? 1.f : (float)(0.5 * apart);
            }
            if (lane == 0) {
                if (n == j && !x.again) p.accepted_len[b] = n;
                if (flags && !x.again && p.status) atomicOr(p.status, flags);
            }
        }
        __syncthreads();
        if (!sh_crossing.again) break;
        __syncthreads();
        r.certain = -1;
        pair = false;
        sum_parts<LT, true, TV, LONG>(r, false, part_vecs, warp, parts, WARPS, smem_addr(sh_weight), smem_addr(sh_apart));
        __syncthreads();
    }
    if (TV && n != j) return;
    const int token = find_token<LT>(r, pair, sh_crossing, sh_warp);
    if (tid == 0) p.next_token[b] = token;
}

// The reward of a round that metasd_verify did not verify, the bandit update and the next selection: a warp per sequence, fp64.  A chain of loads,
// a logarithm and a square root: 3.2 us behind a round of 64 sequences, 4.1 behind one of 1024.  Rows that are not normalised may lie more than 1
// apart; the policies are made for rewards in [0, 1] (EXP3's weights would all become zeros).
__global__ void __launch_bounds__(32) feedback_kernel(const VerifyParams p, const float *d_tv)
{
    __shared__ BanditShared sh;
    launch_dependents();
    grid_dependency_wait();
    const int b = blockIdx.x, lane = threadIdx.x, k = drafted(p.draft_len, b, p.k);
    const BanditStep step = warp_bandit_fetch(p, b, p.st.t[b], p.st.arm[b], sh);
    const double align = p.reward_kind == METASD_REWARD_BD && lane < k ? 1.0 - fmin((double)d_tv[(int64_t)b * p.k + lane], 1.0) : 0.0;
    const double reward = p.reward_kind == METASD_REWARD_BE ? (double)p.accepted_len[b] / (double)k : warp_sum(align) / (double)k;
    warp_bandit_finish(p, b, step, reward, sh);
    if (lane == 0) p.reward[b] = (float)reward;
}

}  // namespace

cudaError_t launch_probs(const ProbsParams &params, int dtype, int n_sm, cudaStream_t stream)
{
    ProbsParams p = params;
    const int vec = dtype == METASD_BF16 ? 8 : 4;
    const long long n_vec = ((long long)p.V + vec - 1) / vec;
    const long long step = 32 * BATCH;      // vectors that a warp reads at once
    p.part_vecs = (int)(step * std::max(1ll, (n_vec + step * MAX_PARTS - 1) / (step * MAX_PARTS)));
    p.parts = (int)((n_vec + p.part_vecs - 1) / p.part_vecs);
    const long long jobs = (long long)p.batch * (p.d_tv ? p.k + 1 : 1);
    // Blocks that share a row.  `rows`: those that are read (with distances the bonus row of a few sequences only; of ragged drafts about half of
    // the slots, whose other blocks end at once).  More blocks a row shorten a launch's last wave of four blocks an SM, and cost a
    // start, a meeting and a smaller stretch each.  Us with 1, 2, 4 and 8 (fp32 rows without distances unless it says so):
    //   V = 128256, rows 100: 53.7, 32.7, 22.4, 24.1; 300: 65.0, 58.8, 51.5, 53.8; 600: 108.0, 91.9, 91.1, 99.9; 900: 141.1, 125.9, 131.4, 145.4
    //   V = 152064, rows 440: 78.0, 84.5, 77.6; 512: 84.8, 90.3, 89.3; 620: 122.5, 105.6, 104.9
    //   V = 128256, bf16 with distances, rows 40: 28.9, 18.5, 13.1, 11.0; 448: 55.4, 48.0, 46.0, 52.4; 1190: 113.5, 103.0, 107.5, 128.1;
    //     1792: 154.0, 152.9, 168.0
    //   V = 50264 with distances, rows 120: 26.8, 18.3, 14.7, 15.8; 300: 32.7, 31.7, 28.7, 32.7; 640: 57.4, 49.0, 50.3, 65.3
    //   V = 32000, bf16, rows 100: 9.4, 8.9, 8.1, 10.1; 300: 16.2, 13.9, 15.6, 23.6; 600: 21.8, 23.8, 28.7; 1000: 30.7, 35.7, 44.6
    // The rule is a simple one and not the table's best everywhere: V = 128256 with distances, rows 448 (0.76 of a wave) take 1; V = 152064, rows 440
    // (0.74) take 2; V = 50264 with distances, rows 500 (0.84) take 1: 41.4 where 2 take 38.8.  0.55: lengths spread evenly over 0 .. k.
    const double rows = !p.d_tv ? p.batch : p.draft_len ? 0.55 * p.batch * (p.k + 1) : (double)p.batch * p.k;
    const auto waves = [&](int blocks) { return rows * blocks / (4.0 * n_sm); };
    const bool lengthy = n_vec >= 8192;     // 128 KB
    int cluster = 1;
    while (cluster <= 8 && !(waves(cluster) >= 0.75 && waves(cluster) <= 1.0)) cluster *= 2;      // one wave, well filled
    if (cluster > 8)
        cluster = waves(8) <= 1.0 ? 8 : waves(4) <= (lengthy ? n_vec >= 24576 ? 2.75 : 2.1 : 1.0) ? 4 : waves(2) <= (lengthy ? 8.0 : 1.35) ? 2 : 1;
    while (cluster > 1 && p.parts <= WARPS * cluster / 2) cluster /= 2;
    auto launch = [&](auto kernel) { return launch_kernel(kernel, (unsigned)(jobs * cluster), THREADS, 0, cluster, true, stream, p); };
    auto pick = [&](auto plain, auto folding) { return p.part_vecs / 32 * (vec / 2) > CHAIN ? launch(folding) : launch(plain); };
    if (dtype == METASD_BF16)
        return p.d_tv ? pick(probs_kernel<__nv_bfloat16, true, false>, probs_kernel<__nv_bfloat16, true, true>)
                      : pick(probs_kernel<__nv_bfloat16, false, false>, probs_kernel<__nv_bfloat16, false, true>);
    return p.d_tv ? pick(probs_kernel<float, true, false>, probs_kernel<float, true, true>)
                  : pick(probs_kernel<float, false, false>, probs_kernel<float, false, true>);
}

cudaError_t launch_feedback(const VerifyParams &p, const float *d_tv, cudaStream_t stream)
{
    return launch_kernel(feedback_kernel, (unsigned)p.batch, 32, 0, 1, true, stream, p, d_tv);
}

}  // namespace metasd
