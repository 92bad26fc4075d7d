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
// is theirs, below 2^-45 of the sum, and next to no draw is that near to an edge.  The lanes' sums join in fp64.
//
// Bound by memory: without distances one row pair per sequence is read (the one that the token is drawn from), with them every
// pair.  A row is cut into parts by its length alone, a warp sums a part, and the parts' sums are put together in one order:
// results do not depend on the launch's shape, and the draw re-reads one part (at most 1/64 of a long row) and not the row.
#include <algorithm>

#include "metasd_staged.cuh"

namespace metasd {

namespace {

constexpr int PROBS_THREADS = 256, PROBS_WARPS = PROBS_THREADS / 32;
constexpr int MAX_PARTS = 256;      // of a row; 8 per lane of the warp that looks for the crossing
constexpr int BATCH = 4;            // vectors of a row that a lane has in flight
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
template <typename LT, bool SHIFTED, bool AGAIN> __device__ __forceinline__ uint4 vector_at(const uint4 *row, int lead, int g, int V)
{
    constexpr int VEC = Logit<LT>::VEC;
    const int n = V - g * VEC;      // entries from here to the row's end
    uint4 v;
    if (!SHIFTED) {
        v = AGAIN ? __ldcg(row + g) : ld_stream(row + g);
    } else {
        v = AGAIN ? __ldcg(row + g) : __ldg(row + g);
        if (lead) {
            uint4 next = make_uint4(0u, 0u, 0u, 0u);
            if (lead + min(n, VEC) > VEC) next = AGAIN ? __ldcg(row + g + 1) : __ldg(row + g + 1);
            v = Logit<LT>::shifted(v, next, lead);
        }
    }
    return n < VEC ? cut<LT>(v, n) : v;
}

// Whether any entry of the vectors may be no probability (NaN, infinite, or with its sign set): the largest bit pattern.
template <typename LT> __device__ __forceinline__ bool suspicious(const uint4 &v)
{
    if constexpr (sizeof(LT) == 2) {
        const uint32_t m = __vmaxu2(__vmaxu2(v.x, v.y), __vmaxu2(v.z, v.w));
        return m >= 0x7F800000u || (m & 0xFFFFu) >= 0x7F80u;
    } else {
        return max(max(v.x, v.y), max(v.z, v.w)) >= 0x7F800000u;
    }
}
__device__ __forceinline__ bool is_probability(float x) { return x >= 0.f && x < INFINITY; }   // -0 is one

// Sums of a lane, as packed pairs.
struct Sums {
    uint64_t over;      // of max(0, p - q), the differences as rounded, rounded again at every addition
    uint64_t rest;      // what these roundings left out
    uint64_t under;     // of max(0, q - p)
    bool bad;
};

__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) { return fma2(b, pack2(-1.f), a); }
__device__ __forceinline__ uint64_t max2(uint64_t a, uint64_t b)
{
    float al, ah, bl, bh;
    unpack2(a, al, ah);
    unpack2(b, bl, bh);
    return pack2(fmaxf(al, bl), fmaxf(ah, bh));
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

// A pair of entries of both rows.  With m = max(p, q), m - q is max(0, p - q) with no comparison of its own.
template <bool TV> __device__ __forceinline__ void add_pair(Sums &s, uint64_t p, uint64_t q)
{
    const uint64_t m = max2(p, q), d = sub2(m, q);
    s.rest = add2(s.rest, sub2(sub2(m, d), q));
    add_exactly(s.over, s.rest, d);
    if (TV) s.under = add2(s.under, sub2(m, p));
}

template <typename LT, bool PAIR, bool TV>
__device__ __forceinline__ void add_vectors(Sums &s, const uint4 &ra, const uint4 &rd, int tok0, int certain)
{
    constexpr int VEC = Logit<LT>::VEC;
    if (suspicious<LT>(ra) || (PAIR && suspicious<LT>(rd))) {
        float p[VEC], q[VEC];
        Logit<LT>::unpack(ra, p);
        Logit<LT>::unpack(rd, q);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (!is_probability(p[e]) || (PAIR && !is_probability(q[e]))) s.bad = true;
    }
    if (PAIR) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) add_pair<TV>(s, pair_at<LT>(ra, i), pair_at<LT>(rd, i));
    } else if (certain < tok0 || certain >= tok0 + VEC) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) add_exactly(s.over, s.rest, pair_at<LT>(ra, i));
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i)
            add_pair<TV>(s, pair_at<LT>(ra, i), pack2(certain == tok0 + 2 * i ? 1.f : 0.f, certain == tok0 + 2 * i + 1 ? 1.f : 0.f));
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

// The sums of the vectors g0 .. g1 - 1 (a multiple of 32 from g0), a lane every 32nd.  The order of additions does not depend on where the rows
// start: off 16-byte boundaries a vector is two loads (the second one's line is in L1), so that half as many are in flight.
template <typename LT, bool PAIR, bool TV, bool SHIFTED>
__device__ __forceinline__ Sums sum_part(const PairOfRows<LT> &r, int g0, int g1)
{
    constexpr int VEC = Logit<LT>::VEC, N = SHIFTED ? BATCH / 2 : BATCH;
    Sums s = {0ull, 0ull, 0ull, false};
    int g = g0 + (threadIdx.x & 31);
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    // whole vectors, whole batches: nothing but loads and sums
    for (int c = g0; c + 32 * N <= min(g1, r.V / VEC); c += 32 * N, g += 32 * N) {
        uint4 ra[N], rd[N];
        if (!SHIFTED) {
#pragma unroll
            for (int i = 0; i < N; ++i) ra[i] = ld_stream(r.a + g + 32 * i);
            if (PAIR) {
#pragma unroll
                for (int i = 0; i < N; ++i) rd[i] = ld_stream(r.d + g + 32 * i);
            }
        } else {
            uint4 na[N], nd[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ra[i] = __ldg(r.a + g + 32 * i);
                na[i] = r.lead_a ? __ldg(r.a + g + 32 * i + 1) : zero;
            }
            if (PAIR) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    rd[i] = __ldg(r.d + g + 32 * i);
                    nd[i] = r.lead_d ? __ldg(r.d + g + 32 * i + 1) : zero;
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ra[i] = Logit<LT>::shifted(ra[i], na[i], r.lead_a);
                if (PAIR) rd[i] = Logit<LT>::shifted(rd[i], nd[i], r.lead_d);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) add_vectors<LT, PAIR, TV>(s, ra[i], PAIR ? rd[i] : zero, (g + 32 * i) * VEC, r.certain);
    }
    // the row's end
#pragma unroll 1
    for (; g < g1; g += 32) {
        const uint4 ra = vector_at<LT, SHIFTED, false>(r.a, r.lead_a, g, r.V);
        const uint4 rd = PAIR ? vector_at<LT, SHIFTED, false>(r.d, r.lead_d, g, r.V) : zero;
        add_vectors<LT, PAIR, TV>(s, ra, rd, g * VEC, r.certain);
    }
    return s;
}

template <typename LT, bool TV>
__device__ __forceinline__ Sums sum_part(const PairOfRows<LT> &r, bool pair, int g0, int g1)
{
    if (pair) return (r.lead_a | r.lead_d) == 0 ? sum_part<LT, true, TV, false>(r, g0, g1) : sum_part<LT, true, TV, true>(r, g0, g1);
    return r.lead_a == 0 ? sum_part<LT, false, TV, false>(r, g0, g1) : sum_part<LT, false, TV, true>(r, g0, g1);
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

// The token at which the sums from `base` on pass the threshold, in the vectors g0 .. g1 - 1, by one warp: the first, else
// (rounding) the last one with weight.  A lane sums BATCH consecutive vectors, so that lane order is token order; then the lanes
// take the entries of the lane that holds the crossing, one each.
template <typename LT>
__device__ __forceinline__ int find_token(const PairOfRows<LT> &r, bool pair, int g0, int g1, double base, double threshold)
{
    constexpr int VEC = Logit<LT>::VEC;
    static_assert(BATCH * VEC <= 32, "an entry per lane");
    const int lane = threadIdx.x & 31;
    const LT *a = reinterpret_cast<const LT *>(r.a) + r.lead_a, *d = reinterpret_cast<const LT *>(r.d) + r.lead_d;
    auto weight = [&](float p, float q, int v) {
        if (!pair) q = v == r.certain ? 1.f : 0.f;
        return p > q ? (double)p - (double)q : 0.0;
    };
    int last = -1;
    for (int c = g0; c < g1; c += 32 * BATCH) {
        double mine = 0.0;
        const int g = c + lane * BATCH;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            uint4 ra = make_uint4(0u, 0u, 0u, 0u), rd = ra;
            if (g + i < g1) {
                ra = vector_at<LT, true, true>(r.a, r.lead_a, g + i, r.V);
                if (pair) rd = vector_at<LT, true, true>(r.d, r.lead_d, g + i, r.V);
            }
            float p[VEC], q[VEC];
            Logit<LT>::unpack(ra, p);
            Logit<LT>::unpack(rd, q);
#pragma unroll
            for (int e = 0; e < VEC; ++e) mine += weight(p[e], q[e], (g + i) * VEC + e);
        }
        const double upto = lanes_up_to(mine);
        bool beyond;
        const int src = crossing_lane(mine, base + upto, threshold, beyond);
        if (src >= 0) {
            const int v = (c + src * BATCH) * VEC + lane;
            double w = 0.0;
            if (lane < BATCH * VEC && v < min(r.V, g1 * VEC)) w = weight(Logit<LT>::scalar_l2(a, v), pair ? Logit<LT>::scalar_l2(d, v) : 0.f, v);
            bool any;
            last = (c + src * BATCH) * VEC + crossing_lane(w, base + __shfl_sync(FULL, upto - mine, src) + lanes_up_to(w), threshold, any);
            if (beyond) return last;
        }
        base += __shfl_sync(FULL, upto, 31);
    }
    return last;
}

template <typename LT, bool TV>
__global__ void __launch_bounds__(PROBS_THREADS, 4) probs_kernel(const ProbsParams p)
{
    constexpr int VEC = Logit<LT>::VEC;
    __shared__ double sh_weight[MAX_PARTS];     // the parts' sums; NaN: the part holds what is no probability
    __shared__ float sh_under[TV ? MAX_PARTS : 1];
    __shared__ int sh_n;
    __shared__ bool sh_again;

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

    // The accept tests, a lane each, by one warp.
    const int32_t *tokens = p.tokens + (int64_t)b * k;
    auto first_rejection = [&]() {
        bool accepted = false;
        uint32_t f = 0;
        if (lane < kb) {
            const int x = __ldg(tokens + lane);
            const float u = __ldg(p.u_accept + (int64_t)b * k + lane);
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
        return __ffs(__ballot_sync(FULL, !accepted)) - 1;   // lanes from kb on never accept
    };
    int n = -1;
    if (!TV || j == kb) {
        if (warp == 0) {
            n = first_rejection();
            if (lane == 0) sh_n = n;
        }
        __syncthreads();
        n = sh_n;
        if (TV && n < kb) return;       // no bonus token
        j = n;
    } else if (rank == 0 && warp == 0) {
        n = first_rejection();
    }
    cluster_arrive_relaxed();           // every CTA of the cluster runs: its shared memory may be written

    PairOfRows<LT> r;
    r.V = V;
    r.n_vec = (V + VEC - 1) / VEC;
    r.a = vectors_of(target + j * p.target_row, r.lead_a);
    bool pair = draft && j < kb;
    r.d = r.a;
    r.lead_d = 0;
    r.certain = -1;
    if (pair) r.d = vectors_of(draft + j * p.draft_row, r.lead_d);
    else if (j < kb) r.certain = __ldg(tokens + j);

    const int parts = p.parts, part_vecs = p.part_vecs;
    const uint32_t weights_at = map_to_rank(smem_addr(sh_weight), 0), under_at = map_to_rank(smem_addr(sh_under), 0);
    bool published = false;
    for (int s = parts * rank / C + warp; s < parts * (rank + 1) / C; s += PROBS_WARPS) {
        const Sums x = sum_part<LT, TV>(r, pair, s * part_vecs, min((s + 1) * part_vecs, r.n_vec));
        const double w = warp_sum(weight_of(x));
        const float under = TV ? warp_sum_f(sum2(x.under)) : 0.f;
        const bool bad = __any_sync(FULL, x.bad);
        if (!published) { cluster_wait(); published = true; }
        if (lane == 0) {
            st_cluster(weights_at + 8u * s, bad ? (double)NAN : w);
            if (TV) st_cluster(under_at + 4u * s, __float_as_int(under));
        }
    }
    if (!published) cluster_wait();
    cluster_sync_all();
    if (rank != 0) return;

    // One warp puts the parts together: lane l holds parts l per .. l per + per - 1.
    const int per = (parts + 31) / 32;
    const bool draws = n == j;      // warp 0 knows n
    for (bool first = true;; first = false) {
        bool again = false;
        if (warp == 0) {
            double mine = 0.0;
            for (int i = 0; i < per; ++i)
                if (lane * per + i < parts) mine += sh_weight[lane * per + i];
            const double upto = lanes_up_to(mine);
            const double total = __shfl_sync(FULL, upto, 31);
            const bool bad = !(total < INFINITY);
            if (TV && first && j < kb) {
                double under = 0.0;
                for (int i = 0; i < per; ++i)
                    if (lane * per + i < parts) under += (double)sh_under[lane * per + i];
                under = warp_sum(under);
                // a token outside the vocabulary has no place in the row
                const bool nowhere = !pair && (r.certain < 0 || r.certain >= V);
                if (lane == 0) p.d_tv[(int64_t)b * k + j] = bad || nowhere ? 1.f : (float)(0.5 * (total + under));
                if (bad) flags |= METASD_STATUS_NONFINITE;
            }
            if (draws) {
                int token = -1;
                if (bad) {
                    flags |= METASD_STATUS_NONFINITE;
                } else if (total > 0.0) {
                    const double threshold = (double)__ldg(p.u_draw + b) * total;
                    bool beyond;
                    const int src = crossing_lane(mine, upto, threshold, beyond);
                    int part = -1;
                    double base = 0.0;
                    if (lane == src) {
                        double run = upto - mine;
                        bool done = false;
                        for (int i = 0; i < per; ++i) {
                            const double w = lane * per + i < parts ? sh_weight[lane * per + i] : 0.0;
                            if (!done && w > 0.0) {
                                part = lane * per + i;
                                base = run;
                                done = run + w > threshold;
                            }
                            run += w;
                        }
                    }
                    part = __shfl_sync(FULL, part, src);
                    base = __shfl_sync(FULL, base, src);
                    token = find_token<LT>(r, pair, part * part_vecs, min((part + 1) * part_vecs, r.n_vec), base, threshold);
                } else if (pair || r.certain >= 0) {
                    again = true;       // nothing is left over of the target's row: it is drawn from as it stands
                } else {
                    flags |= METASD_STATUS_NONFINITE;       // a row of zeros
                }
                if (!again && lane == 0) {
                    p.accepted_len[b] = n;
                    p.next_token[b] = token;
                }
            }
            if (!again && flags && lane == 0 && p.status) atomicOr(p.status, flags);
            if (lane == 0) sh_again = again;
        }
        __syncthreads();
        if (!sh_again) return;
        r.certain = -1;
        pair = false;
        for (int s = warp; s < parts; s += PROBS_WARPS) {
            const Sums x = sum_part<LT, false>(r, false, s * part_vecs, min((s + 1) * part_vecs, r.n_vec));
            const double w = warp_sum(weight_of(x));
            if (lane == 0) sh_weight[s] = w;
        }
        __syncthreads();
    }
}

// The reward of a round that metasd_verify did not verify, the bandit update and the next selection: a warp per sequence.
__global__ void __launch_bounds__(32) feedback_kernel(const VerifyParams p, const float *d_tv)
{
    __shared__ BanditShared sh;
    launch_dependents();
    grid_dependency_wait();
    const int b = blockIdx.x, lane = threadIdx.x, k = drafted(p.draft_len, b, p.k);
    const BanditStep step = warp_bandit_fetch(p, b, p.st.t[b], p.st.arm[b], sh);
    const double align = p.reward_kind == METASD_REWARD_BD && lane < k ? 1.0 - (double)d_tv[(int64_t)b * p.k + lane] : 0.0;
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
    int cluster = 1;
    while (cluster < 8 && jobs * cluster < 2 * n_sm && p.parts > PROBS_WARPS * cluster) cluster *= 2;
    const unsigned grid = (unsigned)(jobs * cluster);
    if (dtype == METASD_BF16)
        return p.d_tv ? launch_kernel(probs_kernel<__nv_bfloat16, true>, grid, PROBS_THREADS, 0, cluster, true, stream, p)
                      : launch_kernel(probs_kernel<__nv_bfloat16, false>, grid, PROBS_THREADS, 0, cluster, true, stream, p);
    return p.d_tv ? launch_kernel(probs_kernel<float, true>, grid, PROBS_THREADS, 0, cluster, true, stream, p)
                  : launch_kernel(probs_kernel<float, false>, grid, PROBS_THREADS, 0, cluster, true, stream, p);
}

cudaError_t launch_feedback(const VerifyParams &p, const float *d_tv, cudaStream_t stream)
{
    return launch_kernel(feedback_kernel, (unsigned)p.batch, 32, 0, 1, true, stream, p, d_tv);
}

}  // namespace metasd
