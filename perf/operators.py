"""What stands next to the draft-verify round in a serving loop: verification from probabilities and given random numbers, and
the block tables and slot maps of the sequences' caches.

A program whose samplers cut the distributions (top-k, min-p, penalties) holds probabilities, not logits, and draws its random
numbers itself: ``verify_probs`` takes both.  Every round it also has to say where the caches' new entries go: the tokens that
each sequence adds to the cache of the model it runs on (the target, or the drafter its bandit chose, which may have fallen
behind), grouped by model, with blocks taken from and given back to each model's pool: ``BlockCache.plan`` and ``release``.

A pass of a "verify" case is one ``verify_probs`` call; a pass of a "cache" case is a plan and the release of what it took (the
drafts were all rejected), which leaves the pools as they were.
"""
import math

import numpy as np
import torch

own = False

SIZE = {"bf16": 2, "fp32": 4}
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}

# Fields of a "verify" case
#   B sequences, k drafted tokens (0: a plain draw from the target), V vocabulary, dtype of the probabilities
#   draft    "rows": the drafter's probabilities;  "tokens": tokens alone (a lookup drafter, certain of what it proposes)
#   tv       the distances d_TV of all k rows are asked for (they feed the bandits), so that every row is read
#   ragged   per-sequence draft lengths in 0 .. k
#   grouped  the drafter's rows lie in the order in which the drafters ran, not in the sequences'
#   pitch    rows are padded to a multiple of 64 entries
#   min_p    entries below this share of the row's largest are cut to zero
VERIFY = dict(kind="verify", dtype="fp32", draft="rows", tv=False, ragged=False, grouped=False, pitch=False, min_p=0.0)

# Fields of a "cache" case
#   B sequences, pools (models with a cache each), page (tokens a block), context (longest sequence), lag (most tokens by which
#   a model's cache may be behind; a third of them are), step (most tokens a round adds), idle (share of sequences that take no
#   part), scarce (the pools have too few free blocks for all)
CACHE = dict(kind="cache", pools=1, page=16, context=4096, lag=0, step=6, idle=0.0, scarce=False)


def _case(base, name, **kw):
    case = dict(base, **kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one chat session on a small model: all latency
        _case(VERIFY, "one_session", B=1, k=4, V=32000),
        # a handful of sessions on a large vocabulary, with the distances
        _case(VERIFY, "few_sessions", B=4, k=8, V=152064, dtype="bf16", tv=True),
        # a vocabulary that is no multiple of anything, drafts of different lengths, rows as the drafters left them
        _case(VERIFY, "odd_ragged", B=96, k=5, V=50257, tv=True, ragged=True, grouped=True),
        # a large batch whose bandits are fed with the distances: every row is read
        _case(VERIFY, "rewarded_batch", B=256, k=7, V=128256, dtype="bf16", tv=True),
        # the largest batch without distances, min-p sampling: one row pair per sequence
        _case(VERIFY, "largest_batch", B=512, k=8, V=152064, min_p=0.02),
        # drafts from a lookup in the prompt, which have no probabilities
        _case(VERIFY, "lookup_drafts", B=64, k=16, V=128256, draft="tokens", pitch=True),
        # no drafts at all: one token per sequence, odd vocabulary
        _case(VERIFY, "single_tokens", B=256, k=0, V=32001, dtype="bf16"),
        # the target's cache of one session
        _case(CACHE, "one_cache", B=1, context=2000),
        # the target's caches of a large batch: k + 1 tokens each
        _case(CACHE, "target_caches", B=1024, context=8192, step=9),
        # the chosen drafters' caches: grouped by drafter, some far behind, some sequences idle
        _case(CACHE, "drafter_caches", B=256, pools=8, context=4096, lag=600, step=5, idle=0.1),
        # an odd block size, and pools that run out of blocks
        _case(CACHE, "scarce_blocks", B=333, pools=3, page=24, context=1500, lag=300, step=8, scarce=True),
        # prompts of a large batch: millions of new entries
        _case(CACHE, "prompts", B=1024, page=64, context=8192, lag=8192, step=1),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        if rng.random() < 0.6:
            k = rng.choice([0, 1, rng.randint(2, 8), rng.randint(2, 8), rng.randint(9, 16)])
            V = _log_uniform(rng, 4000, 262144)
            if rng.random() < 0.6:
                V -= V % 8
            rows = k > 0 and rng.random() < 0.75
            case = _case(VERIFY, None, B=_log_uniform(rng, 1, 1024), k=k, V=V, dtype=rng.choice(["fp32", "fp32", "bf16"]),
                         draft="rows" if rows else "tokens", tv=k > 0 and rng.random() < 0.5, ragged=k > 0 and rng.random() < 0.3,
                         grouped=rows and rng.random() < 0.3, pitch=rng.random() < 0.2, min_p=rng.choice([0.0, 0.0, 0.02, 0.1]))
            if case["B"] * (2 * k + 1) * V <= 1.3e9 and work(case)["bytes"] <= 9e8:
                return case
        else:
            pools = rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 16)])
            context = _log_uniform(rng, 16, 16384)
            case = _case(CACHE, None, B=_log_uniform(rng, 1, 2048), pools=pools, page=rng.choice([1, 8, 16, 32, 64, rng.randint(2, 100)]),
                         context=context, lag=rng.choice([0, 0, rng.randint(0, context), context]), step=rng.randint(1, 17),
                         idle=rng.choice([0.0, 0.0, round(rng.random(), 2)]), scarce=rng.random() < 0.2)
            if case["B"] * context <= 8e6 and pools * case["B"] * (context // case["page"] + 2) <= 4e6:
                return case


# ---------------------------------------------------------------------------------------------------------------- inputs

def _verify_inputs(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    B, k, V = case["B"], case["k"], case["V"]
    dtype = DTYPE[case["dtype"]]
    pitch = (V + 63) // 64 * 64 if case["pitch"] else V
    rows = case["draft"] == "rows" and k > 0
    prior = -1.1 * torch.log(torch.arange(1, V + 1, device=dev, dtype=torch.float32))
    target = torch.zeros((B, k + 1, pitch), dtype=dtype, device=dev)[..., :V]
    draft = torch.zeros((B, k, pitch), dtype=dtype, device=dev)[..., :V] if rows else None
    tokens = torch.zeros((B, k), dtype=torch.int32, device=dev)
    place = torch.randperm(B, generator=g, device=dev).to(torch.int32) if case["grouped"] else None

    def probabilities(logits):
        p = torch.softmax(logits, dim=-1)
        if case["min_p"]:
            p = torch.where(p < case["min_p"] * p.amax(dim=-1, keepdim=True), 0.0, p)
            p /= p.sum(dim=-1, keepdim=True)
        return p

    step = max(1, int(1e8) // ((k + 1) * V))
    for b in range(0, B, step):
        n = min(step, B - b)
        logits = 3.0 * torch.randn((n, k + 1, V), generator=g, device=dev) + prior
        p = probabilities(logits)
        target[b:b + n] = p
        if k == 0:
            continue
        if rows:
            sigma = 0.2 + 2.0 * torch.rand((n, 1, 1), generator=g, device=dev)     # drafters of different quality
            p = probabilities(logits[:, :k] + sigma * torch.randn((n, k, V), generator=g, device=dev))
            if place is None:
                draft[b:b + n] = p
            else:
                draft[place[b:b + n].long()] = p.to(dtype)
        drawn = torch.multinomial(p[:, :k].reshape(n * k, V), 1, generator=g).reshape(n, k)
        if not rows:    # a lookup is right about half of the time
            likely = p[:, :k].argmax(dim=-1)
            drawn = torch.where(torch.rand((n, k), generator=g, device=dev) < 0.5, likely, drawn)
        tokens[b:b + n] = drawn.to(torch.int32)
    s = dict(case, target=target, draft=draft, tokens=tokens if k else None, place=place,
             u_accept=torch.rand((B, k), generator=g, device=dev) if k else None, u_draw=torch.rand(B, generator=g, device=dev),
             lengths=torch.randint(0, k + 1, (B,), generator=g, device=dev).to(torch.int32) if case["ragged"] else None,
             accepted=torch.zeros(B, dtype=torch.int32, device=dev), next=torch.zeros(B, dtype=torch.int32, device=dev),
             d_tv=torch.zeros((B, k), dtype=torch.float32, device=dev) if case["tv"] else None)
    return s


def _lengths(case, seed):
    """Host arrays: tokens in each model's cache [pools, B], lengths after the round [B], the model of each sequence [B]."""
    rng = np.random.default_rng(seed)
    B, P = case["B"], case["pools"]
    context = rng.integers(case["context"] // 2, case["context"] + 1, size=B)
    behind = np.where(rng.random((P, B)) < 0.35, rng.integers(0, case["lag"] + 1, size=(P, B)), 0)
    if case["lag"] >= case["context"]:
        behind = np.maximum(behind, context)      # nothing is cached yet
    cached = np.maximum(context - behind, 0)
    length = context + rng.integers(1, case["step"] + 1, size=B)
    pool = np.where(rng.random(B) < case["idle"], -1, rng.integers(0, P, size=B))
    return cached, length, pool


def _need(case, cached, length, pool):
    """Host: new tokens [B] and new blocks [B] of the sequences that take part."""
    at = np.maximum(pool, 0), np.arange(case["B"])
    new = np.where(pool >= 0, length - cached[at], 0)
    blocks = np.where(pool >= 0, -(-length // case["page"]) + -cached[at] // case["page"], 0)
    return new, blocks


def _room(case):
    """Entries that the output buffers have room for: those of a captured graph, which are made once for rounds of any lengths."""
    most = min(case["lag"], case["context"]) + case["step"]
    new, _ = _need(case, *_lengths(case, 0))
    room = min(case["B"] * most, int(1.1 * new.sum() + 6.0 * math.sqrt(case["B"]) * most))
    return (room + 63) // 64 * 64


def _cache_inputs(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    B, P, page = case["B"], case["pools"], case["page"]
    cached, length, pool = _lengths(case, seed)
    _, blocks = _need(case, cached, length, pool)
    held = -(-cached // page)
    most = int(-(-(case["context"] + case["step"]) // page))
    share = 0.8 if case["scarce"] else 1.0
    spare = [int(share * blocks[pool == i].sum()) + (0 if case["scarce"] else 3) for i in range(P)]
    n_blocks = B * most + 4
    table = torch.full((P, B, most), -1, dtype=torch.int32, device=dev)
    free = torch.full((P, n_blocks), -1, dtype=torch.int32, device=dev)
    lasting = torch.from_numpy(held).to(dev)
    for i in range(P):      # blocks in no order, as a pool that has been in use for a while hands them out
        ids = torch.randperm(n_blocks, generator=g, device=dev).to(torch.int32)
        used = int(held[i].sum())
        table[i][torch.arange(most, device=dev)[None] < lasting[i][:, None]] = ids[:used]
        free[i, :spare[i]] = ids[used:used + spare[i]]
    room = _room(case)

    def ints(x):
        return torch.from_numpy(np.ascontiguousarray(x)).to(torch.int32).to(dev)

    return dict(case, table=table, held=ints(held), free=free, count=ints(np.array(spare)), cached=ints(cached), length=ints(length),
                pool=ints(pool) if P > 1 or case["idle"] else None, room=room,
                order=ints(np.zeros(B)), place=ints(np.zeros(B)), pool_start=ints(np.zeros(P + 1)), token_start=ints(np.zeros(B + 1)),
                slots=torch.zeros(room, dtype=torch.int64, device=dev), position=ints(np.zeros(room)), sequence=ints(np.zeros(room)))


def prepare(case, seed):
    return _verify_inputs(case, seed) if case["kind"] == "verify" else _cache_inputs(case, seed)


# ----------------------------------------------------------------------------------------------------------- plain forms

def _plain_verify(s):
    target, draft, k = s["target"], s["draft"], s["k"]
    B, _, V = target.shape
    dev = target.device
    b, ids = torch.arange(B, device=dev), torch.arange(V, device=dev)
    at = b if s["place"] is None else s["place"].long()
    lengths = torch.full((B,), k, device=dev) if s["lengths"] is None else s["lengths"].long()
    accepted = torch.zeros(B, dtype=torch.long, device=dev)
    d_tv = None
    if k:
        j, x = torch.arange(k, device=dev), s["tokens"].long()
        live = j < lengths[:, None]
        px = target[b[:, None], j, x].double()
        qx = draft[at[:, None], j, x].double() if draft is not None else torch.ones_like(px)
        accept = (s["u_accept"].double() * qx < px) & live
        accepted = accept.long().cumprod(1).sum(1)
        if s["tv"]:
            if draft is not None:
                apart = (target[:, :k].float() - draft[at].float()).abs().sum(-1)
            else:
                apart = target[:, :k].float().sum(-1) - px.float() + (1.0 - px.float()).abs()
            d_tv = torch.where(live, 0.5 * apart, 0.0)
    p = target[b, accepted].double()
    w = p
    if k:
        rejected = accepted < lengths
        j = accepted.clamp(max=k - 1)
        q = draft[at, j].double() if draft is not None else (ids == x[b, j][:, None]).double()
        w = torch.where(rejected[:, None], (p - q).clamp_min(0.0), p)
        w = torch.where((w.sum(1) > 0.0)[:, None], w, p)      # nothing left over: the target's own row
    c = w.cumsum(1)
    token = (c <= s["u_draw"].double()[:, None] * c[:, -1:]).sum(1)
    token = torch.minimum(token, ((w > 0.0) * ids).amax(1))
    out = [accepted.int(), token.int()]
    return out + [d_tv] if s["tv"] else out


def _plain_plan(s):
    table, held, free, count = s["table"], s["held"].long(), s["free"], s["count"].long()
    (P, B, most), page, room = table.shape, s["page"], s["room"]
    dev = table.device
    b, length = torch.arange(B, device=dev), s["length"].long()
    pool = torch.zeros(B, dtype=torch.long, device=dev) if s["pool"] is None else s["pool"].long()
    part = pool >= 0
    g = pool.clamp_min(0)
    cached, has = s["cached"].long()[g, b], held[g, b]
    new = torch.where(part, (length - cached).clamp_min(0), 0)
    need = torch.where(part, ((length + page - 1) // page - has).clamp_min(0), 0)
    # by model, the sequences in order within each; who takes no part comes last
    key = torch.where(part, pool, P)
    order = torch.argsort(key, stable=True)
    place = torch.empty_like(order).scatter(0, order, b)
    zero = torch.zeros(1, dtype=torch.long, device=dev)
    pool_start = torch.cat([zero, (key[None] == torch.arange(P, device=dev)[:, None]).sum(1).cumsum(0)])
    token_start = torch.cat([zero, new[order].cumsum(0)])
    # the pool's free blocks from the end, to one sequence after the other while there are enough
    before = torch.cat([zero, need[order].cumsum(0)])
    before = (before[:-1] - before[pool_start][key[order]])[place]
    served = (need == 0) | (before + need <= count[g])
    taken = torch.where(served, need, 0)
    # entry by entry
    t = torch.arange(room, device=dev)
    live = t < token_start[-1]
    at = torch.searchsorted(token_start[1:], t, right=True).clamp(max=B - 1)
    q = order[at]
    position = cached[q] + t - token_start[at]
    block = (position // page).clamp(0, most - 1)
    fresh = block >= has[q]
    pick = (count[g[q]] - 1 - before[q] - block + has[q]).clamp_min(0)
    block_id = torch.where(fresh, free[g[q], pick], table[g[q], q, block]).long()
    slots = torch.where(served[q], block_id * page + position % page, -1)
    writes = live & fresh & served[q]
    where = torch.where(writes, (g[q] * B + q) * most + block, P * B * most)
    flat = torch.cat([table.reshape(-1), table.new_zeros(1)])
    flat[where] = torch.where(writes, block_id, 0).int()
    table.copy_(flat[:-1].reshape(P, B, most))
    s["held"].copy_(held.index_put((g, b), taken, accumulate=True).int())
    s["count"].copy_((count - torch.zeros_like(count).index_add(0, g, taken)).int())
    return [order.int(), place.int(), pool_start.int(), token_start.int(), torch.where(live, slots, 0),
            torch.where(live, position, 0).int(), torch.where(live, q, 0).int()]


def _plain_release(s, keep):
    table, held, free, count = s["table"], s["held"].long(), s["free"], s["count"].long()
    (P, B, most), n_blocks, page = table.shape, free.shape[1], s["page"]
    dev = table.device
    want = (keep.long() + page - 1) // page
    drop = (held - want).clamp_min(0)
    ends = drop.cumsum(1)
    total = ends[:, -1:]
    e = torch.arange(n_blocks, device=dev).expand(P, n_blocks).contiguous()
    live = e < total
    b = torch.searchsorted(ends, e, right=True).clamp(max=B - 1)
    pools = torch.arange(P, device=dev)[:, None]
    block = (want[pools, b] + e - (ends - drop)[pools, b]).clamp(0, most - 1)
    to = torch.where(live, count[:, None] + total - 1 - e, n_blocks)
    wide = torch.cat([free, free.new_zeros((P, 1))], 1)
    wide.scatter_(1, to, torch.where(live, table[pools, b, block], 0))
    free.copy_(wide[:, :-1])
    s["held"].copy_((held - drop).int())
    s["count"].copy_((count + total[:, 0]).int())


def run(s):
    if own:
        from paper_2604_05417_b200 import binding as M
        if s["kind"] == "verify":
            out = M.ProbsResult(s["accepted"], s["next"], s["d_tv"])
            M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], draft_len=s["lengths"],
                           draft_place=s["place"], want_d_tv=s["tv"], out=out)
            return [s["accepted"], s["next"]] + ([s["d_tv"]] if s["tv"] else [])
        if "cache" not in s:
            s["cache"] = M.BlockCache(s["table"], s["held"], s["free"], s["count"], s["page"])
            s["plan"] = M.CachePlan(s["order"], s["place"], s["pool_start"], s["token_start"], s["slots"], s["position"],
                                    s["sequence"])
        s["cache"].plan(s["length"], s["cached"], pool=s["pool"], out=s["plan"])
        s["cache"].release(s["cached"])
        got = [s["order"], s["place"], s["pool_start"], s["token_start"], s["slots"], s["position"], s["sequence"]]
    elif s["kind"] == "verify":
        return _plain_verify(s)
    else:
        got = _plain_plan(s)
        _plain_release(s, s["cached"])
    return got + [s["table"], s["held"], s["free"], s["count"]]


# ------------------------------------------------------------------------------------------------------ in 64 bits, apart

def _exact_verify(s):
    B, k, V = s["B"], s["k"], s["V"]
    accepted, token, d_tv = np.zeros(B, np.int64), np.zeros(B, np.int64), np.zeros((B, k))
    place = np.arange(B) if s["place"] is None else s["place"].cpu().numpy()
    lengths = np.full(B, k) if s["lengths"] is None else s["lengths"].cpu().numpy()
    u_draw = s["u_draw"].cpu().numpy().astype(np.float64)
    if k:
        tokens, u = s["tokens"].cpu().numpy(), s["u_accept"].cpu().numpy().astype(np.float64)
    for b in range(B):
        target = s["target"][b]
        if k:
            x = torch.from_numpy(tokens[b]).long().to(target.device)
            if s["draft"] is None:
                draft = torch.nn.functional.one_hot(x, V)
            else:
                draft = s["draft"][place[b]]
            at = torch.arange(k, device=x.device)
            px, qx = (v.double().cpu().numpy() for v in (target[at, x], draft[at, x]))
            if s["tv"]:
                n = lengths[b]
                d_tv[b, :n] = (target[:n].double() - draft[:n].double()).abs().sum(1).cpu().numpy() / 2
        n = 0
        while n < lengths[b] and u[b, n] * qx[n] < px[n]:
            n += 1
        accepted[b] = n
        w = target[n].double()
        if n < lengths[b]:
            left = torch.relu(w - draft[n].double())
            w = left if bool((left > 0).any()) else w
        w = w.cpu().numpy()
        reach = np.cumsum(w)
        token[b] = min(np.searchsorted(reach, u_draw[b] * reach[-1], side="right"), np.flatnonzero(w)[-1])
    out = [accepted, token]
    return out + [d_tv] if s["tv"] else out


def _exact_cache(s):
    P, B, most = s["table"].shape
    page, room = s["page"], s["room"]
    table, held, free, count, cached, length = (s[n].cpu().numpy().astype(np.int64)
                                                for n in ("table", "held", "free", "count", "cached", "length"))
    pool = np.zeros(B, np.int64) if s["pool"] is None else s["pool"].cpu().numpy()
    first = held.copy()
    order, starts, token_start = [], [0], [0]
    slots, position, sequence = (np.zeros(room, np.int64) for _ in range(3))
    for i in list(range(P)) + [-1]:
        short = False
        for b in np.flatnonzero(pool == i):
            order.append(b)
            if i < 0:
                token_start.append(token_start[-1])
                continue
            pos = np.arange(cached[i, b], max(length[b], cached[i, b]))
            t = token_start[-1]
            token_start.append(t + len(pos))
            need = max(0, -(-length[b] // page) - held[i, b])
            short = need > 0 and (short or need > count[i])
            if need and not short:
                table[i, b, held[i, b]:held[i, b] + need] = free[i, count[i] - need:count[i]][::-1]
                held[i, b] += need
                count[i] -= need
            failed = need and short
            slots[t:t + len(pos)] = -1 if failed else table[i, b, pos // page] * page + pos % page
            position[t:t + len(pos)], sequence[t:t + len(pos)] = pos, b
            short = short or failed
        if i >= 0:
            starts.append(len(order))
    for i in range(P):
        back = []
        for b in range(B):
            back += table[i, b, -(-cached[i, b] // page):held[i, b]].tolist()
            held[i, b] = min(held[i, b], -(-cached[i, b] // page))
        free[i, count[i]:count[i] + len(back)] = back[::-1]
        count[i] += len(back)
    place = np.zeros(B, np.int64)
    place[np.array(order)] = np.arange(B)
    assert np.array_equal(held, np.minimum(first, -(-cached // page)))
    return [np.array(order), place, np.array(starts), np.array(token_start), slots, position, sequence, table, held, free, count]


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_verify(s) if case["kind"] == "verify" else _exact_cache(s)


# ------------------------------------------------------------------------------------------------------------------ work

def work(case):
    if case["kind"] == "verify":
        B, k, V = case["B"], case["k"], case["V"]
        mean = k / 2 if case["ragged"] else k
        sides = 2 if case["draft"] == "rows" and k else 1
        # with distances every drafted row (pair), else the one that the next token is drawn from
        rows = B * sides * (mean if case["tv"] else 1)
        # subtract, cut at zero, add; the same for the distance's absolute value
        flops = rows * V * (3.0 if case["tv"] else 2.0)
        small = B * (k * 24 + 16)
        return {"bytes": float(rows * V * SIZE[case["dtype"]] + small), "flops": float(flops)}
    cached, length, pool = _lengths(case, 0)
    new, blocks = _need(case, cached, length, pool)
    B, P = case["B"], case["pools"]
    # slot, position and sequence of every entry; each new block's id read and written by the plan and by the release
    moved = 16.0 * new.sum() + 16.0 * blocks.sum() + B * 36.0 + P * B * 8.0 + P * 24.0
    return {"bytes": float(moved), "flops": float(8 * new.sum() + 20 * B)}
