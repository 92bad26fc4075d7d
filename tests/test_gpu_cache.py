"""metasd_cache_plan and metasd_cache_release on the GPU against a plain Python walk: every number is equal."""
import numpy as np
import pytest
import torch

from _cache_reference import Caches
from paper_2604_05417_b200 import binding as M

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)


def ints(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).to(DEV)


def same(cache, ref):
    """Tables (as far as they count), free lists and counts."""
    held, count = cache.held.cpu().numpy(), cache.free_count.cpu().numpy()
    table, free = cache.block_table.cpu().numpy(), cache.free_blocks.cpu().numpy()
    for g in range(ref.pools):
        assert count[g] == len(ref.free[g]) and free[g, :count[g]].tolist() == ref.free[g]
        for b in range(ref.batch):
            assert table[g, b, :held[g, b]].tolist() == ref.table[g][b], (g, b)


def pair(pools, batch, max_blocks, n_blocks, page, seed=0):
    """Empty caches on both sides, with pools that hand out blocks in no order."""
    rng = np.random.default_rng(seed)
    free = np.stack([rng.permutation(n_blocks) for _ in range(pools)])
    cache = M.BlockCache.empty(pools, batch, max_blocks, n_blocks, page)
    cache.free_blocks.copy_(ints(free))
    return cache, Caches(pools, batch, max_blocks, page, free.tolist())


def plan_both(cache, ref, length, cached, pool=None, room=None, outputs=None):
    """One plan on both sides; every output is compared, what lies behind the last entry too."""
    B = len(length)
    cached = np.asarray(cached)
    want = ref.plan(length, np.broadcast_to(cached, (ref.pools, B)), pool, room or (1 << 30))
    room = room or max(1, len(want[4]) + 5)
    out = outputs or M.CachePlan(*[ints(np.full(n, -7)) for n in (B, B, ref.pools + 1, B + 1)],
                                 torch.full((room,), -7, dtype=torch.int64, device=DEV), ints(np.full(room, -7)), ints(np.full(room, -7)))
    cache.plan(ints(length), ints(cached), pool=None if pool is None else ints(pool), out=out)
    for got, ref_out in zip((out.order, out.place, out.pool_start, out.token_start), want[:4]):
        assert got is None or got.tolist() == ref_out
    n = len(want[4])
    for i, got in enumerate((out.slot_map, out.position, out.sequence)):
        if got is not None:
            assert got[:n].tolist() == [e[i] for e in want[4]]
            assert (got[n:] == -7).all()
    same(cache, ref)
    return out, want


@pytest.mark.parametrize("pools,batch,page", [(1, 1, 16), (1, 1, 1), (1, 31, 16), (3, 33, 7), (8, 64, 16), (32, 100, 3), (2, 1025, 5), (5, 2100, 64)])
def test_rounds_of_a_serving_loop(pools, batch, page):
    """Prompts, rounds with rejected drafts, finished queries and drafters that have fallen behind."""
    rng = np.random.default_rng(batch)
    most = 40
    cache, ref = pair(pools, batch, most, batch * most, page, seed=1)
    lengths = rng.integers(0, 20 * page + 1, size=batch)        # committed tokens; a few sequences have none yet
    cached = np.zeros((pools, batch), dtype=np.int64)
    for t in range(6):
        pool = rng.integers(-1, pools, size=batch) if t else rng.integers(0, pools, size=batch)
        goal = np.minimum(lengths + rng.integers(0, 6, size=batch), most * page)
        plan_both(cache, ref, goal, cached, pool)
        at = np.maximum(pool, 0), np.arange(batch)
        cached[at] = np.where(pool >= 0, np.maximum(cached[at], goal), cached[at])
        lengths = np.minimum(lengths + rng.integers(0, 4, size=batch), goal)
        done = rng.random(batch) < 0.1
        lengths[done] = 0
        cached = np.minimum(cached, lengths)                    # what was rejected or finished is not kept
        cache.release(ints(cached))
        ref.release(cached)
        same(cache, ref)
    assert cache.last_status() == 0


@pytest.mark.parametrize("lengths", [[70000], [1, 1, 70000, 1], [0] * 700 + [30000] + [0] * 700 + [9000] + [0] * 3, [2049, 2047, 2048, 0, 1, 4096]])
def test_long_and_uneven_prompts(lengths):
    """Entries of one sequence over many blocks of threads; places without entries between them."""
    cache, ref = pair(1, len(lengths), 4400, 6000, 16, seed=2)
    plan_both(cache, ref, lengths, np.zeros(len(lengths), dtype=np.int64))
    cache.release(ints(np.zeros(len(lengths))))
    ref.release([[0] * len(lengths)])
    same(cache, ref)
    assert cache.free_count.tolist() == [6000]


@pytest.mark.parametrize("batch,pools", [(9000, 3), (65535, 1), (20000, 16)])
def test_very_many_sequences(batch, pools):
    """More sequences than a block has threads, and than its shared memory has places."""
    rng = np.random.default_rng(batch)
    page, most = 4, 5
    cache, ref = pair(pools, batch, most, batch * 3, page, seed=batch)
    cached = np.zeros((pools, batch), dtype=np.int64)
    pool = rng.integers(-1, pools, size=batch)
    goal = np.where(rng.random(batch) < 0.3, rng.integers(0, most * page + 1, size=batch), 0)
    plan_both(cache, ref, goal, cached, pool if pools > 1 else None)
    keep = np.minimum(rng.integers(0, most * page, size=(pools, batch)), goal)
    cache.release(ints(keep))
    ref.release(keep)
    same(cache, ref)
    have = np.zeros((pools, batch), dtype=np.int64)
    at = np.maximum(pool, 0), np.arange(batch)
    have[at] = np.where(pool >= 0, keep[at], 0) if pools > 1 else keep[0]
    plan_both(cache, ref, goal, have, pool if pools > 1 else None)


def test_tables_beyond_32_bits():
    """Block tables with more than 2^31 entries in all, and more blocks in a step than 2^31 if everyone took all."""
    batch, most = 60000, 18000
    cache = M.BlockCache.empty(2, batch, most, 200000, 16)
    assert cache.block_table.numel() > 2 ** 31
    lengths = np.zeros(batch, dtype=np.int64)
    lengths[[0, 777, 40000, batch - 1]] = [5, 16 * 300, 16 * most, 33]
    pool = np.ones(batch, dtype=np.int64)
    out = cache.plan(ints(lengths), ints(np.zeros(batch)), pool=ints(pool), max_tokens=400000)
    assert cache.last_status() == 0
    need = -(-lengths // 16)
    first = 0
    for b in np.flatnonzero(lengths):
        ids = np.arange(first, first + need[b])      # the pool hands out 0, 1, 2, ..
        assert np.array_equal(cache.block_table[1, b, :need[b]].cpu().numpy(), ids)
        start = int(out.token_start[int(out.place[b])])
        assert np.array_equal(out.slot_map[start:start + lengths[b]].cpu().numpy(), first * 16 + np.arange(lengths[b]))
        first += need[b]
    assert int(cache.held[1].sum()) == first and int(cache.free_count[1]) == 200000 - first
    cache.release(ints(np.zeros(batch)))
    assert cache.last_status() == 0 and cache.free_count.tolist() == [200000, 200000]
    assert torch.equal(cache.free_blocks[0], cache.free_blocks[1]) and int(cache.held.sum()) == 0


def test_the_longest_table():
    """One sequence with 2^31 - 1 blocks of one entry: planned, and given back."""
    n = 2 ** 31 - 1
    def blocks():
        return torch.arange(n - 1, -1, -1, dtype=torch.int32, device=DEV)
    cache = M.BlockCache(torch.full((1, 1, n), -1, dtype=torch.int32, device=DEV), ints([[0]]), blocks().view(1, n), ints([n]), 1)
    out = M.CachePlan(None, None, None, ints([-7, -7]), torch.full((n,), -7, dtype=torch.int64, device=DEV), None, None)
    cache.plan(ints([n]), ints([0]), out=out)
    assert out.token_start.tolist() == [0, n] and cache.held.item() == n and cache.free_count.item() == 0 and cache.last_status() == 0
    for t in (out.slot_map, cache.block_table[0, 0]):      # the pool hands out 0, 1, 2, ..
        for at in range(0, n, 2 ** 28):
            part = t[at:at + 2 ** 28]
            assert torch.equal(part, torch.arange(at, at + len(part), dtype=t.dtype, device=DEV))
    del out
    cache.free_blocks.fill_(-1)
    cache.release(ints([0]))
    assert cache.free_count.item() == n and cache.held.item() == 0 and cache.last_status() == 0
    assert torch.equal(cache.free_blocks[0], blocks())


@pytest.mark.parametrize("batch,pools,page,longest", [(3, 2, 1, 5000), (45, 1, 1, 3000), (200, 2, 1, 1500), (700, 1, 2, 700), (70, 3, 3, 3100)])
def test_releases_of_uneven_tables(batch, pools, page, longest):
    """A few long tables among short and empty ones: a row's blocks given back by one warp each, and by all together."""
    rng = np.random.default_rng(longest)
    most = -(-longest // page)
    cache, ref = pair(pools, batch, most, batch * most // 4 + 4 * most, page, seed=batch)
    for t in range(3):
        goal = np.where(rng.random(batch) < 0.1, rng.integers(longest // 2, longest + 1, size=batch), rng.integers(0, 40, size=batch))
        goal[rng.random(batch) < 0.4] = 0
        for g in range(pools):
            have = np.array([[len(ref.table[i][b]) * page for b in range(batch)] for i in range(pools)])
            plan_both(cache, ref, np.maximum(goal, have[g]), have, np.full(batch, g))
        keep = np.where(rng.random((pools, batch)) < 0.5, 0, rng.integers(0, longest, size=(pools, batch)))
        cache.release(ints(keep))
        ref.release(keep)
        same(cache, ref)
    cache.release(ints(np.zeros(batch)))
    ref.release(np.zeros((pools, batch)))
    same(cache, ref)
    assert cache.last_status() in (0, M.STATUS_NO_BLOCKS)


def test_a_release_undoes_a_plan():
    cache, ref = pair(4, 50, 30, 800, 8, seed=3)
    rng = np.random.default_rng(3)
    cached = np.zeros((4, 50), dtype=np.int64)
    before = cache.free_blocks.clone()
    a, _ = plan_both(cache, ref, rng.integers(1, 200, size=50), cached, rng.integers(0, 4, size=50))
    cache.release(ints(cached))
    ref.release(cached)
    same(cache, ref)
    assert torch.equal(cache.free_blocks, before)


def test_too_few_blocks():
    """From the first sequence on that cannot be served none of its pool gets blocks; those that need none are planned."""
    cache, ref = pair(2, 8, 10, 9, 4, seed=4)
    plan_both(cache, ref, [8, 8, 3, 4, 4, 1, 2, 8], [0] * 8, [0, 0, 0, 0, 1, 1, 1, 1])
    assert cache.last_status() == 0
    cached = [[8, 8, 3, 4, 0, 0, 0, 0], [0, 0, 0, 0, 4, 1, 2, 8]]
    out, want = plan_both(cache, ref, [10, 30, 4, 5, 6, 2, 40, 9], cached, [0, 0, 0, 0, 1, 1, 1, 1])
    slots = [e for e in want[4] if e[0] >= 0]
    assert {e[2] for e in slots} == {0, 2, 4, 5} and cache.last_status() == M.STATUS_NO_BLOCKS
    # with room again the same step is planned
    cache.release(ints([0, 8, 3, 4, 4, 1, 0, 0]))
    ref.release([[0, 8, 3, 4, 4, 1, 0, 0]] * 2)
    same(cache, ref)
    plan_both(cache, ref, [0, 12, 4, 5, 6, 2, 0, 0], np.minimum(cached, [0, 8, 3, 4, 4, 1, 0, 0]), [0, 0, 0, 0, 1, 1, 1, 1])


@pytest.mark.parametrize("room", [1, 2, 7, 99, 2048, 2049])
def test_steps_with_more_entries_than_the_outputs_have_room_for(room):
    lengths = [3, 40, 2000, 5, 0, 7, 100]
    cache, ref = pair(1, 7, 300, 2000, 8, seed=5)
    plan_both(cache, ref, lengths, [0] * 7, room=room)
    assert cache.last_status() == (M.STATUS_TRUNCATED if sum(lengths) > room else 0)


def test_lengths_pools_and_counts_outside_their_range():
    cache, ref = pair(2, 6, 4, 30, 8, seed=6)
    plan_both(cache, ref, [8] * 6, [0] * 6, [0, 0, 0, 1, 1, 1])
    cached = [[8, 8, 8, 0, 0, 0], [0, 0, 0, 8, 8, 8]]
    # beyond the table, negative, beyond what is cached
    plan_both(cache, ref, [33, -1, 12, 32, 9, 9], np.where(np.arange(6) == 4, 9, cached), [0, 0, 0, 1, 1, 1])
    assert cache.last_status() == M.STATUS_BAD_LENGTH
    plan_both(cache, ref, [13] * 6, np.minimum(cached, 8), [0, 2, 99, -1, 2 ** 31 - 1, -2 ** 31])
    assert cache.last_status() == M.STATUS_BAD_INDEX
    plan_both(cache, ref, [2 ** 31 - 1] * 6, [0] * 6)
    assert cache.last_status() == M.STATUS_BAD_LENGTH
    cache.release(ints([-1, 2 ** 31 - 1, 0, 8, 1, -2 ** 31]))
    ref.release([[-1, 2 ** 31 - 1, 0, 8, 1, -2 ** 31]] * 2)
    same(cache, ref)
    assert cache.last_status() == M.STATUS_BAD_LENGTH
    # counts that were written over: everything stays inside the buffers, and is flagged
    cache.held[0, 0], cache.free_count[1] = 1000, -5
    cache.plan(ints([32] * 6), ints([0] * 6), max_tokens=400)
    assert cache.last_status() & M.STATUS_BAD_STATE
    cache.held.fill_(4)
    cache.free_count.fill_(30)
    cache.release(ints([0] * 6))        # more blocks than the lists have room for
    assert cache.last_status() == M.STATUS_BAD_STATE and cache.free_count.tolist() == [30, 30]


def test_slots_beyond_32_bits():
    page = 1 << 20
    cache = M.BlockCache.empty(1, 2, 3, 8, page)
    cache.free_blocks[0, :8] = torch.tensor([2 ** 31 - 1 - i for i in range(8)], dtype=torch.int64).int().to(DEV)
    cache.block_table[0, 1, 0] = 2 ** 31 - 9
    cache.held[0, 1] = 1
    out = cache.plan(ints([3, page + 2]), ints([0, page - 2]), max_tokens=64)
    first, second = 2 ** 31 - 8, 2 ** 31 - 7
    assert out.token_start.tolist() == [0, 3, 7]
    assert out.slot_map[:7].tolist() == [first * page + i for i in range(3)] + [(2 ** 31 - 9) * page + page - 2 + i for i in range(2)] + [
        second * page + i for i in range(2)]


def test_outputs_that_are_not_asked_for_and_unaligned_ones():
    cache, ref = pair(2, 40, 20, 900, 4, seed=7)
    rng = np.random.default_rng(7)
    lengths, pool = rng.integers(0, 60, size=40), rng.integers(0, 2, size=40)
    room = int(lengths.sum()) + 3
    slots = torch.full((room + 1,), -7, dtype=torch.int64, device=DEV)[1:]
    positions = torch.full((room + 1,), -7, dtype=torch.int32, device=DEV)[1:]
    plan_both(cache, ref, lengths, [0] * 40, pool, room, M.CachePlan(None, None, None, ints(np.full(41, -7)), slots, positions, None))
    cache.release(ints([0] * 40))
    ref.release([[0] * 40] * 2)
    plan_both(cache, ref, lengths, [0] * 40, pool, room, M.CachePlan(None, ints(np.full(40, -7)), None, ints(np.full(41, -7)),
                                                                     slots.clone().fill_(-7), None, None))


def test_fewer_sequences_than_the_cache_has():
    cache, ref = pair(2, 100, 8, 300, 4, seed=8)
    plan_both(cache, ref, [9] * 37, [0] * 37, [b % 2 for b in range(37)])
    cache.release(ints([4] * 20))
    ref.release([[4] * 20] * 2)
    same(cache, ref)


@pytest.mark.parametrize("step", [3, 400])
def test_captured_and_replayed_on_another_stream(step):
    """A captured step is planned anew at every replay, from what the tables and lengths then hold."""
    batch, page = 24, 8
    cache, ref = pair(3, batch, 200, 4000, page, seed=9)
    rng = np.random.default_rng(9)
    length, cached, pool = ints(np.zeros(batch)), ints(np.zeros((3, batch))), ints(rng.integers(0, 3, size=batch))
    room = batch * step
    out = M.CachePlan(*[ints(np.full(n, -7)) for n in (batch, batch, 4, batch + 1)],
                      torch.full((room,), -7, dtype=torch.int64, device=DEV), ints(np.full(room, -7)), ints(np.full(room, -7)))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        cache.plan(length, cached, pool=pool, out=out)
        cache.release(cached)
    goal = np.zeros(batch, dtype=np.int64)
    have = np.zeros((3, batch), dtype=np.int64)
    for t in range(3):
        goal = goal + rng.integers(0, step + 1, size=batch)
        length.copy_(ints(goal))
        graph.replay()
        torch.cuda.synchronize()
        want = ref.plan(goal, have, pool.tolist())
        ref.release(have)
        assert out.token_start.tolist() == want[3] if sum(goal) <= room else cache.last_status() == M.STATUS_TRUNCATED
        if sum(goal) <= room:
            assert out.slot_map[:len(want[4])].tolist() == [e[0] for e in want[4]]
        same(cache, ref)


def test_refusals_on_the_device():
    cache = M.BlockCache.empty(2, 8, 4, 30, 8)
    good = dict(length=ints([1] * 8), cached=ints([0] * 8), pool=ints([0] * 8), max_tokens=8)
    cache.plan(**good)
    for name, values in dict(length=[ints([1] * 8).long(), ints([1] * 8).cpu()], cached=[ints([0] * 7), ints(np.zeros((3, 8))), ints([0] * 16)[::2]],
                             pool=[ints([0] * 9), ints([0] * 8).float()], max_tokens=[None]).items():
        for value in values:
            with pytest.raises(ValueError):
                cache.plan(**dict(good, **{name: value}))
    for bad in (ints([0] * 8).long(), ints(np.zeros((3, 8))), ints([0] * 8).cpu()):
        with pytest.raises(ValueError):
            cache.release(bad)
    for n in (0, 9):        # more sequences than there are tables, or none
        with pytest.raises(M.MetasdError):
            cache.plan(ints([1] * n), ints([0] * n), max_tokens=8)
        with pytest.raises(M.MetasdError):
            cache.release(ints([0] * n))
    with pytest.raises(M.MetasdError):
        cache.plan(ints([1] * 8), ints([0] * 8), max_tokens=0)
    with pytest.raises(M.MetasdError):
        M.BlockCache(cache.block_table, cache.held, cache.free_blocks, cache.free_count, 0)
    with pytest.raises(M.MetasdError):
        M.BlockCache.empty(33, 8, 4, 30, 8)
    with pytest.raises(ValueError):
        M.BlockCache(cache.block_table, cache.held.t(), cache.free_blocks, cache.free_count, 8)
