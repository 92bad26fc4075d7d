"""Refusals of metasd_verify_probs, metasd_cache_plan and metasd_cache_release, on the host: before any CUDA call, so that they are
the same with and without a device; and the plain walks that the GPU tests compare with, on cases worked by hand."""
import ctypes as C
import importlib.util
import os
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import _probs_reference as R
from _cache_reference import Caches
from paper_2604_05417_b200 import binding as M
from paper_2604_05417_b200 import build as B
from paper_2604_05417_b200 import study


@pytest.fixture(scope="module")
def lib():
    B.build()
    return M.load_library()


BUFFER = C.create_string_buffer(256)
AT = (C.addressof(BUFFER) + 15) // 16 * 16      # an aligned address; no call below gets as far as using it


def probs_call(lib, **kw):
    a = dict(ctx=None, device=0, batch=4, k=2, vocab=10, dtype=M.FP32, target=AT, tss=30, trs=10, draft=AT, dss=20, drs=10, place=None,
             tokens=AT, draft_len=None, ua=AT, ud=AT, seed=0, acc=AT, tok=AT, d_tv=None, reward=None, status=None, stream=None)
    assert set(kw) <= set(a)
    return lib.metasd_verify_probs(*dict(a, **kw).values())


def test_verify_probs_checks_its_arguments(lib):
    for kw in (dict(batch=0), dict(batch=65536), dict(k=-1), dict(k=17), dict(vocab=0), dict(target=None), dict(ud=None), dict(acc=None),
               dict(tok=None), dict(tokens=None), dict(ua=None), dict(tss=-1), dict(trs=-1), dict(dss=-1), dict(drs=-1),
               dict(target=AT + 2), dict(draft=AT + 1), dict(dtype=M.BF16, target=AT + 1), dict(reward=AT)):
        assert probs_call(lib, **kw) == M.ERR_INVALID_ARGUMENT, kw
    for kw in (dict(dtype=2), dict(dtype=-1), dict(vocab=(1 << 30) + 1)):
        assert probs_call(lib, **kw) == M.ERR_UNSUPPORTED, kw


def cache_struct(**kw):
    a = dict(block_table=AT, held=AT, free_blocks=AT, free_count=AT, workspace=AT, status=None, n_pools=2, max_batch=8, max_blocks=4,
             n_blocks=30, page_size=8, device=0)
    assert set(kw) <= set(a)
    return M.MetasdCache(**dict(a, **kw))


BAD_CACHES = [dict(block_table=None), dict(held=None), dict(free_blocks=None), dict(free_count=None), dict(workspace=None),
              dict(workspace=AT + 8), dict(n_pools=0), dict(n_pools=33), dict(max_batch=0), dict(max_batch=65536), dict(max_blocks=0),
              dict(n_blocks=0), dict(page_size=0), dict(page_size=-1)]


def test_cache_calls_check_their_arguments(lib):
    def plan(cache, **kw):
        a = dict(batch=4, pool=None, cached=AT, stride=0, length=AT, max_tokens=16, order=None, place=None, pool_start=None,
                 token_start=AT, slot_map=AT, position=None, sequence=None, stream=None)
        assert set(kw) <= set(a)
        return lib.metasd_cache_plan(None if cache is None else C.byref(cache), *dict(a, **kw).values())

    def release(cache, batch=4, keep=AT, stride=0):
        return lib.metasd_cache_release(None if cache is None else C.byref(cache), batch, keep, stride, None)

    for kw in BAD_CACHES:
        assert plan(cache_struct(**kw)) == M.ERR_INVALID_ARGUMENT, kw
        assert release(cache_struct(**kw)) == M.ERR_INVALID_ARGUMENT, kw
    assert plan(None) == release(None) == M.ERR_INVALID_ARGUMENT
    good = cache_struct()
    for kw in (dict(batch=0), dict(batch=9), dict(cached=None), dict(length=None), dict(token_start=None), dict(slot_map=None),
               dict(max_tokens=0), dict(stride=-1)):
        assert plan(good, **kw) == M.ERR_INVALID_ARGUMENT, kw
    for kw in (dict(batch=0), dict(batch=9), dict(keep=None), dict(stride=-1)):
        assert release(good, **kw) == M.ERR_INVALID_ARGUMENT, kw
    for n, p in ((0, 1), (65536, 1), (1, 0), (1, 33), (-1, -1)):
        assert lib.metasd_cache_workspace_bytes(n, p) == 0
    assert lib.metasd_cache_workspace_bytes(100, 3) >= 100 * 32 and lib.metasd_cache_workspace_bytes(1, 1) > 0


def test_the_cache_mirror_matches_the_header():
    assert C.sizeof(M.MetasdCache) == 6 * 8 + 6 * 4


def test_tensors_on_the_host_are_refused(lib):
    t = torch.zeros((2, 2, 8))
    with pytest.raises(ValueError):
        M.verify_probs(t, t[:, :1], torch.zeros((2, 1), dtype=torch.int32), torch.zeros((2, 1)), torch.zeros(2))
    i = torch.zeros((1, 2, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        M.BlockCache(i, i[:, :, 0], i[:, 0], i[:, 0, 0], 8)


def test_calls_convert_as_ctypes_does(lib):
    """The extension module's calls: the library's own answers, and NotImplemented for what it leaves to ctypes."""
    if M._call is None:
        pytest.skip("not built for this interpreter")
    t = torch.zeros(8, dtype=torch.int32)
    probs = [lib.verify_probs_at, None, 0, 0, 1, 8, M.FP32, t, 8, 8, t, 8, 8, None, t, None, t, t, 0, t, t, None, None, None, None]
    plan = [lib.cache_plan_at, None, 1, None, t, 0, t, 8, None, None, None, t, t, None, None, None]
    release = [lib.cache_release_at, None, 1, t, 0, None]
    for fn, args, tensors in ((M._call.verify_probs, probs, (7, 10, 14, 16, 17, 19, 20)), (M._call.cache_plan, plan, (4, 6, 11, 12)),
                              (M._call.cache_release, release, (3,))):
        assert fn(*args) == M.ERR_INVALID_ARGUMENT      # no sequences; no cache
        for at in tensors:
            with pytest.raises(AttributeError):
                fn(*(args[:at] + [12345] + args[at + 1:]))
        assert fn(*(args[:2] + [1.0] + args[3:])) is NotImplemented
        with pytest.raises(TypeError):
            fn(*args[:-1])


def test_tensors_are_checked_alike_with_and_without_the_extension_module(lib):
    """Type, shape, device (-1: the host) and contiguity, of every tensor that is not None; what is no tensor is an AttributeError."""
    t = torch.zeros((4, 3), dtype=torch.int32)
    for are in [M._are] + ([M._call.are] if M._call is not None else []):
        assert are(-1, torch.int32, (4, 3)) and are(-1, torch.int32, (4, 3), None, t, t.clone())
        assert are(-1, torch.int32, (0,), torch.zeros(0, dtype=torch.int32)) and are(-1, torch.int32, (3,), t[1])
        for bad in (t.long(), t[:, :2], t[0], t.t(), t.t().contiguous(), torch.zeros((4, 6), dtype=torch.int32)[:, ::2], t.float()):
            assert not are(-1, torch.int32, (4, 3), t, bad)
        assert not are(0, torch.int32, (4, 3), t)       # on another device
        with pytest.raises(AttributeError):
            are(-1, torch.int32, (4, 3), t, 12345)
    with pytest.raises(ValueError, match="keep: a contiguous torch.int32 tensor of shape .4, 3. on cuda:0 is due, not torch.int64"):
        M._expect("keep", t.long(), torch.int32, (4, 3), 0)
    with pytest.raises(ValueError, match="is due, not NoneType"):
        M._expect("keep", None, torch.int32, (4, 3), 0)


def test_reference_verification_by_hand():
    p = np.array([[[0.5, 0.25, 0.25], [0.0, 1.0, 0.0]]])
    q = np.array([[[0.25, 0.75, 0.0]]])
    x = np.array([[1]])
    for u, accepted in ((0.33, 1), (1 / 3 + 1e-9, 0)):      # p/q = 1/3
        a, token, d, _ = R.verify(p, q, x, np.array([[u]]), np.array([0.4]))
        # rejected: (0.25, 0, 0.25) is left, 0.4 of it lies in its first half
        assert a[0] == accepted and token[0] == (1 if accepted else 0) and d[0, 0] == 0.5
    assert R.verify(p, q, x, np.array([[0.9]]), np.array([0.5]))[1][0] == 2       # strictly above half
    a, token, d, _ = R.verify(p, None, x, np.array([[0.9]]), np.array([0.9]))      # certain of token 1
    assert a[0] == 0 and token[0] == 2 and d[0, 0] == 0.75


def test_reference_caches_by_hand():
    c = Caches(2, 3, 4, 4, [[10, 11, 12], [20, 21]])
    order, place, start, tokens, entries = c.plan([5, 1, 2], [[0] * 3] * 2, [1, 0, 1])
    assert (order, place, start, tokens) == ([1, 0, 2], [1, 0, 2], [0, 1, 3], [0, 1, 6, 8])
    # pool 0 gives block 12; pool 1 gives 21 and 20 to sequence 0 and has none left for sequence 2
    assert [e[0] for e in entries] == [48, 84, 85, 86, 87, 80, -1, -1]
    c.release([[0, 1, 0], [4, 0, 0]])
    assert c.free == [[10, 11], [20]] and c.table[1][0] == [21]


@pytest.mark.parametrize("seed", range(3))
def test_serving_bookkeeping_where_pools_run_out(seed):
    """The serving loop's lengths over plans by the plain walk: caches never count entries that had no slots, so that every plan has the entries
    that its sequences lack."""
    rng = np.random.default_rng(seed)
    N, B, k, page, longest, blocks = 3, 12, 4, 4, 60, 60
    refs = [Caches(n, B, (longest + 2 * k) // page + 1, page, [list(range(blocks))] * n) for n in (N, 1)]

    def ints(x):
        return torch.as_tensor(np.asarray(x), dtype=torch.int32)

    def prompts():
        return ints(rng.integers(8, longest // 2, B))

    length, in_drafters, in_target = prompts(), torch.zeros((N, B), dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    went_without = 0
    for t in range(40):
        arm, accepted = ints(rng.integers(0, N, B)), ints(rng.integers(0, k + 1, B))
        goal_d, goal_t = length + (k - 1), length + k
        plans = []
        for ref, goal, cached, pool in ((refs[0], goal_d, in_drafters, arm), (refs[1], goal_t, in_target[None], torch.zeros_like(arm))):
            order, place, _, start, entries = ref.plan(goal.tolist(), cached.tolist(), pool.tolist())
            place, start = torch.tensor(place), torch.tensor(start)
            assert torch.equal(start[place + 1] - start[place], (goal - cached[pool.long(), torch.arange(B)]).long())
            plans.append(SimpleNamespace(place=place, token_start=start, slot_map=torch.tensor([e[0] for e in entries])))
            served = study.has_slots(plans[-1])
            assert [len(ref.table[g][b]) * page >= goal[b] for b, g in enumerate(pool.tolist())] == served.tolist()
            went_without += int((~served).sum())
        before = in_target
        in_drafters, in_target, after = study.advance(*plans, arm, length, accepted, goal_d, in_drafters, in_target)
        assert torch.equal(after, length + accepted + 1) and torch.equal(in_target, torch.where(served, length + accepted, before))
        done = after >= longest
        length = torch.where(done, prompts(), after)
        in_target, in_drafters = torch.where(done, 0, in_target), torch.where(done, 0, in_drafters)
        refs[0].release(in_drafters.tolist())
        refs[1].release(in_target[None].tolist())
    assert went_without > 0


@pytest.mark.parametrize("seed", range(8))
def test_measured_plain_plans_where_pools_run_out(seed):
    """The plain form that the measured plans are compared with, against the plain walk: nobody behind a sequence that goes without gets blocks,
    needs none in between or not."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("measured_operators", path)
    operators = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(operators)
    rng = np.random.default_rng(seed)
    P, B, page, most, n_blocks = 2, 14, 4, 8, 100
    cached = rng.integers(0, 3 * page, (P, B))
    length = cached.max(0) + rng.choice([1, 1, 2, 9], B)
    pool = rng.integers(-1, P, B)
    pool[2:4], length[2:4] = [0, 1], most * page      # these need four blocks at least, of three and two
    held = -(-cached // page)
    held += rng.integers(0, 2, (P, B))      # some have a block to spare: they need none
    ref = Caches(P, B, most, page, [list(range(3 - g)) for g in range(P)])
    table = np.full((P, B, most), -1)
    for g in range(P):
        for b in range(B):
            ref.table[g][b] = rng.integers(50, 90, held[g, b]).tolist()
            table[g, b, :held[g, b]] = ref.table[g][b]
    free = np.full((P, n_blocks), -1)
    for g in range(P):
        free[g, :len(ref.free[g])] = ref.free[g]

    def ints(x):
        return torch.as_tensor(np.asarray(x), dtype=torch.int32)

    s = dict(table=ints(table), held=ints(held), free=ints(free), count=ints([len(f) for f in ref.free]), cached=ints(cached), length=ints(length),
             pool=ints(pool), page=page, room=400)
    got = operators._plain_plan(s)
    want = ref.plan(length, cached, pool)
    entries = want[4]
    assert [g.tolist() for g in got[:4]] == [list(w) for w in want[:4]]
    for i in range(3):
        assert got[4 + i][:len(entries)].tolist() == [e[i] for e in entries] and not got[4 + i][len(entries):].any()
    assert any(e[0] == -1 for e in entries) and any(e[0] >= 0 for e in entries)
    for g in range(P):
        assert s["count"][g] == len(ref.free[g]) and [len(t) for t in ref.table[g]] == s["held"][g].tolist()
