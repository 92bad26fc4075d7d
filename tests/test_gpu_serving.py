"""Selection, cache plans, verification from probabilities, reward, bandits and releases as a serving loop runs them, round after
round, against the plain walks over the same numbers."""
import numpy as np
import pytest
import torch

import _probs_reference as R
from _cache_reference import Caches
from paper_2604_05417_b200 import binding as M
from paper_2604_05417_b200 import study
from paper_2604_05417_b200.workloads import Workload

pytestmark = pytest.mark.gpu


def workload(**kw):
    return Workload(**dict(dict(name="serving", B=23, N=4, k=4, V=1009, rounds=60, temperature=0.8, dtype="fp32", bandit="ucb",
                                sigmas=(0.3, 0.8, 1.6, 3.0), schedule="permute", period=10), **kw))


def table_of(cache, ref):
    held, table = cache.held.cpu().numpy(), cache.block_table.cpu().numpy()
    free, count = cache.free_blocks.cpu().numpy(), cache.free_count.cpu().numpy()
    for g in range(ref.pools):
        assert free[g, :count[g]].tolist() == ref.free[g]
        for b in range(ref.batch):
            assert table[g, b, :held[g, b]].tolist() == ref.table[g][b]


@pytest.mark.parametrize("bandit,page,B", [("ucb", 16, 23), ("ducb", 5, 40), ("rand", 7, 3)])
def test_serving_loop_against_plain_walks(bandit, page, B):
    wl = workload(B=B, bandit=bandit)
    refs, last = None, None
    switched = finished = 0
    for r in study.serving_rounds(wl, 40, bandit, page=page, longest=60):
        n = {name: r[name].cpu().numpy().astype(np.int64) for name in ("arm", "length", "in_drafters", "in_target", "goal_d", "goal_t")}
        if refs is None:
            blocks = r["drafters"].free_blocks.shape[1]
            most = r["drafters"].block_table.shape[2]
            free = list(range(blocks - 1, -1, -1))
            refs = [Caches(wl.N, B, most, page, [free] * wl.N), Caches(1, B, most, page, [free])]
        else:       # what the loop gave back since the last round
            refs[0].release(n["in_drafters"])
            refs[1].release(n["in_target"][None])
            finished += int((n["in_target"] == 0).sum())
            switched += int((n["arm"] != last).sum())
        last = n["arm"]
        for ref, plan, goal, cached, pool, cache in ((refs[0], r["plan_d"], n["goal_d"], n["in_drafters"], n["arm"], r["drafters"]),
                                                     (refs[1], r["plan_t"], n["goal_t"], n["in_target"][None], None, r["target_cache"])):
            want = ref.plan(goal, cached, pool)
            assert plan.order.tolist() == want[0] and plan.place.tolist() == want[1]
            assert plan.pool_start.tolist() == want[2] and plan.token_start.tolist() == want[3]
            total = len(want[4])
            assert total > 0 and plan.slot_map[:total].tolist() == [e[0] for e in want[4]]
            assert plan.position[:total].tolist() == [e[1] for e in want[4]] and plan.sequence[:total].tolist() == [e[2] for e in want[4]]
            table_of(cache, ref)
        p, q, u, v = (r[name].double().cpu().numpy() for name in ("target", "draft", "u_accept", "u_draw"))
        accepted, token, d_tv, near = R.verify(p, q, r["tokens"].cpu().numpy(), u, v)
        assert near == 0
        assert np.array_equal(r["result"].accepted_len.cpu().numpy(), accepted)
        assert np.array_equal(r["result"].next_token.cpu().numpy(), token)
        # distances within 34 half steps of fp32 (each difference, chains of fewer than 32 additions, the result); of their mean one more rounding
        assert np.allclose(r["result"].d_tv.cpu().numpy(), d_tv, rtol=34 * 2.0 ** -24, atol=0)
        assert np.allclose(r["result"].reward.cpu().numpy(), 1.0 - d_tv.mean(axis=1), rtol=0, atol=35 * 2.0 ** -24)
        assert r["msd"].last_status() == r["drafters"].last_status() == r["target_cache"].last_status() == 0
    assert finished > 0 and switched > 0


def test_serving_run_of_the_study():
    res = study.serving_run(workload(B=16, dtype="bf16"), 30, "ducb", longest=80)
    assert res["status"] == 0 and 0.0 < res["best_arm_ratio"] <= 1.0 and 1.0 <= res["block_efficiency"] <= 5.0
    assert res["drafter_entries"] > 0 and res["target_entries"] > 0 and res["blocks_held"] > 0


def test_serving_loop_that_runs_out_of_blocks():
    """Sequences that a pool has no blocks for are flagged and planned again when there is room; nothing is lost or given twice."""
    wl = workload(B=12)
    for r in study.serving_rounds(wl, 25, "ucb", page=4, longest=60, pool_blocks=60):
        for cache, goal in ((r["drafters"], r["goal_d"]), (r["target_cache"], r["goal_t"])):
            held, table = cache.held.cpu().numpy(), cache.block_table.cpu().numpy()
            free, count = cache.free_blocks.cpu().numpy(), cache.free_count.cpu().numpy()
            for g in range(table.shape[0]):
                ids = free[g, :count[g]].tolist() + [i for b in range(wl.B) for i in table[g, b, :held[g, b]]]
                assert sorted(ids) == list(range(60))
        if r["t"] == 0:
            assert r["target_cache"].last_status() == M.STATUS_NO_BLOCKS
            assert (r["plan_t"].slot_map[:int(r["plan_t"].token_start[-1])] == -1).any()


def test_sequences_without_blocks_are_planned_again():
    """What had no slots is not taken for cached: no cache holds more entries than its blocks have room for, every plan has the entries
    that its sequences lack, and sequences that went without get their slots in later rounds of the same query."""
    wl, page = workload(B=12), 4
    waiting, last = np.zeros(wl.B, bool), None
    went_without = got_them_later = 0
    for r in study.serving_rounds(wl, 25, "ucb", page=page, longest=60, pool_blocks=60):
        arm, at = r["arm"].cpu().numpy(), np.arange(wl.B)
        in_target = r["in_target"].cpu().numpy()
        if last is not None:        # the target's cache behind a round without slots: as it was, or the query ended
            assert np.all((in_target == last) | (in_target == 0) | ~waiting)
            waiting &= in_target == last
        for cache, plan, goal, cached in ((r["drafters"], r["plan_d"], r["goal_d"], r["in_drafters"]),
                                          (r["target_cache"], r["plan_t"], r["goal_t"], r["in_target"][None])):
            assert cache.last_status() in (0, M.STATUS_NO_BLOCKS)
            held, cached, goal = (x.cpu().numpy() for x in (cache.held, cached, goal))
            assert np.all(cached <= held * page)
            row = arm if len(held) > 1 else 0 * arm
            start, place = plan.token_start.cpu().numpy(), plan.place.cpu().numpy()
            assert np.array_equal(start[place + 1] - start[place], goal - cached[row, at])
            served = plan.slot_map.cpu().numpy()[start[place]] >= 0
            assert np.array_equal(served, held[row, at] * page >= goal)
        got_them_later += int((waiting & served).sum())     # of the target's cache
        went_without += int((~served).sum())
        waiting, last = ~served, in_target
    assert went_without > 0 and got_them_later > 0
