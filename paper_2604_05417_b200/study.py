"""Synthetic counterpart of the paper's reward study: block divergence (BD) against block efficiency (BE).

The paper compares its two alignment rewards on real drafters: their means and variances, how often BE is exactly
zero, and how quickly a bandit fed with either reward settles on the best drafter (Sec. 2.3: the BE definition and
the lemma that relates E[r^BE] to E[r^BD]; Theorem 1's feedback signal; the reward-statistics table; the best-arm-ratio
figure).  This module
produces the same quantities for the synthetic workloads, whose generator knows which drafter is best for every
sequence in every round.  Every round runs through the library (C ABI, CUDA kernels); what is computed here is
bookkeeping on its outputs: means, variances, counts.

    python -m paper_2604_05417_b200.study --workload cfg2_nonstationary --rounds 300 [--bandits ucb,ducb] [--serve 100]

prints one JSON object and a table.  With --serve it also runs rounds as a serving loop does, from probabilities that are cut (min-p) and random
numbers of its own, with the paged caches of the target and of every drafter: how many entries the drafters' caches
have to catch up with when the bandit moves (the paper's switching cost), and how many blocks the caches hold.
"""
from __future__ import annotations

import argparse
import json
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

from . import binding as M
from .workloads import WORKLOADS, RoundGenerator, Workload


class RunningMoments:
    """Mean and (population) variance of a stream of arrays."""

    def __init__(self):
        self.n, self.s1, self.s2 = 0, 0.0, 0.0

    def add(self, x):
        x = np.asarray(x, dtype=np.float64)
        self.n += x.size
        self.s1 += float(x.sum())
        self.s2 += float((x * x).sum())

    @property
    def mean(self):
        return self.s1 / self.n if self.n else float("nan")

    @property
    def var(self):
        return max(self.s2 / self.n - self.mean ** 2, 0.0) if self.n else float("nan")


def both_rewards(res: M.VerifyResult, k: int):
    """(r_BD, r_BE) per sequence from one round's outputs: BD = 1 - mean_j d_TV (from the per-position diagnostics),
    BE = N_acc / k."""
    D = res.diag_fields()[2].cpu().numpy().astype(np.float64)
    return 1.0 - D.mean(axis=1), res.accepted_len.cpu().numpy().astype(np.float64) / k


def drafter_reward_statistics(wl: Workload, rounds: int, device=0, seed: int = 0, lib_seed: int = 99) -> List[dict]:
    """Plays every drafter in turn for `rounds` rounds on all sequences (no bandit: the rows are gathered for a
    fixed drafter index) and returns, per NOISE LEVEL of the drafter (the generator's alignment knob; which drafter
    has which level differs between sequences and over time): mean and variance of BD and BE, the share of rounds
    with BE = 0, the mean accepted length and the block efficiency 1 + E[N_acc]."""
    dev = torch.device("cuda", device)
    gen = RoundGenerator(wl, device=dev, seed=seed)
    acc: Dict[float, dict] = {}
    for i in range(wl.N):
        msd = M.MetaSD(wl.B, 1, wl.k, wl.V, dtype=wl.dtype, bandit="ucb", device=device)
        for t in range(rounds):
            rd = gen.gathered_round(t, np.full(wl.B, i))
            res = msd.verify(rd["target"], rd["draft"], rd["tokens"], wl.temperature, lib_seed, want_diag=True)
            r_bd, r_be = both_rewards(res, wl.k)
            level = np.round(np.asarray(rd["sigma"], dtype=np.float64), 3)
            for value in np.unique(level):
                pick = level == value
                a = acc.setdefault(float(value), dict(bd=RunningMoments(), be=RunningMoments(), zero=0))
                a["bd"].add(r_bd[pick])
                a["be"].add(r_be[pick])
                a["zero"] += int((r_be[pick] == 0).sum())
        msd.close()
    rows = []
    for value in sorted(acc):
        bd, be = acc[value]["bd"], acc[value]["be"]
        rows.append(dict(sigma=value, samples=be.n, mean_bd=bd.mean, var_bd=bd.var, mean_be=be.mean, var_be=be.var,
                         be_zero_ratio=acc[value]["zero"] / be.n, mean_accepted=be.mean * wl.k,
                         block_efficiency=1.0 + be.mean * wl.k))
    return add_feedback_signal(rows)


def feedback_signal(mean_best: float, var_best: float, mean_i: float, var_i: float) -> float:
    """The bandit feedback signal of a suboptimal drafter i under one reward design (the equation of Theorem 1):
    R = Delta_i^2 / max(Var[r_i], Var[r_best]) with Delta_i = mu_best - mu_i.  Infinite when neither reward varies."""
    gap, spread = mean_best - mean_i, max(var_i, var_best)
    if spread > 0.0:
        return gap * gap / spread
    return float("inf") if gap != 0.0 else float("nan")


def add_feedback_signal(rows: List[dict]) -> List[dict]:
    """Adds `signal_bd` and `signal_be` to the rows of drafter_reward_statistics: the feedback signal of every
    drafter against the best one, which is the row with the smallest noise level (the generator's best drafter;
    its own signal is NaN)."""
    best = min(rows, key=lambda r: r["sigma"])
    for r in rows:
        if r is best:
            r["signal_bd"] = r["signal_be"] = float("nan")
        else:
            r["signal_bd"] = feedback_signal(best["mean_bd"], best["var_bd"], r["mean_bd"], r["var_bd"])
            r["signal_be"] = feedback_signal(best["mean_be"], best["var_be"], r["mean_be"], r["var_be"])
    return rows


def bandit_run(wl: Workload, rounds: int, reward: int, bandit: str, device=0, seed: int = 0, lib_seed: int = 99,
               window: int = 25) -> dict:
    """`rounds` rounds of the workload with the bandit choosing the drafter (pointer-table mode) and `reward`
    (M.REWARD_BD or M.REWARD_BE) fed back.  Returns the best-arm ratio per round (share of sequences that played the
    drafter with the smallest noise level that round) and per window of rounds, the arm histogram, means and
    variances of both rewards, the BE zero ratio and the block efficiency 1 + E[N_acc]."""
    dev = torch.device("cuda", device)
    gen = RoundGenerator(wl, device=dev, seed=seed)
    msd = M.MetaSD(wl.B, wl.N, wl.k, wl.V, dtype=wl.dtype, bandit=bandit, beta=wl.beta, gamma=wl.gamma, window=wl.tau,
                   reward=reward, device=device)
    ratio = np.zeros(rounds)
    hist = np.zeros(wl.N, dtype=np.int64)
    bd, be, zero, acc = RunningMoments(), RunningMoments(), 0, RunningMoments()
    for t in range(rounds):
        arm = msd.select().cpu().numpy()
        rd = gen.table_round(t)
        table = M.pointer_table(rd["drafts"])
        res = msd.verify(rd["target"], None, rd["tokens"], wl.temperature, lib_seed, drafter_table=table,
                         token_arm_stride=wl.B * wl.k, want_diag=True)
        r_bd, r_be = both_rewards(res, wl.k)
        bd.add(r_bd)
        be.add(r_be)
        zero += int((r_be == 0).sum())
        acc.add(res.accepted_len.cpu().numpy())
        ratio[t] = float((arm == gen.best_arm(t)).mean())
        hist += np.bincount(arm, minlength=wl.N)
    status = msd.last_status()
    msd.close()
    n_win = (rounds + window - 1) // window
    return dict(workload=wl.name, bandit=bandit, reward="BD" if reward == M.REWARD_BD else "BE", rounds=rounds,
                best_arm_ratio=float(ratio.mean()),
                best_arm_ratio_by_window=[float(ratio[w * window:(w + 1) * window].mean()) for w in range(n_win)],
                window=window, arm_histogram=hist.tolist(), mean_bd=bd.mean, var_bd=bd.var, mean_be=be.mean,
                var_be=be.var, be_zero_ratio=zero / be.n, block_efficiency=1.0 + acc.mean, status=status)


def cut_probabilities(logits: torch.Tensor, temperature: float, min_p: float) -> torch.Tensor:
    """softmax(logits / T) in fp32 without the entries below min_p times the row's largest (min-p sampling)."""
    p = torch.softmax(logits.float() / temperature, dim=-1)
    if min_p > 0.0:
        p = torch.where(p < min_p * p.amax(dim=-1, keepdim=True), 0.0, p)
        p /= p.sum(dim=-1, keepdim=True)
    return p


def has_slots(plan: M.CachePlan) -> torch.Tensor:
    """[B]: whether the plan has slots for the entries that a sequence adds (one at least); its pool may have had too few blocks."""
    return plan.slot_map[plan.token_start[plan.place.long()].long()] >= 0


def advance(plan_d: M.CachePlan, plan_t: M.CachePlan, arm: torch.Tensor, length: torch.Tensor, accepted: torch.Tensor, goal_d: torch.Tensor,
            in_drafters: torch.Tensor, in_target: torch.Tensor):
    """What is cached behind a round, and the sequences' lengths: in_drafters [N, B], in_target [B], length [B].  A cache whose plan had no
    slots for a sequence holds what it held: the round's entries were not kept, and the next plan has them again."""
    at, played = torch.arange(length.shape[0], device=length.device), arm.long()
    stays = length + accepted           # the accepted drafts; the token behind them has been through no model
    had = in_drafters[played, at]
    in_drafters = in_drafters.clone()
    in_drafters[played, at] = torch.where(has_slots(plan_d), torch.maximum(had, torch.minimum(goal_d, stays)), had)
    return in_drafters, torch.where(has_slots(plan_t), stays, in_target), stays + 1


def serving_rounds(wl: Workload, rounds: int, bandit: str, device=0, seed: int = 0, min_p: float = 0.02, page: int = 16, longest: int = 400,
                   pool_blocks: Optional[int] = None):
    """The serving loop of Algorithm 1 around the library: per round the drafters are selected, the drafters' and the target's caches are
    planned, the round is verified from cut probabilities and given random numbers (the drafters' rows in the order in which the
    drafters hold them), and what was rejected or finished is given back.  Yields a dict per round; its tensors are the
    loop's own and change with the next one.

    Of a sequence with `length` tokens the target's cache holds all but the last.  A drafter that is chosen brings its own cache up to
    date and adds its drafts but the last; of these the accepted ones stay.  Where a pool has too few blocks (pool_blocks) for a sequence, the
    round's entries of its cache are not kept and are planned again with the next round's.  A query ends at `longest` tokens: its bandit starts anew
    and a prompt of another length takes its place."""
    dev, i32 = torch.device("cuda", device), torch.int32
    B, N, k = wl.B, wl.N, wl.k
    T = wl.temperature if wl.temperature > 0 else 1.0
    gen = RoundGenerator(wl, device=dev, seed=seed)
    g = torch.Generator(device=dev).manual_seed(seed + 1)
    most = (longest + 2 * k) // page + 1
    blocks = B * most if pool_blocks is None else pool_blocks
    msd = M.MetaSD(B, N, k, wl.V, dtype=wl.dtype, bandit=bandit, beta=wl.beta, gamma=wl.gamma, window=wl.tau, device=device)
    drafters = M.BlockCache.empty(N, B, most, blocks, page, device)
    target = M.BlockCache.empty(1, B, most, blocks, page, device)

    def prompts():
        return torch.randint(8, longest // 2, (B,), generator=g, device=dev).to(i32)

    length, at = prompts(), torch.arange(B, device=dev)
    in_target, in_drafters = torch.zeros(B, dtype=i32, device=dev), torch.zeros((N, B), dtype=i32, device=dev)
    room = B * (longest + 2 * k)
    try:
        for t in range(rounds):
            arm = msd.select()
            goal_d, goal_t = length + (k - 1), length + k
            plan_d = drafters.plan(goal_d, in_drafters, pool=arm, max_tokens=room)
            plan_t = target.plan(goal_t, in_target, max_tokens=room)
            rd = gen.gathered_round(t, arm.cpu().numpy())
            p, q = cut_probabilities(rd["target"], T, min_p), cut_probabilities(rd["draft"], T, min_p)
            tokens = torch.multinomial(q.reshape(B * k, wl.V), 1, generator=g).reshape(B, k).to(i32)
            held = torch.empty_like(q)
            held[plan_d.place.long()] = q
            u, v = torch.rand((B, k), generator=g, device=dev), torch.rand(B, generator=g, device=dev)
            res = msd.verify_probs(p, held, tokens, u, v, seed=seed, draft_place=plan_d.place, want_d_tv=True)
            yield dict(t=t, arm=arm, length=length, in_drafters=in_drafters, in_target=in_target, goal_d=goal_d, goal_t=goal_t, plan_d=plan_d,
                       plan_t=plan_t, target=p, draft=q, tokens=tokens, u_accept=u, u_draw=v, result=res, msd=msd, drafters=drafters,
                       target_cache=target, best_arm=gen.best_arm(t))
            in_drafters, in_target, length = advance(plan_d, plan_t, arm, length, res.accepted_len, goal_d, in_drafters, in_target)
            done = length >= longest
            length = torch.where(done, prompts(), length)
            in_target = torch.where(done, 0, in_target)
            in_drafters = torch.where(done, 0, in_drafters)
            target.release(in_target)
            drafters.release(in_drafters)
            msd.reset(torch.where(done, at, -1).to(i32))      # ids outside the batch are passed over
    finally:
        msd.close()


def serving_run(wl: Workload, rounds: int, bandit: str, **options) -> dict:
    """serving_rounds, summed up: entries that the drafters' and the target's caches add per sequence and round (k - 1 drafts
    and k + 1 tokens if nobody fell behind and all was accepted), the share of sequences and rounds whose drafter
    had more than k + 1 tokens to catch up with (the first use of every drafter on a query, by its prompt, is among them; a drafter that missed one
    short round is not), blocks held per sequence, the best-arm ratio and the block efficiency."""
    entries_d = entries_t = behind = held = acc = best = 0.0
    status = 0
    for r in serving_rounds(wl, rounds, bandit, **options):
        played = r["in_drafters"][r["arm"].long(), torch.arange(wl.B, device=r["arm"].device)]
        behind += float((r["length"] - played > wl.k + 1).float().mean())
        entries_d += float(r["plan_d"].token_start[-1]) / wl.B
        entries_t += float(r["plan_t"].token_start[-1]) / wl.B
        held += float(r["drafters"].held.sum() + r["target_cache"].held.sum()) / wl.B
        acc += float(r["result"].accepted_len.float().mean())
        best += float((r["arm"].cpu().numpy() == r["best_arm"]).mean())
        status |= r["msd"].last_status() | r["drafters"].last_status() | r["target_cache"].last_status()
    return dict(workload=wl.name, bandit=bandit, rounds=rounds, drafter_entries=entries_d / rounds, target_entries=entries_t / rounds,
                behind_ratio=behind / rounds, blocks_held=held / rounds, best_arm_ratio=best / rounds,
                block_efficiency=1.0 + acc / rounds, status=status)


def constant_alignment_rows(B: int, k: int, V: int, alphas, dtype=torch.float32, device="cuda", seed: int = 0):
    """Rows with a prescribed alignment 1 - d_TV(p_j, q_j) = alphas[b, j]: the drafter puts all its mass on one
    token x (which is therefore the drafted token), the target gives x the probability alpha and a second token the
    rest, so the accept test passes with probability alpha, independently per position (the paper's Assumption 1).
    Returns target [B, k+1, V], draft [B, k, V], tokens [B, k]."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    alphas = torch.as_tensor(np.asarray(alphas, dtype=np.float64)).reshape(B, k)
    x = torch.randint(0, V, (B, k), generator=g)
    y = (x + 1 + torch.randint(0, V - 1, (B, k), generator=g)) % V           # a second token, different from x
    neg = -1.0e4                                                              # probability exactly 0 after the softmax
    target = torch.full((B, k + 1, V), neg, dtype=torch.float64)
    draft = torch.full((B, k, V), neg, dtype=torch.float64)
    bi, ji = torch.meshgrid(torch.arange(B), torch.arange(k), indexing="ij")
    tiny = 1e-300
    target[bi, ji, x] = torch.log(alphas.clamp_min(tiny))
    target[bi, ji, y] = torch.log((1.0 - alphas).clamp_min(tiny))
    target[:, k, 0] = 0.0                                                     # the bonus row: any distribution
    draft[bi, ji, x] = 0.0
    return (target.to(dtype).to(device), draft.to(dtype).to(device), x.to(torch.int32).to(device))


def format_table(rows: Sequence[Dict], columns: Sequence[str]) -> str:
    out = ["| " + " | ".join(columns) + " |", "|" + "---|" * len(columns)]
    for r in rows:
        out.append("| " + " | ".join(("%.4f" % r[c]) if isinstance(r[c], float) else str(r[c]) for c in columns) + " |")
    return "\n".join(out)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="cfg2_nonstationary", choices=sorted(WORKLOADS))
    ap.add_argument("--rounds", type=int, default=300)
    ap.add_argument("--batch", type=int, default=0)
    ap.add_argument("--bandits", default="ucb,ducb")
    ap.add_argument("--window", type=int, default=25)
    ap.add_argument("--drafter-rounds", type=int, default=10, help="rounds per drafter of the reward-statistics table")
    ap.add_argument("--serve", type=int, default=0, help="rounds of the serving loop with paged caches, per bandit")
    args = ap.parse_args()
    wl = WORKLOADS[args.workload]
    if args.batch:
        wl = wl.scaled(B=args.batch)
    report = {"workload": wl.name, "B": wl.B, "rounds": args.rounds}
    report["drafters"] = drafter_reward_statistics(wl, args.drafter_rounds)
    report["runs"] = [bandit_run(wl, args.rounds, reward, bandit, window=args.window)
                      for bandit in args.bandits.split(",") for reward in (M.REWARD_BD, M.REWARD_BE)]
    if args.serve:
        report["serving"] = [serving_run(wl, args.serve, bandit) for bandit in args.bandits.split(",")]
    print(json.dumps(report))
    print(format_table(report["drafters"], ["sigma", "samples", "mean_bd", "var_bd", "mean_be", "var_be", "be_zero_ratio",
                                            "block_efficiency", "signal_bd", "signal_be"]))
    print(format_table(report["runs"], ["bandit", "reward", "best_arm_ratio", "mean_bd", "var_bd", "mean_be", "var_be",
                                        "be_zero_ratio", "block_efficiency"]))
    if args.serve:
        print(format_table(report["serving"], ["bandit", "drafter_entries", "target_entries", "behind_ratio", "blocks_held", "best_arm_ratio",
                                               "block_efficiency"]))
    for r in report["runs"]:
        print("%s/%s best-arm ratio per %d rounds: %s" % (r["bandit"], r["reward"], r["window"],
                                                         " ".join("%.2f" % v for v in r["best_arm_ratio_by_window"])))


if __name__ == "__main__":
    main()
