"""metasd_verify_probs on the GPU against its definition in float64: whole numbers are equal, distances within the roundings of
their sums, and what no row should do to its neighbours."""
import numpy as np
import pytest
import torch

import _probs_reference as R
from paper_2604_05417_b200 import binding as M

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
# d_TV: one rounding of each difference, sums of non-negative fp32 numbers in chains of fewer than 32 additions, one rounding at
# the end: below 34 half steps of 2^-24, relative to the value
TV_RELATIVE = 34 * 2.0 ** -24


def rows(shape, seed, cut=0.0, spread=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    p = torch.softmax(spread * torch.randn(shape, generator=g, device=DEV), -1)
    if cut:
        p = torch.where(p < cut * p.amax(-1, keepdim=True), 0.0, p)
        p /= p.sum(-1, keepdim=True)
    return p


def inputs(B, k, V, dtype, seed=0, certain=False, cut=0.0, agree=0.5):
    """Target and draft rows that agree on `agree` of their mass, tokens that the drafter may have drawn, uniforms."""
    target = rows((B, k + 1, V), seed, cut)
    draft = agree * target[:, :k] + (1 - agree) * rows((B, k, V), seed + 1, cut)
    g = torch.Generator(device=DEV).manual_seed(seed + 2)
    tokens = torch.zeros((B, k), dtype=torch.int32, device=DEV)
    if k:
        source = target[:, :k] if certain else draft
        tokens = torch.multinomial(source.reshape(B * k, V), 1, generator=g).reshape(B, k).to(torch.int32)
    return dict(target=target.to(DTYPES[dtype]), draft=None if certain or k == 0 else draft.to(DTYPES[dtype]), tokens=tokens,
                u_accept=torch.rand((B, k), generator=g, device=DEV), u_draw=torch.rand(B, generator=g, device=DEV))


def host(x):
    return None if x is None else x.double().cpu().numpy()


def check(s, lengths=None, place=None, status=0, near=0):
    """Both forms of the call, with and without distances, against the definition."""
    ref = R.verify(host(s["target"]), host(s["draft"]), s["tokens"].cpu().numpy(), host(s["u_accept"]), host(s["u_draw"]),
                   None if lengths is None else lengths.cpu().numpy(), None if place is None else place.cpu().numpy())
    assert ref[3] <= near, "the inputs hold draws next to an edge: another seed is due"
    k = s["tokens"].shape[1]
    for tv in (False, True):
        word = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = M.ProbsResult(torch.full((len(s["u_draw"]),), -7, dtype=torch.int32, device=DEV),
                            torch.full((len(s["u_draw"]),), -7, dtype=torch.int32, device=DEV),
                            torch.full((len(s["u_draw"]), k), -7.0, device=DEV))
        M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], draft_len=lengths, draft_place=place,
                       want_d_tv=tv, out=out, status=word)
        assert np.array_equal(out.accepted_len.cpu().numpy(), ref[0])
        assert np.array_equal(out.next_token.cpu().numpy(), ref[1])
        d_tv = out.d_tv.cpu().numpy().astype(np.float64)
        given = ~np.isnan(ref[2])
        if tv:
            assert np.all(np.abs(d_tv - ref[2])[given] <= TV_RELATIVE * np.abs(ref[2][given]))
        assert np.all(d_tv[~given if tv else np.ones_like(given)] == -7.0)     # left as they were
        if status is not None:
            assert word.item() == status
    return ref


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 5, 7, 8, 9, 31, 63, 127, 129, 511, 512, 513, 1000, 1023, 1025, 4097, 16387])
def test_small_and_odd_vocabularies(V, dtype):
    s = inputs(6, 3, V, dtype, seed=V, agree=0.5)
    # rounded to bf16 a row need not sum to one, and p may be below q everywhere: the target's own row is then drawn from
    check(s, status=None)


@pytest.mark.parametrize("B,k,V,dtype,cut", [(1, 4, 32000, "fp32", 0.0), (3, 8, 152064, "bf16", 0.0), (2, 16, 131073, "fp32", 0.02),
                                             (40, 5, 50257, "fp32", 0.0), (40, 5, 50257, "bf16", 0.05), (300, 2, 32001, "bf16", 0.0),
                                             (1, 1, 262144, "fp32", 0.0), (2, 1, 262147, "bf16", 0.0)])
def test_serving_sizes(B, k, V, dtype, cut):
    check(inputs(B, k, V, dtype, seed=11 + B, cut=cut), status=None)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [8, 129, 32001])
def test_certain_drafters(V, dtype):
    check(inputs(9, 5, V, dtype, seed=V, certain=True), status=None)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,V", [(1, 5), (7, 32001), (260, 1024)])
def test_plain_draws_without_drafts(B, V, dtype):
    s = inputs(B, 0, V, dtype, seed=B)
    check(s, status=0)
    out = M.verify_probs(s["target"], None, None, None, s["u_draw"])
    assert (out.accepted_len == 0).all()


def test_ragged_lengths_and_rows_in_the_drafters_order():
    s = inputs(33, 6, 5003, "fp32", seed=5)
    g = torch.Generator().manual_seed(1)
    lengths = torch.randint(0, 7, (33,), generator=g).to(torch.int32).to(DEV)
    place = torch.randperm(33, generator=g).to(torch.int32).to(DEV)
    check(s, lengths, status=None)
    check(s, lengths, place, status=None)
    moved = torch.empty_like(s["draft"])
    moved[place.long()] = s["draft"]
    a = M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], draft_len=lengths, want_d_tv=True)
    b = M.verify_probs(s["target"], moved, s["tokens"], s["u_accept"], s["u_draw"], draft_len=lengths, draft_place=place, want_d_tv=True)
    assert torch.equal(a.accepted_len, b.accepted_len) and torch.equal(a.next_token, b.next_token) and torch.equal(a.d_tv, b.d_tv)
    # behind a sequence's rows nothing is read
    for t in (s["target"], s["draft"]):
        for i in range(33):
            t[i, int(lengths[i]) + (t is s["target"]):] = float("nan")
    c = M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], draft_len=lengths, want_d_tv=True)
    assert torch.equal(a.accepted_len, c.accepted_len) and torch.equal(a.next_token, c.next_token) and torch.equal(a.d_tv, c.d_tv)


def test_lengths_and_places_outside_their_range():
    s = inputs(6, 3, 257, "fp32", seed=8)
    lengths = torch.tensor([-4, 0, 1, 3, 4, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    check(s, lengths, status=M.STATUS_BAD_LENGTH)
    place = torch.tensor([0, -1, 6, 3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    check(s, None, place, status=M.STATUS_BAD_INDEX)
    # a sequence that drafted nothing needs no draft rows
    lengths = torch.tensor([3, 0, 0, 3, 0, 0], dtype=torch.int32, device=DEV)
    check(s, lengths, place, status=0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 2, 3, 5, 7])
def test_rows_of_any_stride_and_start(offset, dtype):
    B, k, V = 5, 3, 1537
    s = inputs(B, k, V, dtype, seed=3)
    want = check(s, status=None)
    plain = M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], want_d_tv=True)

    def spread(t, gap):
        wide = torch.full((B, t.shape[1] + 1, V + gap), float("nan"), dtype=t.dtype, device=DEV)
        view = wide.reshape(-1)[offset:offset + B * (t.shape[1] + 1) * (V + gap) - 16].as_strided(
            (B, t.shape[1], V), ((t.shape[1] + 1) * (V + gap), V + gap, 1))
        view.copy_(t)
        return view
    moved = dict(s, target=spread(s["target"], 18), draft=spread(s["draft"], 23))
    got = check(moved, status=None)
    assert all(np.array_equal(a, b, equal_nan=True) for a, b in zip(want[:3], got[:3]))
    again = M.verify_probs(moved["target"], moved["draft"], s["tokens"], s["u_accept"], s["u_draw"], want_d_tv=True)
    assert torch.equal(plain.d_tv, again.d_tv)      # bit for bit, wherever the rows start


def test_rows_that_all_sequences_share():
    s = inputs(1, 2, 3001, "fp32", seed=9)
    B = 50
    g = torch.Generator(device=DEV).manual_seed(4)
    shared = dict(target=s["target"].expand(B, 3, 3001), draft=s["draft"].expand(B, 2, 3001), tokens=s["tokens"].expand(B, 2).contiguous(),
                  u_accept=torch.rand((B, 2), generator=g, device=DEV), u_draw=torch.rand(B, generator=g, device=DEV))
    check(shared, status=None)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), -0.25, -1e-30])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_entries_that_are_no_probabilities(value, dtype):
    """They spoil the row that holds them and no other."""
    s = inputs(8, 3, 2051, dtype, seed=21)
    s["u_accept"][:] = torch.tensor([0.999999, 1e-6, 0.999999, 1e-6, 0.3, 0.3, 1e-6, 0.999999], device=DEV)[:, None]
    s["target"][0, 0, 17] = value
    s["target"][1, 3, 2050] = value
    s["draft"][2, 0, 1024] = value
    s["draft"][3, 1, 0] = value
    s["target"][4, 1, int(s["tokens"][4, 1])] = value      # the drafted token's own entry
    s["draft"][5, 0, int(s["tokens"][5, 0])] = value
    clean = inputs(8, 3, 2051, dtype, seed=21)
    clean["u_accept"] = s["u_accept"]
    got, want = check(s, status=None), check(clean, status=None)
    assert np.array_equal(got[0][6:], want[0][6:]) and np.array_equal(got[1][6:], want[1][6:])
    word = torch.zeros(1, dtype=torch.int32, device=DEV)
    M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], want_d_tv=True, status=word)
    assert word.item() & M.STATUS_NONFINITE


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_negative_zero_is_a_zero(dtype):
    s = inputs(4, 2, 1029, dtype, seed=2, cut=0.1)
    want = check(s, status=None)
    for t in (s["target"], s["draft"]):
        t.copy_(torch.where(t == 0, -0.0, t))
        assert torch.signbit(t).any()
    got = check(s, status=None)
    assert all(np.array_equal(a, b, equal_nan=True) for a, b in zip(want[:3], got[:3]))


def test_edges_of_the_draw():
    """Exact sums: a threshold on an edge belongs to the entry behind it; entries without mass are never drawn."""
    V = 16
    p = torch.zeros((6, 1, V), device=DEV)
    p[:, 0, 3], p[:, 0, 7], p[:, 0, 12] = 0.25, 0.5, 0.25
    u = torch.tensor([0.0, 0.25 - 2.0 ** -24, 0.25, 0.75 - 2.0 ** -24, 0.75, 1.0 - 2.0 ** -24], device=DEV)
    out = M.verify_probs(p, None, None, None, u)
    assert out.next_token.tolist() == [3, 3, 7, 7, 12, 12]
    out = M.verify_probs(p, None, None, None, torch.tensor([1.0, 2.0, float("nan"), -1.0, float("inf"), -float("inf")], device=DEV))
    assert out.next_token.tolist() == [12, 12, 12, 3, 12, 3]       # uniforms outside [0, 1): the last, or the first, with mass


def test_accept_test_is_strict_and_exact():
    V = 8
    p, q = torch.zeros((4, 2, V), device=DEV), torch.zeros((4, 1, V), device=DEV)
    p[:, 0, 2], p[:, 0, 5], p[:, 1, 1] = 0.25, 0.75, 1.0
    q[:, 0, 2], q[:, 0, 4] = 0.5, 0.5
    tokens = torch.full((4, 1), 2, dtype=torch.int32, device=DEV)
    u = torch.tensor([[0.5], [0.5 - 2.0 ** -25], [0.0], [0.75]], device=DEV)
    out = M.verify_probs(p, q, tokens, u, torch.full((4,), 0.1, device=DEV))
    assert out.accepted_len.tolist() == [0, 1, 1, 0]
    assert out.next_token.tolist() == [5, 1, 1, 5]


def test_tokens_outside_the_vocabulary_zero_rows_and_empty_residuals():
    V = 40
    s = inputs(7, 2, V, "fp32", seed=30)
    s["tokens"][0, 0], s["tokens"][1, 1], s["tokens"][2, 0] = -1, V, 2 ** 31 - 1
    s["u_accept"][1, 0] = 0.0
    s["target"][3] = 0.0
    s["draft"][4] = 1.0                      # above p everywhere: nothing is left, p itself is drawn from
    s["u_accept"][4] = 0.999
    s["draft"][5, 0] = 0.0                   # q(x) = 0 < p(x): accepted, flagged
    s["u_accept"][5] = 0.5
    ref = check(s, status=M.STATUS_TOKEN_OOR | M.STATUS_NONFINITE | M.STATUS_Q_ZERO)
    assert ref[1][3] == -1 and ref[0][4] == 0 and ref[0][5] >= 1 and ref[0][0] == 0 and ref[0][1] == 1
    s = inputs(5, 1, V, "bf16", seed=31, certain=True)
    s["tokens"][0], s["tokens"][1], s["tokens"][2] = -5, V, 2 ** 31 - 1
    s["target"][3, 0] = 0.0
    s["target"][3, 0, int(s["tokens"][3, 0])] = 0.5     # all its mass on the token that is rejected
    s["u_accept"][:] = 0.75
    ref = check(s, status=M.STATUS_TOKEN_OOR)
    assert ref[1][3] == int(s["tokens"][3, 0]) and (ref[2][:3] == 1).all()


def test_mass_at_every_place_is_found():
    """One entry holds all the mass, at each end of vectors, trips and parts."""
    V = 70001
    spots = [0, 1, 3, 4, 7, 8, 31, 127, 128, 255, 511, 512, 513, 1023, 1024, 2047, 2048, 4095, 4096, 35000, 65535, 65536, 69999, 70000]
    for dtype in ("fp32", "bf16"):
        p = torch.zeros((len(spots), 1, V), dtype=DTYPES[dtype], device=DEV)
        p[torch.arange(len(spots)), 0, torch.tensor(spots)] = 0.3
        for u in (0.0, 0.5, 1.0 - 2.0 ** -24):
            out = M.verify_probs(p, None, None, None, torch.full((len(spots),), u, device=DEV))
            assert out.next_token.tolist() == spots


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_parts_of_several_batches(dtype):
    """Vocabularies of which a part is read in several steps, and looked through in several."""
    V = 1200003
    check(inputs(2, 1, V, dtype, seed=70, cut=0.01), status=None)
    spots = [0, 511, 512, 5119, 5120, 5121, 10239, 10240, 20480, 600000, 1199999, 1200000, 1200002]
    p = torch.zeros((len(spots), 1, V), dtype=DTYPES[dtype], device=DEV)
    p[torch.arange(len(spots)), 0, torch.tensor(spots)] = 0.3
    out = M.verify_probs(p, None, None, None, torch.full((len(spots),), 0.7, device=DEV))
    assert out.next_token.tolist() == spots


def test_rows_beyond_32_bit_offsets():
    V, k = 4099, 2
    s = inputs(2, k, V, "bf16", seed=71)
    far = 2 ** 31 + 77
    def apart(t):
        wide = torch.zeros(far + t.shape[1] * V + 16, dtype=t.dtype, device=DEV)
        view = wide.as_strided((2, t.shape[1], V), (far, V, 1))
        view.copy_(t)
        return view
    check(dict(s, target=apart(s["target"]), draft=apart(s["draft"])), status=None)


def test_the_smallest_numbers():
    """Rows of subnormal numbers: what is left over of them is drawn from all the same."""
    V = 600
    s = inputs(6, 2, V, "fp32", seed=72)
    s["target"].mul_(2.0 ** -130)
    s["draft"].mul_(2.0 ** -130)
    assert float(s["target"].max()) < 2.0 ** -126
    ref = R.verify(host(s["target"]), host(s["draft"]), s["tokens"].cpu().numpy(), host(s["u_accept"]), host(s["u_draw"]))
    out = M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"])
    assert ref[3] == 0 and (ref[1] >= 0).all()
    assert np.array_equal(out.accepted_len.cpu().numpy(), ref[0]) and np.array_equal(out.next_token.cpu().numpy(), ref[1])


def test_calls_on_two_streams_at_once():
    """Stateless calls share nothing: two streams that run side by side give what each gives alone."""
    s = [inputs(64, 4, 32000, dtype, seed=80 + i) for i, dtype in enumerate(("fp32", "bf16"))]
    call = lambda x: M.verify_probs(x["target"], x["draft"], x["tokens"], x["u_accept"], x["u_draw"], want_d_tv=True)
    want = [call(x) for x in s]
    streams = [torch.cuda.Stream() for _ in s]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(call(s[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for out in got[i]:
            for name in ("accepted_len", "next_token", "d_tv"):
                assert torch.equal(getattr(out, name), getattr(want[i], name))


def test_a_contexts_round_captured_and_replayed():
    """Every replay is the context's next round."""
    B, K, k, V = 10, 4, 3, 2003
    ctx = [M.MetaSD(B, K, k, V, dtype="bf16", bandit="ducb") for _ in range(2)]
    s = inputs(B, k, V, "bf16", seed=90)
    args = (s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"])
    out, arm = ctx[0].verify_probs(*args), ctx[0].select()
    ctx[0].reset()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx[0].verify_probs(*args, out=out)
        ctx[0].select(out=arm)
    for t in range(7):
        more = inputs(B, k, V, "bf16", seed=91 + t)
        for name in s:
            s[name].copy_(more[name])
        graph.replay()
        want = ctx[1].verify_probs(*args)
        assert torch.equal(arm, ctx[1].select())
        for name in ("accepted_len", "next_token", "reward"):
            assert torch.equal(getattr(out, name), getattr(want, name))
    assert ctx[0].state_export() == ctx[1].state_export()
    for c in ctx:
        c.close()


@pytest.mark.parametrize("V,dtype", [(50257, "fp32"), (32000, "bf16")])
def test_results_do_not_depend_on_the_batch(V, dtype):
    """Alone, in a few and in many: the launch's shape changes, no bit of the results does."""
    s = inputs(400, 2, V, dtype, seed=50)
    whole = M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], want_d_tv=True)
    fast = M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"])
    assert torch.equal(whole.accepted_len, fast.accepted_len) and torch.equal(whole.next_token, fast.next_token)
    for n in (1, 2, 5, 17, 60, 151):
        for first in (0, 400 - n):
            part = {name: t[first:first + n].contiguous() for name, t in s.items()}
            for tv in (False, True):
                out = M.verify_probs(part["target"], part["draft"], part["tokens"], part["u_accept"], part["u_draw"], want_d_tv=tv)
                assert torch.equal(out.accepted_len, whole.accepted_len[first:first + n])
                assert torch.equal(out.next_token, whole.next_token[first:first + n])
                if tv:
                    assert torch.equal(out.d_tv, whole.d_tv[first:first + n])


def test_captured_replayed_and_on_another_stream():
    s, other = inputs(20, 4, 9001, "fp32", seed=60), inputs(20, 4, 9001, "fp32", seed=61)
    want = [M.verify_probs(x["target"], x["draft"], x["tokens"], x["u_accept"], x["u_draw"], want_d_tv=True) for x in (s, other)]
    out = M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], want_d_tv=True)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        M.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], want_d_tv=True, out=out)
    for x, w in ((s, want[0]), (other, want[1])):
        for name in s:
            s[name].copy_(x[name])
        for t in (out.accepted_len, out.next_token, out.d_tv):
            t.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.accepted_len, w.accepted_len) and torch.equal(out.next_token, w.next_token) and torch.equal(out.d_tv, w.d_tv)


@pytest.mark.parametrize("bandit", ["ucb", "ducb", "swucb", "exp3", "rand", "petc"])
@pytest.mark.parametrize("reward", [M.REWARD_BD, M.REWARD_BE])
def test_rounds_of_a_context_feed_its_bandits(bandit, reward):
    """Against metasd_verify on the same rows: the distances, and with them the rewards and the bandits, are the same; the block
    efficiency is this round's own."""
    B, K, k, V = 12, 3, 4, 1531
    ctx = [M.MetaSD(B, K, k, V, dtype="fp32", bandit=bandit, reward=reward, window=6, gamma=0.3) for _ in range(2)]
    g = torch.Generator(device=DEV).manual_seed(7)
    lengths = torch.randint(1, k + 1, (B,), generator=g, device=DEV).to(torch.int32)
    for c in ctx:
        c.set_draft_lengths(lengths)
    for t in range(9):
        arms = [c.select() for c in ctx]
        if reward == M.REWARD_BD:
            assert torch.equal(*arms)
        logits = 2.0 * torch.randn((B, k + 1, V), generator=g, device=DEV)
        noise = 0.2 + 0.5 * arms[1].float()
        drafted = logits[:, :k] + noise[:, None, None] * torch.randn((B, k, V), generator=g, device=DEV)
        target, draft = torch.softmax(logits.double(), -1).float(), torch.softmax(drafted.double(), -1).float()
        tokens = torch.multinomial(draft.reshape(B * k, V), 1, generator=g).reshape(B, k).to(torch.int32)
        u, v = torch.rand((B, k), generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
        res = ctx[0].verify(logits, drafted, tokens, 1.0, 99)
        got = ctx[1].verify_probs(target, draft, tokens, u, v, seed=99, want_d_tv=t % 2 == 0)
        ref = R.verify(host(target), host(draft), tokens.cpu().numpy(), host(u), host(v), lengths.cpu().numpy())
        assert np.array_equal(got.accepted_len.cpu().numpy(), ref[0]) and np.array_equal(got.next_token.cpu().numpy(), ref[1])
        if reward == M.REWARD_BD:
            assert torch.allclose(got.reward, res.reward, rtol=0, atol=1e-5)
            want = 1.0 - np.nansum(ref[2], 1) / lengths.cpu().numpy()
            # the mean of up to four distances, each within TV_RELATIVE, and one rounding
            assert np.all(np.abs(got.reward.cpu().numpy() - want) <= TV_RELATIVE + 2.0 ** -24)
        else:
            assert np.allclose(got.reward.cpu().numpy(), ref[0] / lengths.cpu().numpy(), rtol=2.0 ** -23, atol=0)
    states = [M.parse_state(c.state_export(), B, K, 6) for c in ctx]
    assert np.array_equal(states[0]["t"], states[1]["t"]) and (states[1]["t"] == 9).all()
    if reward == M.REWARD_BD:
        np.testing.assert_allclose(states[1]["stat_a"], states[0]["stat_a"], rtol=0, atol=1e-5)
    assert ctx[1].last_status() == 0
    for c in ctx:
        c.close()


def test_refusals_on_the_device():
    s = inputs(4, 2, 100, "fp32")

    def call(**kw):
        a = dict(s, **kw)
        return M.verify_probs(a["target"], a["draft"], a["tokens"], a["u_accept"], a["u_draw"], draft_len=a.get("lengths"),
                              draft_place=a.get("place"), out=a.get("out"), status=a.get("status"))
    call()
    bad = dict(target=[s["target"].half(), s["target"].cpu(), s["target"][0], s["target"].transpose(1, 2), s["target"][..., ::2]],
               draft=[s["draft"].bfloat16(), s["draft"][:, :1], s["draft"].cpu(), s["draft"].transpose(0, 2)],
               tokens=[s["tokens"].long(), s["tokens"][:3], s["tokens"].t()], u_accept=[s["u_accept"].double(), s["u_accept"][:, :1]],
               u_draw=[s["u_draw"].double(), s["u_draw"][:3], s["u_draw"][:, None]], lengths=[s["tokens"][:, 0].long(), s["tokens"][:3, 0]],
               place=[s["tokens"][:, 0].float()], status=[torch.zeros(1, device=DEV)],
               out=[M.ProbsResult(s["tokens"][:, 0], s["u_draw"].int())])
    for name, values in bad.items():
        for value in values:
            with pytest.raises(ValueError):
                call(**{name: value})
    ctx = M.MetaSD(4, 2, 2, 100, dtype="fp32")
    with pytest.raises(M.MetasdError):
        ctx.verify_probs(s["target"][..., :99], s["draft"][..., :99], s["tokens"], s["u_accept"], s["u_draw"])   # another vocabulary
    with pytest.raises(M.MetasdError):
        ctx.verify_probs(s["target"][:, :1], None, None, None, s["u_draw"])                                      # no drafts to reward
    ctx.close()
    with pytest.raises(M.MetasdError):
        ctx.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"])


@pytest.mark.parametrize("sign", [1, -1])
def test_sums_of_very_long_rows(sign):
    """Half of the mass ends 2^-32 in front of the end of an entry, or behind it, in a row of 2^24 entries that starts with a large one
    among small ones: all are multiples of 2^-39 and add up to less than 8, so that sums in fp64 are exact."""
    V, delta = 1 << 24, sign * 2.0 ** -32
    w = np.full(V, 2.0 ** -22)
    w[:104960] = 2.0 ** -24 - 2.0 ** -39
    w[0] = 1.0
    upto = np.cumsum(w[:-1])
    m = int(np.searchsorted(upto, upto[-1] / 2)) + 2
    w[-1] = 2.0 * (upto[m] - delta) - upto[-1]
    assert 0.0 < w[-1] <= 2.0 ** -19 and float(np.float32(w[-1])) == w[-1]
    upto = np.cumsum(w)
    assert upto[m] - upto[-1] / 2 == delta
    row = torch.from_numpy(w.astype(np.float32)).to(DEV)
    u = torch.full((1,), 0.5, device=DEV)
    want = [m if sign > 0 else m + 1]
    assert M.verify_probs(row.view(1, 1, V), None, None, None, u).next_token.tolist() == want
    # the same as what is left over of a row pair, token 3 rejected
    q = torch.where(torch.arange(V, device=DEV) % 3 == 0, 2.0 ** -20, 0.0)
    p = row + q
    assert torch.equal(p.double() - q.double(), row.double())
    tokens, u_accept = torch.full((1, 1), 3, dtype=torch.int32, device=DEV), torch.full((1, 1), 2.0, device=DEV)
    out = M.verify_probs(torch.stack([p, row]).view(1, 2, V), q.view(1, 1, V), tokens, u_accept, u)
    assert out.accepted_len.tolist() == [0] and out.next_token.tolist() == want


@pytest.mark.parametrize("places", [(0, 128), (5, 150000), (7, 199999)])
def test_sums_beyond_fp32_count_as_not_finite(places):
    """Wherever in the row the large entries lie: in one lane's sum, in one part's, or in different parts."""
    V, most = 200000, float(torch.finfo(torch.float32).max)
    p = torch.full((4, 2, V), 0.25, device=DEV)
    for b, (x, y) in enumerate([(2.0 ** 127, most - 2.0 ** 127), (2.0 ** 127, 2.0 ** 127), (most, most), (3e38, 1e36)]):
        p[b, 0] = 0.0
        p[b, 0, places[0]], p[b, 0, places[1]] = x, y
    u = torch.zeros(4, device=DEV)
    word = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = M.verify_probs(p[:, :1], None, None, None, u, status=word)
    assert out.next_token.tolist() == [places[0], -1, -1, places[0]] and word.item() == M.STATUS_NONFINITE
    # distances from a row of zeros
    tokens, u_accept = torch.full((4, 1), 1, dtype=torch.int32, device=DEV), torch.full((4, 1), 0.5, device=DEV)
    word.zero_()
    out = M.verify_probs(p, torch.zeros((4, 1, V), device=DEV), tokens, u_accept, u, want_d_tv=True, status=word)
    want = 0.5 * np.array([most, 2.0, 2.0, 3.01e38])
    assert np.all(np.abs(out.d_tv.cpu().numpy()[:, 0] - want) <= TV_RELATIVE * want)
    assert word.item() == M.STATUS_NONFINITE | M.STATUS_Q_ZERO


@pytest.mark.parametrize("bandit", ["ucb", "ducb", "swucb", "exp3", "petc"])
def test_rewards_of_rows_that_are_not_normalised(bandit):
    """Their distances may be above one; the rewards stay in [0, 1], the states finite."""
    B, K, k, V = 5, 2, 3, 300
    s = inputs(B, k, V, "fp32", seed=95)
    s["target"][1:] *= 1e5
    s["draft"][2:] *= 1e8
    ctx = M.MetaSD(B, K, k, V, dtype="fp32", bandit=bandit, window=6, gamma=0.3)
    for _ in range(8):
        out = ctx.verify_probs(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_draw"], want_d_tv=True)
        d_tv = host(out.d_tv)
        assert (d_tv[0] < 1).all() and (d_tv[1:] > 1e4).all()
        want = 1.0 - np.minimum(d_tv, 1.0).mean(1)
        assert np.all(np.abs(host(out.reward) - want) <= 2.0 ** -24) and not host(out.reward)[1:].any()
    blob = ctx.state_export()
    state = M.parse_state(blob, B, K, 6)
    assert np.isfinite(state["stat_a"]).all() and np.isfinite(state["win_reward"]).all()
    ctx.state_import(blob)
    ctx.close()
