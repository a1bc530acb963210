"""GPU parity of sampling against the float64 oracle.

Tokens must be equal.  The two sides add the same float64 weights in other orders,
n of them, which moves a running sum by at most n 2^-53 of itself: the oracle's
margin (its distance from the nearest border) says where that could matter, and
no case here comes near (asserted: margin above 2^-53 V, except where the weights
are whole numbers and the sums exact).  logprob: float64, rounded once to float32:
half a step, 2^-24 |lp|, and the sums' 2^-53 n.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import pctree_sample as SO
from paper_2608_02123_amd import pctree as P

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def up(x, dt):
    return None if x is None else torch.from_numpy(np.asarray(x, dt)).cuda()


def check(logits, u, exact_sums=False, sampler=None, **par):
    """Runs rows of a device tensor against the oracle."""
    T, V = logits.shape
    kinds = dict(temperature=np.float32, top_k=np.int32, top_p=np.float32, min_p=np.float32)
    par = {n: None if v is None else np.broadcast_to(np.asarray(v, kinds[n]), (T,)).copy() for n, v in par.items()}
    u = np.asarray(u, np.float32)
    s = sampler or P.Sampler(T, V)
    s.workspace.fill_(0xA5)
    tok, lp = s(logits, up(u, np.float32), **{n: up(v, kinds[n]) for n, v in par.items()})
    torch.cuda.synchronize()
    x = logits.detach().cpu().double().numpy()
    want, wlp, margin = SO.sample(x, u.astype(np.float64), **par)
    if not exact_sums:
        assert margin.min() > V * 2.0 ** -53, "inputs on a border"
    tok, lp = tok.cpu().numpy(), lp.cpu().numpy().astype(np.float64)
    bad = np.nonzero(tok != want)[0]
    assert len(bad) == 0, [(int(t), int(tok[t]), int(want[t]), float(margin[t]),
                            {n: v[t] for n, v in par.items() if v is not None}) for t in bad[:5]]
    fin = np.isfinite(wlp)
    assert np.array_equal(fin, np.isfinite(lp))
    assert (np.abs(lp - wlp)[fin] <= 2.0 ** -24 * np.abs(wlp[fin]) + V * 2.0 ** -52).all()


def rows(seed, T, V, dt, sigma=2.0, head=10.0):
    """Logits with a bulk and a head that falls like a power of the rank."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, V, generator=g) * sigma
    n = min(64, V)
    for t in range(T):
        at = torch.randperm(V, generator=g)[:n]
        x[t, at] += (head - 1.3 * torch.log(torch.arange(1, n + 1.0))).clamp_min(0)
    return x.to(DT[dt]).cuda()


FILTERS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=20), dict(top_k=50, top_p=0.9), dict(top_p=0.95),
           dict(top_p=0.5), dict(min_p=0.05), dict(min_p=0.3, top_k=5), dict(min_p=0.01, top_p=0.8, temperature=1.3),
           dict(top_k=400, top_p=0.99), dict(top_k=3000), dict(temperature=0.0)]


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("V", [1, 2, 7, 64, 513, 2047, 2048, 2049, 4099, 50021])
def test_filters(dt, V):
    T = 6
    x = rows(V, T, V, dt)
    u = np.random.default_rng(V).random(T)
    for f in FILTERS:
        print(f"[sample] {dt} V {V} {f}", flush=True)
        check(x, u, exact_sums=V <= 2, **f)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("V", [151936, 163841, 400003, 1 << 20])
def test_large_vocabularies(dt, V):
    T = 3
    x = rows(V, T, V, dt)
    u = np.random.default_rng(V).random(T)
    for f in FILTERS:
        print(f"[sample] {dt} V {V} {f}", flush=True)
        check(x, u, **f)


@pytest.mark.parametrize("dt", list(DT))
def test_each_row_has_its_own_parameters(dt):
    rng = np.random.default_rng(1)
    T, V = 96, 6007
    x = rows(2, T, V, dt, head=12.0)
    par = dict(temperature=rng.choice([0.0, 0.5, 1.0, 1.5], T), top_k=rng.choice([0, -3, 1, 5, 50, 90, 500, 9000], T),
               top_p=rng.choice([1.0, 0.3, 0.9, 0.99, 2.0], T), min_p=rng.choice([0.0, -1.0, 0.02, 0.5], T))
    check(x, rng.random(T), **par)


@pytest.mark.parametrize("T", [2, 5])
def test_open_rows(T):
    """Rows whose kept set is large: nearly flat logits, top_p and large top_k; few rows
    are cut by one workgroup, more by launches of their own."""
    rng = np.random.default_rng(5)
    for dt, V, sigma in (("f32", 151936, 1.0), ("bf16", 151936, 0.3), ("f32", 151936, 1e-3), ("f32", 30000, 1e-6),
                         ("bf16", 151936, 1e-3), ("f16", 50000, 0.1)):
        x = rows(7, T, V, dt, sigma=sigma, head=0.0)
        for f in (dict(top_p=0.9), dict(top_p=0.5, temperature=2.0), dict(top_k=20000, top_p=0.7),
                  dict(top_k=V // 2), dict(min_p=0.9, top_p=0.6), dict()):
            print(f"[sample] open {dt} {V} {sigma} {f}", flush=True)
            check(x, rng.random(T), **f)


@pytest.mark.parametrize("T", [1, 3, 4])
def test_open_rows_beside_rows_of_a_top_k(T):
    """A top_k of zero in a call that has the others': few rows come without histograms."""
    rng = np.random.default_rng(T)
    for dt, V, sigma in (("bf16", 151936, 1.0), ("f32", 40001, 0.2)):
        x = rows(T, T, V, dt, sigma=sigma, head=0.0)
        for f in (dict(top_p=0.9), dict(min_p=0.05), dict(min_p=0.05, top_p=0.7)):
            for k in (np.zeros(T), np.arange(T) * 30, -np.ones(T)):
                print(f"[sample] {dt} {V} {f} {k}", flush=True)
                check(x, rng.random(T), top_k=k, **f)


def test_open_rows_in_two_rounds():
    T, V = 1100, 4000
    x = rows(8, T, V, "bf16", sigma=0.5, head=3.0)
    rng = np.random.default_rng(12)
    check(x, rng.random(T), top_p=rng.choice([0.9, 0.99, 1.0], T), min_p=rng.choice([0.0, 0.1], T))


@pytest.mark.parametrize("V", [100, 5000, 151936])
def test_equal_logits(V):
    """Ties go by token: the weights are whole numbers and the sums exact."""
    u = np.array([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24])
    T = len(u)
    flat = torch.full((T, V), 1.5, device="cuda")
    for f in (dict(), dict(top_k=10), dict(top_k=V // 2), dict(top_p=0.5), dict(top_p=0.25, top_k=V - 1),
              dict(min_p=1.0), dict(top_p=0.0), dict(temperature=0.0), dict(temperature=0.01, top_p=0.75)):
        check(flat, u, exact_sums=True, **f)
    # two levels, the upper one far above: only its ties share
    two = torch.full((T, V), -300.0, device="cuda")
    two[:, 3::7] = 500.0
    for f in (dict(), dict(top_k=5), dict(top_p=0.5), dict(min_p=0.1)):
        check(two, u, exact_sums=True, **f)


@pytest.mark.parametrize("low", [-float("inf"), torch.finfo(torch.float32).min, -1e30])
def test_masked_vocabularies(low):
    V, T = 151936, 5
    g = torch.Generator().manual_seed(3)
    x = torch.full((T, V), low)
    for t, n in enumerate((1, 3, 60, 300, 5000)):
        at = torch.randperm(V, generator=g)[:n]
        x[t, at] = torch.randn(n, generator=g)
    u = np.random.default_rng(0).random(T)
    for dt in ("f32", "bf16"):
        for f in FILTERS:
            check(x.to(DT[dt]).cuda(), u, exact_sums=True, **f)


def test_values_that_are_no_numbers():
    inf, nan = float("inf"), float("nan")
    V = 3000
    x = torch.randn(8, V, generator=torch.Generator().manual_seed(1))
    x[0] = -inf
    x[1] = nan
    x[2, ::3] = nan
    x[3, 17], x[3, 400] = inf, inf
    x[4, ::2] = -inf
    x[5] = -inf
    x[5, 77] = -3.0
    x[6] = inf
    x[7, 5] = inf
    u = [0.5, 0.5, 0.3, 0.7, 0.1, 0.9, 0.4, 0.4]
    for f in (dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=2500, top_p=0.9),
              dict(temperature=float("inf")), dict(temperature=0.0), dict(temperature=1e-30),
              dict(temperature=float("inf"), min_p=1.0, top_p=0.5)):
        for dt in DT:
            check(x.to(DT[dt]).cuda(), u, exact_sums=True, **f)


def test_uniforms_at_and_past_the_ends():
    V = 20000
    u = np.array([0.0, -0.5, float("nan"), 1.0, 2.0, float("inf"), 2.0 ** -24, 1 - 2.0 ** -24], np.float32)
    x = rows(9, len(u), V, "f32")
    for f in (dict(), dict(top_k=30), dict(top_p=0.9), dict(top_k=10000, top_p=0.95)):
        check(x, u, exact_sums=True, **f)


def _few_tokens(T, V, values, seed=1):
    """Rows of -inf but for a logit of 0 at token 5 and `values` at random later ones."""
    at = torch.randperm(V - 6, generator=torch.Generator().manual_seed(seed))[:len(values)] + 6
    x = torch.full((T, V), -float("inf"))
    x[:, 5] = 0.0
    x[:, at] = torch.tensor(values)
    return x.cuda()


@pytest.mark.parametrize("n", [40, 99, 1500])
def test_the_last_token_of_a_weight_that_rounding_loses(n):
    """A uniform of 1 takes the last kept token of positive weight, though e^-46 adds
    nothing to a running sum that holds 1, and not one of weight 0 behind it."""
    V = 5000
    u = np.array([1.0, 1.5, float("inf")], np.float32)
    zeros = [-46.0] * (n - n // 3) + [-800.0] * (n // 3)
    for f in (dict(top_k=n + 1), dict(top_k=n // 2), dict(top_k=3000), dict(min_p=1e-30), dict(),
              dict(top_k=n + 1, min_p=1e-30, temperature=0.9)):
        for values in ([-46.0] * n, zeros):
            print(f"[sample] {n} {f} {values[-1]}", flush=True)
            check(_few_tokens(len(u), V, values, n), u, exact_sums=True, **f)


@pytest.mark.parametrize("V,sigma", [(20000, 2.0), (151936, 0.5)])
def test_a_uniform_of_one_over_rounded_sums(V, sigma):
    """However a path adds the kept weights, none of its sums passes their total."""
    T = 24
    x = rows(V + 1, T, V, "f32", sigma=sigma, head=6.0)
    for f in (dict(), dict(top_k=20), dict(top_k=64), dict(top_k=100), dict(top_k=900), dict(top_k=3000),
              dict(top_p=0.9), dict(min_p=0.05), dict(min_p=0.01, top_p=0.7), dict(top_k=900, temperature=3.0)):
        print(f"[sample] {V} {f}", flush=True)
        check(x, np.ones(T, np.float32), exact_sums=True, **f)


def test_parameters_that_are_no_numbers():
    nan = float("nan")
    x = rows(10, 4, 5000, "bf16")
    u = [0.2, 0.4, 0.6, 0.8]
    s = P.Sampler(4, 5000)
    a = s(x, up(u, np.float32), temperature=up([nan] * 4, np.float32))[0]
    assert torch.equal(a.long(), x.float().argmax(1))
    b = s(x, up(u, np.float32), top_p=up([nan] * 4, np.float32), min_p=up([nan] * 4, np.float32))[0]
    assert torch.equal(b, s(x, up(u, np.float32))[0])


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("off,gap", [(0, 3), (1, 0), (5, 8), (3, 1)])
def test_rows_at_any_alignment(dt, off, gap):
    T, V = 5, 4001
    store = torch.full((off + T * (V + gap) + 8,), float("inf"), dtype=DT[dt], device="cuda")
    view = store[off:off + T * (V + gap)].unflatten(0, (T, V + gap))[:, :V]
    view.copy_(rows(11, T, V, dt))
    u = np.random.default_rng(off).random(T)
    for f in FILTERS:
        check(view, u, **f)


def test_more_rows_than_one_round():
    """Calls of more rows than the workspace holds go round by round."""
    T, V = 2100, 2500
    x = rows(15, T, V, "bf16", sigma=1.0, head=4.0)
    rng = np.random.default_rng(4)
    check(x, rng.random(T), top_p=rng.choice([0.9, 1.0, 0.5], T), top_k=rng.choice([0, 0, 40, 1200], T))


def test_fewer_rows_than_the_sampler_has():
    s = P.Sampler(40, 5000)
    x = rows(12, 7, 5000, "bf16")
    check(x, np.random.default_rng(2).random(7), sampler=s, top_k=20)


def test_repeats_streams_and_graphs():
    """One row's token does not depend on its place, on another stream or on a replay."""
    T, V = 40, 30011
    x = rows(13, T, V, "bf16", head=6.0)
    rng = np.random.default_rng(3)
    u = up(rng.random(T), np.float32)
    par = dict(top_k=up(rng.choice([0, 20, 3000], T), np.int32), top_p=up(rng.choice([1.0, 0.9], T), np.float32),
               temperature=up(rng.choice([0.0, 0.8, 1.0], T), np.float32))
    s = P.Sampler(T, V)
    tok, lp = s(x, u, **par)
    perm = torch.randperm(T, device="cuda")
    t2, l2 = s(x[perm], u[perm], **{n: v[perm] for n, v in par.items()})
    assert torch.equal(tok[perm], t2) and torch.equal(lp[perm], l2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    t3, l3 = s(x, u, stream=side, **par)
    side.synchronize()
    assert torch.equal(tok, t3) and torch.equal(lp, l3)
    out = torch.empty_like(tok), torch.empty_like(lp)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s(x, u, token=out[0], logprob=out[1], **par)
    for i in range(4):
        x.copy_(rows(20 + i, T, V, "bf16", head=6.0))
        u.copy_(up(rng.random(T), np.float32))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        want = s(x, u, **par)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i


def test_sampled_trees_are_accepted():
    """Sampled tokens drive the greedy walk: the accepted path follows the children that
    were sampled, and the bonus is the last node's own sample."""
    rng = np.random.default_rng(6)
    R, N, V = 3, 24, 999
    from paper_2608_02123_amd import synth
    tok, par = np.zeros((R, N), np.int32), np.zeros((R, N), np.int32)
    for r in range(R):
        tok[r], par[r], _ = synth.random_tree(rng, N, N, 6, V)
    x = rows(14, R * N, V, "f32")
    u = rng.random(R * N)
    token, parent = (torch.from_numpy(a).cuda() for a in (tok, par))
    # sampled at some nodes to be one of the children
    for r in range(R):
        for i in range(1, N):
            if rng.random() < 0.4:
                x[r * N + par[r, i], int(tok[r, i])] = 40.0
    target, _ = P.sample(x, up(u, np.float32), top_p=up(np.full(R * N, 0.9), np.float32))
    count = torch.full((R,), N, dtype=torch.int32, device="cuda")
    rws, nrows = P.build_retrieve(parent, count, 6)
    acc = P.accept_greedy(token, rws, nrows, target.view(R, N))
    want, _, _ = SO.sample(x.cpu().double().numpy(), u.astype(np.float32).astype(np.float64),
                           top_p=np.full(R * N, 0.9, np.float32))
    want = want.reshape(R, N)
    for r in range(R):
        node, n = 0, 0
        while True:
            kids = [i for i in range(1, N) if par[r, i] == node and tok[r, i] == want[r, node]]
            if not kids:
                break
            node, n = kids[0], n + 1
        assert int(acc["accept_len"][r]) == n and int(acc["bonus"][r]) == want[r, node]
