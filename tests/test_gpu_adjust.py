"""GPU parity of penalties, biases and masks on logits against the float64 oracle.

Tolerance: five float32 operations, each off by 2^-24 of the magnitudes that are added (the
oracle's ``mag``), then one rounding to the logits' type, u |y|: |err| <= 5 * 2^-24 mag + u |y|
(float16's smallest half step 2^-25).  Logits that nothing concerns keep their bits.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import pctree_step as SO
from paper_2608_02123_amd import pctree as P
from paper_2608_02123_amd import synth

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def up(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ragged(rng, R, low, high, V, wild=False):
    """(list, start, count) with some tokens outside the vocabulary."""
    count = rng.integers(low, high + 1, R).astype(np.int32)
    start = (np.cumsum(count) - count).astype(np.int32)
    tokens = np.minimum(rng.zipf(1.3, max(int(count.sum()), 1)) - 1, 10 * V) * 37 % (V + 3 if wild else V)
    if wild and len(tokens) > 2:
        tokens[0] = -1
    return tokens.astype(np.int32), start, count


def case(rng, R, rows, V, dt, *, history=(0, 200), bias=0, tree=False, grammar=None, penalties=True, gap=0, wild=True):
    T = R * (rows + gap)
    a = {"row_start": (np.arange(R) * (rows + gap)).astype(np.int32),
         "row_count": rng.integers(1, rows + 1, R).astype(np.int32) if not tree else np.full(R, rows, np.int32)}
    if history:
        a["history"], a["history_start"], a["history_count"] = ragged(rng, R, *history, V, wild)
        a["prompt_count"] = (a["history_count"] * rng.random(R)).astype(np.int32)
    if penalties:
        a["repetition"] = rng.choice([1.0, 1.1, 1.3, 0.8], R).astype(np.float32)
        a["frequency"] = rng.choice([0.0, 0.1, 0.7, -0.3], R).astype(np.float32)
        a["presence"] = rng.choice([0.0, 0.2, 1.5], R).astype(np.float32)
    if bias:
        a["bias_token"], a["bias_start"], a["bias_count"] = ragged(rng, R, 0, bias, V, wild)
        a["bias_value"] = (rng.standard_normal(len(a["bias_token"])) * 5).astype(np.float32)
        a["bias_value"][::7] = -np.inf
    if tree:
        par = np.full((R, rows), -1, np.int32)
        for r in range(R):
            _, par[r], _ = synth.random_tree(rng, rows, rows, 16, V)
        a["token"] = rng.integers(-1, min(V, 12) + 1, (R, rows)).astype(np.int32)  # (the same tokens again and again)
        a["mask"] = P.build_mask(up(par), up(a["row_count"])).cpu().numpy()
    if grammar:
        W = (V + 31) // 32
        M = grammar
        words = rng.integers(0, 2 ** 32, (M, W), dtype=np.uint32) & rng.integers(0, 2 ** 32, (M, W), dtype=np.uint32)
        words[:, ::3] = 0
        words[:, 1::3] = 0xffffffff
        a["allowed"] = words.view(np.int32)
        a["allowed_row"] = rng.integers(-1, M + 1, T).astype(np.int32)
    logits = torch.randn(T, V, generator=torch.Generator().manual_seed(int(rng.integers(1 << 30)))) * 4
    logits[0, :3] = torch.tensor([float("inf"), float("-inf"), 0.0])[:V]
    return logits.to(dt).cuda(), a


def check(logits, a, max_rows=None, stride=0):
    dt = logits.dtype
    if stride:
        wide = torch.full((logits.shape[0], logits.shape[1] + stride), 5.0, dtype=dt, device="cuda")
        wide[:, :logits.shape[1]] = logits
        logits = wide[:, :logits.shape[1]]
    before = logits.clone()
    x0 = before.double().cpu().numpy()
    want, mag, hit = SO.adjust(x0, a["row_start"], a["row_count"], max_rows or len(x0),
                               **{k: v for k, v in a.items() if k not in ("row_start", "row_count")})
    with np.errstate(over="ignore"):
        want_t = torch.from_numpy(want).to(dt).double().numpy()  # (what the type rounds to infinity)
    assert P.adjust_logits(logits, up(a["row_start"]), up(a["row_count"]), max_rows=max_rows,
                           **{k: up(v) for k, v in a.items() if k not in ("row_start", "row_count")}) is logits
    got = logits.double().cpu().numpy()
    same = torch.equal(logits[torch.from_numpy(~hit).cuda()], before[torch.from_numpy(~hit).cuda()])
    assert same, "logits that nothing concerns changed"
    odd = ~np.isfinite(want_t)
    assert np.array_equal(got[odd], want_t[odd], equal_nan=True)
    tol = 5 * 2.0 ** -24 * mag + HALF[dt] * np.abs(want) + 2.0 ** -25 * (dt == torch.float16)
    err = np.abs(got - want)
    assert (err[~odd] <= tol[~odd]).all(), float(np.nanmax((err / np.maximum(tol, 1e-30))[~odd]))
    if stride:
        assert (wide[:, -stride:] == 5).all()
    return logits


@pytest.mark.parametrize("dt", list(HALF))
@pytest.mark.parametrize("V", [1, 31, 33, 1000, 4095, 4096, 4104, 50021])
def test_penalties(dt, V):
    rng = np.random.default_rng(V)
    check(*case(rng, 5, 2, V, dt, gap=1))


@pytest.mark.parametrize("dt", list(HALF))
@pytest.mark.parametrize("V", [7, 1000, 8200])
@pytest.mark.parametrize("kw", [dict(bias=30, penalties=False, history=None), dict(bias=300), dict(grammar=3),
                                dict(grammar=4, bias=40, tree=True), dict(tree=True), dict(tree=True, history=None),
                                dict(grammar=2, penalties=False, history=None)])
def test_parts(dt, V, kw):
    rng = np.random.default_rng((V, len(kw)))
    check(*case(rng, 3, 20, V, dt, **kw), stride=24)


def test_trees_of_many_nodes():
    """More nodes than a wave has lanes, most of them with tokens of one segment."""
    rng = np.random.default_rng(1)
    logits, a = case(rng, 2, 300, 5000, torch.float32, tree=True, grammar=5, history=(20, 50))
    check(logits, a)
    a["allowed_row"][:] = -1
    check(case(rng, 2, 300, 5000, torch.float32)[0], a)


@pytest.mark.parametrize("R,rows,V", [(1, 1, 1800), (2, 3, 1800), (1, 70, 300), (40, 9, 2100), (70, 4, 2100), (90, 13, 4100)])
def test_tables_that_hold_most_of_the_vocabulary(R, rows, V):
    """Rows that a workgroup has one, a few or many of, and tokens that its waves share."""
    rng = np.random.default_rng((R, rows))
    logits, a = case(rng, R, rows, V, torch.bfloat16, tree=True, grammar=3, bias=200, history=(1000, 3500))
    a["token"] = rng.integers(-1, V + 1, (R, rows)).astype(np.int32)
    check(logits, a, max_rows=rows)
    a["row_count"] = rng.integers(0, rows + 1, R).astype(np.int32)
    check(case(rng, R, rows, V, torch.bfloat16)[0], a)


def test_long_histories():
    rng = np.random.default_rng(2)
    check(*case(rng, 2, 1, 151936, torch.bfloat16, history=(40000, 60000), wild=False))


def test_a_mask_for_every_row_and_rows_of_none():
    rng = np.random.default_rng(3)
    logits, a = case(rng, 4, 3, 1000, torch.float16, grammar=12)
    del a["allowed_row"]
    check(logits, a)
    a["row_start"] = np.array([-1, 12, 3, 11], np.int32)
    a["row_count"] = np.array([5, 1, -2, 100], np.int32)
    check(logits, a, max_rows=2)


def test_a_mask_that_allows_nothing_leaves_nothing():
    logits = torch.zeros(2, 100, device="cuda")
    allowed = np.zeros((1, 4), np.int32)
    a = {"row_start": np.zeros(1, np.int32), "row_count": np.array([2], np.int32), "allowed": allowed,
         "allowed_row": np.array([0, 5], np.int32)}
    check(logits, a)
    token, logprob = P.sample(logits, torch.full((2,), 0.5, device="cuda"))
    assert token[0] == -1 and logprob[0] == -np.inf and token[1] >= 0


def test_of_a_tokens_biases_the_last_holds():
    V = 5000
    a = {"row_start": np.array([0, 1], np.int32), "row_count": np.array([1, 1], np.int32),
         "bias_token": np.array([4999, 3, 3, 4999, 3, 3, 7], np.int32),
         "bias_value": np.array([1, 2, 4, 8, 16, 32, 64], np.float32),
         "bias_start": np.array([0, 4], np.int32), "bias_count": np.array([4, 50], np.int32)}
    x = check(torch.zeros(2, V, device="cuda"), a)
    assert x[0, 3] == 4 and x[0, 4999] == 8 and x[1, 3] == 32 and x[1, 7] == 64 and x[1, 4999] == 0


def test_odd_parameters_count_as_off():
    rng = np.random.default_rng(5)
    logits, a = case(rng, 6, 1, 2000, torch.float32, history=(50, 90))
    a["repetition"] = np.array([0.0, -1.0, np.nan, np.inf, 1.0, 1.5], np.float32)
    a["frequency"] = np.array([np.nan, np.inf, 0.0, 0.0, 0.0, -np.inf], np.float32)
    a["presence"] = np.array([0.0, -np.inf, np.nan, 0.0, 0.0, np.inf], np.float32)
    before = logits.clone()
    after = check(logits, a)
    assert torch.equal(after[:5], before[:5]) and not torch.equal(after[5], before[5])


def test_ranges_past_the_lists_are_clamped():
    rng = np.random.default_rng(6)
    logits, a = case(rng, 4, 1, 500, torch.bfloat16, bias=20, history=(5, 20))
    n = len(a["history"])
    a["history_start"] = np.array([-5, n + 9, n - 2, 0], np.int32)
    a["history_count"] = np.array([10, 10, 1000, -1], np.int32)
    a["prompt_count"] = np.array([100, 1, -1, 5], np.int32)
    a["bias_start"] = np.array([2 ** 31 - 1, -7, 3, 0], np.int32)
    a["bias_count"] = np.array([5, 4, 2 ** 31 - 1, -3], np.int32)
    check(logits, a)


def test_nan_stays_and_what_no_row_holds_keeps_its_bits():
    """A NaN logit of a token that only another branch of the tree holds keeps its payload; one
    that is penalised stays NaN; a forbidden one becomes -inf."""
    x = torch.zeros(3, 100, dtype=torch.int16, device="cuda")
    x[:, 7], x[:, 9], x[:, 50] = 0x7f91, 0x7fa5, 0x7fc1
    x = x.view(torch.bfloat16)
    before = x.clone()
    allowed = np.full((1, 4), -1, np.int32)
    allowed[0, 1] = ~(1 << 18)  # token 50
    a = {"row_start": np.zeros(1, np.int32), "row_count": np.array([3], np.int32),
         "token": np.array([[1, 7, 9]], np.int32), "mask": np.array([[[1], [3], [5]]], np.int32),
         "presence": np.ones(1, np.float32), "allowed": allowed, "allowed_row": np.zeros(3, np.int32)}
    P.adjust_logits(x, up(a["row_start"]), up(a["row_count"]), **{k: up(v) for k, v in a.items() if k[:3] != "row"})
    assert (x[:, 50] == -np.inf).all() and (x[:, 1] == -1).all()
    bits, was = x.view(torch.int16), before.view(torch.int16)
    assert bits[0, 7] == was[0, 7] and bits[2, 7] == was[2, 7] and bits[0, 9] == was[0, 9] and bits[1, 9] == was[1, 9]
    assert torch.isnan(x[1, 7]) and torch.isnan(x[2, 9])


def test_empty_lists():
    x = torch.randn(2, 300, generator=torch.Generator().manual_seed(0)).cuda()
    before, e = x.clone(), torch.zeros(0, dtype=torch.int32, device="cuda")
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    rows = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    P.adjust_logits(x, rows, i + 1, history=e, history_start=i, history_count=i, prompt_count=i,
                    presence=torch.ones(2, device="cuda"), bias_token=e, bias_value=e.float(), bias_start=i,
                    bias_count=i)
    assert torch.equal(x, before)


def test_logits_past_32_bits():
    """Rows whose offsets pass 2^32 bytes, one of them with a mask."""
    V, T = 151936, 15000  # 4.6 GB
    x = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([T - 2, 0], dtype=torch.int32, device="cuda")
    count = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
    tokens = torch.tensor([5, V - 1, V - 1, 70000], dtype=torch.int32, device="cuda")
    allowed = torch.full((1, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    allowed[0, 1] = 0  # tokens 32 to 63
    which = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    which[T - 1] = 0
    ones = torch.ones(2, device="cuda")
    P.adjust_logits(x, rows, count, max_rows=2, history=tokens, history_start=up(np.array([0, 3], np.int32)),
                    history_count=up(np.array([3, 1], np.int32)), frequency=ones, allowed=allowed, allowed_row=which)
    assert x[T - 2, 5] == -1 and x[T - 1, V - 1] == -2 and x[0, 70000] == -1 and x[0, 5] == 0
    assert (x[T - 1, 32:64] == -np.inf).all() and (x[T - 2, 32:64] == 0).all() and x[T - 1, 64] == 0
    x[T - 2:, 5] = x[T - 2:, V - 1] = x[0, 70000] = 0
    x[T - 1, 32:64] = 0
    assert int(torch.count_nonzero(x.view(torch.int16).view(-1, V)[::100]).item()) == 0
    assert not x[T - 3:].view(torch.int32).any()


def test_refusals():
    x = torch.zeros(2, 100, device="cuda")
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    f = torch.ones(2, device="cuda")
    words = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    for kw, error in ((dict(history=i), P.PCTreeError), (dict(history=i.long()), TypeError),
                      (dict(repetition=i), TypeError), (dict(repetition=f[:1]), ValueError),
                      (dict(bias_token=i, bias_value=f[:1], bias_start=i, bias_count=i), ValueError),
                      (dict(bias_token=i, bias_value=f), P.PCTreeError),
                      (dict(token=words), P.PCTreeError), (dict(mask=words), ValueError),
                      (dict(allowed=words[:, :3]), ValueError), (dict(allowed=words.float()), TypeError),
                      (dict(allowed_row=i), P.PCTreeError), (dict(allowed=words[:1].contiguous()), P.PCTreeError),
                      (dict(max_rows=3), P.PCTreeError), (dict(max_rows=1 << 32), ValueError),
                      (dict(prompt_count=i), P.PCTreeError)):
        with pytest.raises(error):
            P.adjust_logits(x, i, i, **kw)
    with pytest.raises(ValueError):
        P.adjust_logits(x.t(), i, i)
    with pytest.raises(ValueError):
        P.adjust_logits(x, i[:1], i)
