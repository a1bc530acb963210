"""CPU checks of sampling: pins of the oracle, refusals of the C ABI and the binding."""
from __future__ import annotations

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import pctree_sample as SO
from paper_2608_02123_amd import pctree as P

A = 0x100000


def test_oracle_by_hand():
    # weights 8, 4, 2, 1, 1 (of 16): tokens 2, 0, 4, 1, 3 by weight
    x = np.log([4.0, 1.0, 8.0, 1.0, 2.0])
    tok = lambda u, **kw: SO.sample_row(x, u, **kw)[0]  # noqa: E731
    # running shares by token: .25, .3125, .8125, .875, 1
    assert [tok(u) for u in (0.0, 0.24, 0.26, 0.32, 0.8, 0.82, 0.9, 0.999)] == [0, 0, 1, 2, 2, 3, 4, 4]
    assert [tok(u, top_k=2) for u in (0.3, 0.34)] == [0, 2]            # weights 4, 8
    assert [tok(u, top_p=0.5) for u in (0.0, 0.99)] == [2, 2]          # 8 of 16 reach it
    assert [tok(u, top_p=0.51) for u in (0.3, 0.34)] == [0, 2]
    assert [tok(u, min_p=0.25) for u in (0.28, 0.29, 0.86)] == [0, 2, 4]  # 4, 8, 2
    assert [tok(u, top_k=4, top_p=0.85) for u in (0.28, 0.86)] == [0, 4]  # 8, 4 and 2 reach 12.75 of 15
    assert SO.sample_row(x, 0.5, temperature=0.0)[:2] == (2, 0.0)
    assert math.isclose(SO.sample_row(x, 0.0)[1], math.log(0.25))
    # temperature 1/2 squares the weights: 16, 1, 64, 1, 4 of 86
    assert [tok(u, temperature=0.5) for u in (0.18, 0.19, 0.2)] == [0, 1, 2]


def test_oracle_against_enumeration():
    """Sampled frequencies over an even grid of uniforms are the kept shares."""
    rng = np.random.default_rng(0)
    x = rng.normal(0, 2, 12)
    grid = (np.arange(20000) + 0.5) / 20000
    for kw in (dict(), dict(top_k=5), dict(top_p=0.7), dict(min_p=0.1), dict(temperature=0.7, top_k=8, top_p=0.9)):
        got = np.bincount([SO.sample_row(x, u, **kw)[0] for u in grid[::20]], minlength=12) / 1000
        w = np.exp((x - x.max()) / kw.get("temperature", 1.0))
        keep = np.argsort(-x)[:kw.get("top_k", 12)]
        keep = keep[w[keep] >= kw.get("min_p", 0)]
        if "top_p" in kw:
            c = np.cumsum(w[keep]) / w[keep].sum()
            keep = keep[:int((c < kw["top_p"]).sum()) + 1]
        share = np.zeros(12)
        share[keep] = w[keep] / w[keep].sum()
        assert np.abs(got - share).max() < 2e-3


def test_oracle_edges():
    inf, nan = math.inf, math.nan
    assert SO.sample_row([-inf, -inf], 0.5)[0] == -1
    assert SO.sample_row([nan, 1.0, -inf], 0.99)[0] == 1
    assert SO.sample_row([0.0, inf, 3.0, inf], 0.6)[0] == 3
    assert SO.sample_row([1.0, 1.0, 1.0, 1.0], 0.5)[0] == 2
    assert SO.sample_row([1.0, 1.0, 1.0, 1.0], 1.5)[0] == 3
    assert SO.sample_row([1.0, 1.0], 0.0, top_p=0.0)[0] == 0


def call(**kw):
    names = ["logits", "dtype", "rows", "vocab", "row_stride", "uniform", "temperature", "top_k", "top_p", "min_p",
             "token", "logprob", "workspace", "workspace_bytes"]
    ok = dict(zip(names, [A, P.BF16, 4, 1000, 1000, A, A, A, A, A, A, A, A, 1 << 30]))
    ok.update(kw)
    return P.lib().pctree_sample(*(ok[n] for n in names), None)


def test_refusals():
    for kw in (dict(logits=None), dict(uniform=None), dict(token=None), dict(dtype=3), dict(dtype=-1), dict(rows=0),
               dict(vocab=0), dict(row_stride=999), dict(row_stride=1 << 62), dict(logits=A + 1), dict(uniform=A + 2),
               dict(temperature=A + 1), dict(top_k=A + 2), dict(top_p=A + 3), dict(min_p=A + 1), dict(token=A + 2),
               dict(logprob=A + 1), dict(dtype=P.F32, logits=A + 2)):
        assert call(**kw) == P.ERR_INVALID_ARGUMENT, kw
    assert call(vocab=(1 << 20) + 1, row_stride=1 << 21) == P.ERR_UNSUPPORTED
    assert call(rows=1 << 30, vocab=1 << 20, row_stride=1 << 20) == P.ERR_UNSUPPORTED
    need = P.lib().pctree_sample_workspace_bytes(4, 1000)
    assert need > 0
    for kw in (dict(workspace=None), dict(workspace=A + 128), dict(workspace_bytes=need - 1)):
        assert call(**kw) == P.ERR_WORKSPACE, kw
    for r, v in ((0, 10), (10, 0), (1, (1 << 20) + 1), (1 << 30, 1 << 20)):
        assert P.lib().pctree_sample_workspace_bytes(r, v) == 0


def test_binding_refusals():
    with pytest.raises(P.PCTreeError):
        P.Sampler(0, 100, device="cpu")
    with pytest.raises(P.PCTreeError):
        P.Sampler(1, 1 << 21, device="cpu")
    s = P.Sampler(4, 100, device="cpu")
    u = torch.zeros(2)
    with pytest.raises(TypeError):
        s(torch.zeros(2, 100, dtype=torch.float64), u)
    for bad in (torch.zeros(2, 99), torch.zeros(5, 100), torch.zeros(100), torch.zeros(100, 2).t(),
                torch.zeros(1, 100).expand(2, 100)):
        with pytest.raises(ValueError):
            s(bad, u)
    with pytest.raises(ValueError):  # (host tensors)
        s(torch.zeros(2, 100), u)
    with pytest.raises(ValueError):
        P.sample(torch.zeros(2, 100), u)
    assert ctypes.sizeof(ctypes.c_float) == 4
