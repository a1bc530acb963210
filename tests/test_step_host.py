"""CPU refusals of the norm and of what is done to logits: the C ABI and the binding."""
from __future__ import annotations

import ctypes
import pathlib
import re

import pytest
import torch

from paper_2608_02123_amd import pctree as P

A = 0x100000  # a suitably aligned address that nothing reads


def norm(**kw):
    f = dict(x=A, weight=A, residual=A, out=A, scale=A, x_stride=4096, residual_stride=4096, out_stride=4096, rows=5,
             width=4096, group=128, dtype=P.BF16, eps=1e-6)
    f.update(kw)
    return P.lib().pctree_rms_norm(ctypes.byref(P._Norm(*(f[n] for n, _ in P._Norm._fields_))), None)


def adjust(**kw):
    f = {n: A for n, t in P._Adjust._fields_ if t is ctypes.c_void_p}
    f.update(row_stride=1000, rows=6, vocab=1000, requests=2, max_rows=4, history_total=50, bias_total=7, budget=4,
             masks=3, dtype=P.BF16)
    f.update(kw)
    return P.lib().pctree_adjust_logits(ctypes.byref(P._Adjust(*(f[n] for n, _ in P._Adjust._fields_))), None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), 1), (dict(out=None), 1), (dict(rows=0), 1), (dict(width=0), 1), (dict(width=100, x_stride=104), 1),
    (dict(dtype=P.F32), 1), (dict(dtype=7), 1), (dict(group=-1), 1), (dict(group=16), 1), (dict(group=100), 1),
    (dict(x=A + 8), 1), (dict(weight=A + 2), 1), (dict(residual=A + 8), 1), (dict(out=A + 4), 1),
    (dict(scale=None, out=A + 8), 1), (dict(scale=A + 2), 1), (dict(x_stride=4088), 1), (dict(x_stride=4100), 1),
    (dict(residual_stride=4088), 1), (dict(out_stride=4095), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
    (dict(eps=float("inf")), 1), (dict(x_stride=1 << 62), 1),
    (dict(width=32776, x_stride=32776, residual_stride=32776, out_stride=32776), 2), (dict(rows=(1 << 21) + 1), 2)])
def test_norms_that_are_refused(kw, code):
    assert norm(**kw) == code
    assert P.lib().pctree_rms_norm(None, None) == P.ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), 1), (dict(row_start=None), 1), (dict(row_count=None), 1), (dict(rows=0), 1), (dict(vocab=0), 1),
    (dict(requests=0), 1), (dict(max_rows=0), 1), (dict(max_rows=7), 1), (dict(row_stride=999), 1), (dict(dtype=3), 1),
    (dict(row_stride=1 << 62), 1), (dict(logits=A + 1), 1), (dict(logits=A + 2, dtype=P.F32), 1),
    (dict(history=None), 1), (dict(history_start=None), 1), (dict(history_count=None), 1), (dict(history_total=0), 1),
    (dict(history=None, history_start=None, history_count=None, history_total=0), 1),  # prompt_count stays
    (dict(bias_value=None), 1), (dict(bias_start=None), 1), (dict(bias_count=None), 1), (dict(bias_total=0), 1),
    (dict(bias_token=None), 1), (dict(token=None), 1), (dict(mask=None), 1), (dict(budget=0), 1), (dict(masks=0), 1),
    (dict(allowed=None), 1), (dict(allowed=None, masks=0), 1), (dict(allowed_row=None, masks=5), 1),
    (dict(repetition=A + 2), 1), (dict(bias_token=A + 1), 1), (dict(allowed=A + 2), 1),
    (dict(vocab=(1 << 20) + 1, row_stride=1 << 21), 2), (dict(requests=70000), 2), (dict(budget=1025), 2),
    (dict(history_total=1 << 29), 2), (dict(vocab=1 << 20, row_stride=1 << 20, requests=65535, rows=65535), 2),
    (dict(vocab=1 << 20, row_stride=1 << 20, rows=1 << 22, masks=1), 2)])
def test_adjustments_that_are_refused(kw, code):
    assert adjust(**kw) == code
    assert P.lib().pctree_adjust_logits(None, None) == P.ERR_INVALID_ARGUMENT


def test_binding_refuses_host_tensors_and_types():
    x, i = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for call, error in ((lambda: P.rms_norm(x), ValueError), (lambda: P.rms_norm(x.float()), TypeError),
                        (lambda: P.rms_norm([1.0]), TypeError), (lambda: P.adjust_logits(x, i, i), ValueError),
                        (lambda: P.adjust_logits(x.double(), i, i), TypeError),
                        (lambda: P.adjust_logits(x[0], i, i), ValueError)):
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("total", [1 << 29, (1 << 31) - 200, (1 << 31) - 1])
def test_lists_of_biases_past_a_counters_range(total):
    """A thread's counter passes a request's entries by up to a workgroup's step."""
    assert adjust(bias_total=total) == P.ERR_UNSUPPORTED
    assert adjust(history_total=total) == P.ERR_UNSUPPORTED


def test_dynamic_lds_is_as_aligned_as_its_stores():
    """The launch's LDS begins behind a kernel's own, at the array's alignment: what is written there in
    16 bytes has to ask for as many."""
    found = 0
    for path in sorted((pathlib.Path(P.__file__).parent / "csrc").glob("*.hip")):
        text = path.read_text()
        for align, name in re.findall(r"extern __shared__ (__attribute__\(\(aligned\(16\)\)\) )?\w+ (\w+)\[\]", text):
            names, more = set(), {name}
            while more:  # what points into it
                names |= more
                more = {a for n in names for a in re.findall(rf"\* (\w+) = (?:\(\w+\*\))?\(?{n}\b", text)} - names
            wide = any(re.search(rf"\(u?\w*x4\*\)\(?{n}\b", text) for n in names)
            assert align or not wide, f"{path.name}: {name}"
            found += wide
    assert found
