"""CPU checks of pages in 8 bits: the oracle's numbers, scales and rounding against torch's
conversions and direct search, and the refusals of the C ABI and of the binding."""
from __future__ import annotations

import ctypes
import inspect
import math

import numpy as np
import pytest
import torch

from oracle import pctree_held as HO
from paper_2608_02123_amd import pctree as P
from test_paged_host import A, BAD_APPENDS, BAD_BATCHES, append, batch, cache


def cache8(block=16, k_scale=A, v_scale=A, scale_stride=None, **kw):
    c = cache(**kw)
    n = max(c.kv_heads * (c.page_size // block if block > 0 else 1), 1)
    return P._PagedCache8(c, k_scale, v_scale, n if scale_stride is None else scale_stride, block)


def do_append(c=None, b=None, a=None):
    return P.lib().pctree_append_paged8(ctypes.byref(c or cache8()), ctypes.byref(b or batch()),
                                        ctypes.byref(a or append()), None)


def do_attention(c=None, b=None, q=A, heads=32, scale=0.1, mask=None, budget=0, out=A, ws=A, nb=1 << 40):
    return P.lib().pctree_paged_attention8(ctypes.byref(c or cache8()), ctypes.byref(b or batch()), q, heads, scale,
                                           mask, budget, out, ws, nb, None)


def test_numbers_are_torchs():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(HO.NUMBERS, got, equal_nan=True)
    assert HO.NUMBERS[126] == 448.0 and HO.NUMBERS[1] == 2.0 ** -9


def test_hold_is_the_nearest_number():
    """Over random values, all ties and the ends, against torch's conversion."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(20000, generator=g) * torch.exp2(torch.randint(-14, 9, (20000,), generator=g).float())
    pos = torch.from_numpy(HO.NUMBERS[:127]).float()
    x = torch.cat([x.clamp(-448, 448), pos, -pos, (pos[1:] + pos[:-1]) / 2, -(pos[1:] + pos[:-1]) / 2])
    assert np.array_equal(HO.hold(x.double().numpy(), 127), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    odd = HO.hold([math.inf, -math.inf, math.nan, 465.0, 464.0, -449.0], 127)
    assert list(odd & 127) == [127, 127, 127, 127, 126, 126]


@pytest.mark.parametrize("x,s", [(0.0, 16), (448.0, 127), (math.nextafter(448.0, 1e9), 128), (1.0, 119),
                                 (1.75, 119), (math.nextafter(1.75, 2.0), 120), (3.4e38, 246), (1e-40, 16)])
def test_scales(x, s):
    assert HO.scale_byte(x) == s
    if 16 < s < 246:  # the smallest that will do
        assert x <= 448 * 2.0 ** (s - 127) and x > 448 * 2.0 ** (s - 128)


def test_rescaling_keeps_what_stays_normal():
    b = np.arange(256, dtype=np.uint8)
    v = HO.NUMBERS * 2.0 ** 3
    with np.errstate(invalid="ignore"):
        for k in range(1, 14):
            got = HO.values(HO.rescale(b, 130, 130 + k)[None, :, None], np.array([[130 + k]], np.uint8))[0, :, 0]
            normal = np.abs(HO.NUMBERS) >= 2.0 ** (k - 6)
            assert np.array_equal(got[normal], v[normal])
            err = np.abs(got - v)[~normal & ~np.isnan(v)]
            assert (err <= 2.0 ** (k - 10 + 3)).all()  # half a step of the smallest numbers
    assert (HO.rescale(b, 130, 140)[[127, 255]] & 127 == 127).all()


@pytest.mark.parametrize("kw,code", [
    (dict(block=0), 1), (dict(block=-8), 1), (dict(block=4), 2), (dict(block=24), 2), (dict(block=128, page_size=256), 2),
    (dict(block=32, page_size=16), 1), (dict(scale_stride=7), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1),
    (dict(page_stride=8 * 16 * 128 + 8), 1), (dict(k=A + 8), 1), (dict(head_dim=96), 2), (dict(pages=0), 1),
    (dict(dtype=P.F32), 1), (dict(page_size=24), 2), (dict(scale_stride=1 << 62), 1)])
def test_caches_that_are_refused(kw, code):
    assert do_append(c=cache8(**kw)) == code
    assert do_attention(c=cache8(**kw)) == code
    if not {"k_scale", "v_scale", "k"} & set(kw):
        assert P.lib().pctree_paged_attention8_workspace_bytes(ctypes.byref(cache8(**kw)), ctypes.byref(batch()),
                                                               32) == 0


@pytest.mark.parametrize("kw,code", BAD_BATCHES)
def test_batches_that_are_refused(kw, code):
    assert do_append(b=batch(**kw)) == code
    assert do_attention(b=batch(**kw)) == code


@pytest.mark.parametrize("kw,code", BAD_APPENDS)
def test_appends_that_are_refused(kw, code):
    assert do_append(a=append(**kw)) == code


def test_null_structs_and_operands():
    c, b, a = cache8(), batch(), append()
    f, g = P.lib().pctree_append_paged8, P.lib().pctree_paged_attention8
    for args in ((None, b, a), (c, None, a), (c, b, None)):
        assert f(*(ctypes.byref(x) if x is not None else None for x in args), None) == P.ERR_INVALID_ARGUMENT
    assert g(None, ctypes.byref(b), A, 32, 0.1, None, 0, A, A, 1 << 40, None) == P.ERR_INVALID_ARGUMENT
    for kw in (dict(q=None), dict(out=None), dict(heads=12), dict(scale=0.0), dict(mask=A, budget=0)):
        assert do_attention(**kw) == P.ERR_INVALID_ARGUMENT, kw
    need = P.lib().pctree_paged_attention8_workspace_bytes(ctypes.byref(c), ctypes.byref(b), 32)
    assert need > 0
    assert do_attention(nb=need - 1) == do_attention(ws=None) == P.ERR_WORKSPACE
    assert do_append(b=batch(rows=1 << 23, max_rows=1), c=cache8()) == P.ERR_UNSUPPORTED  # a launch's limit


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 32, 8), (64, 28, 4), (128, 8, 1)])
@pytest.mark.parametrize("R,T,most", [(1, 1, 1), (64, 64, 1), (1, 300, 300), (24, 900, 300), (200, 200, 1)])
@pytest.mark.parametrize("slots,page", [(64, 16), (1000, 16), (70000, 64), (300, 4)])
def test_an_objects_workspace_serves_both_kinds_of_pages(D, Hq, Hkv, R, T, most, slots, page):
    b = batch(requests=R, rows=T, max_rows=most, max_pages=-(-slots // page))
    c = cache8(block=8, kv_heads=Hkv, head_dim=D, page_size=page) if page >= 8 else None
    plain = cache(kv_heads=Hkv, head_dim=D, page_size=page)
    w8 = P.lib().pctree_paged_attention8_workspace_bytes(ctypes.byref(c), ctypes.byref(b), Hq) if c else 0
    w16 = P.lib().pctree_paged_attention_workspace_bytes(ctypes.byref(plain), ctypes.byref(b), Hq)

    class Batch:
        sizes, idx, _ref, device = (R, b.max_pages, T, most), -1, ctypes.byref(b), "meta"
    assert P.PagedAttention(Batch, Hq, Hkv, D, page).ws_bytes == max(w8, w16)


def test_compact_refusals():
    names = ["pool", "group_stride", "page_stride", "scale", "scale_group_stride", "scale_page_stride", "groups",
             "pages", "heads", "page_size", "head_dim", "block", "page_table", "max_pages", "prefix_len",
             "accept_node", "accept_len", "requests", "budget", "max_depth"]
    ok = dict(zip(names, [A, 1 << 20, 8 * 16 * 128, A, 160, 16, 4, 10, 8, 16, 128, 8, A, 20, A, A, A, 2, 64, 16]))

    def call(**kw):
        return P.lib().pctree_compact_paged8(*({**ok, **kw}[n] for n in names), None)

    for kw in (dict(pool=None), dict(scale=None), dict(page_table=None), dict(block=0), dict(block=32),
               dict(scale_page_stride=15), dict(scale_group_stride=-1), dict(scale_group_stride=16),
               dict(group_stride=1 << 14), dict(head_dim=8), dict(max_depth=-1), dict(page_stride=8 * 16 * 128 + 8)):
        assert call(**kw) == P.ERR_INVALID_ARGUMENT, kw
    for kw in (dict(head_dim=96, page_stride=1 << 15), dict(block=4, scale_page_stride=64, scale_group_stride=1 << 12),
               dict(max_depth=64), dict(requests=70000), dict(budget=1025)):
        assert call(**kw) == P.ERR_UNSUPPORTED, kw


def test_binding_refuses_what_is_no_held_cache():
    k = torch.zeros(4, 2, 16, 128, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.zeros(4, 2, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    bf = torch.bfloat16
    for bad in ((k, k, s, None, bf), (k, k, None, s, bf), (k, k, s.view(torch.uint8), s, bf), (k, k, s, s, torch.float32),
                (k.to(bf), k.to(bf), s, s, bf), (k.view(torch.uint8), k, s, s, bf)):
        with pytest.raises(TypeError):
            P._held_cache(*bad, -1)
    with pytest.raises(ValueError):  # host tensors
        P._held_cache(k, k, s, s, bf, 0)
    with pytest.raises(TypeError):  # pages in 8 bits without scales
        P._paged_cache(k, k, 0)


@pytest.mark.parametrize("call,names", [
    (P.PagedAttention.__call__, "self q k_cache v_cache batch mask out stream"),
    (P.paged_attention, "q k_cache v_cache batch mask scale out stream"),
    (P.compact_paged, "pool page_table prefix_len accept_node accept_len budget stream"),
    (P.append_paged, "batch k_cache v_cache k v q")])
def test_arguments_by_position(call, names):
    """Those of 16-bit pages keep their places; scales come by name."""
    p = inspect.signature(call).parameters.values()
    assert [x.name for x in p if x.kind is x.POSITIONAL_OR_KEYWORD] == names.split()


@pytest.mark.parametrize("groups,heads,D", [((1 << 25) - 1, 8, 128), ((1 << 26) + 64, 1, 64), (1 << 14, 1 << 13, 64)])
def test_compactions_past_a_launch(groups, heads, D):
    """A wave for every group and head: more than 2^32 - 1 threads cannot be launched."""
    block = heads * 8 * D
    assert P.lib().pctree_compact_paged8(A, block, block, A, heads, heads, groups, 1, heads, 8, D, 8, A, 20, A, A, A,
                                         2, 64, 16, None) == P.ERR_UNSUPPORTED


def test_rows_that_are_no_tensors():
    k = torch.zeros(4, 2, 16, 128, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.zeros(4, 2, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)

    class Batch:
        b = batch(requests=2, rows=3, max_rows=2, max_pages=4)
        idx, rows, requests, sizes, _ref, device = -1, 3, 2, (2, 4, 3, 2), ctypes.byref(b), "meta"
    for bad in (None, [1.0], 3):
        with pytest.raises(TypeError):
            P.append_paged(Batch, k, k, bad, bad, k_scale=s, v_scale=s)
        with pytest.raises(TypeError):
            P.PagedAttention(Batch, 2, 2, 128, 16)(bad, k, k, Batch, k_scale=s, v_scale=s)
