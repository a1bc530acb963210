"""CPU checks of the paged-cache calls: refusals of the C ABI and of the binding."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2608_02123_amd import pctree as P

A = 0x100000  # a suitably aligned address that nothing reads


def cache(**kw):
    f = dict(k=A, v=A, page_stride=8 * 16 * 128, pages=10, page_size=16, kv_heads=8, head_dim=128, dtype=P.BF16)
    f.update(kw)
    if "page_stride" not in kw:
        f["page_stride"] = max(f["kv_heads"] * f["page_size"] * f["head_dim"], 0) // 8 * 8
    return P._PagedCache(*(f[n] for n, _ in P._PagedCache._fields_))


def batch(**kw):
    f = dict(row_start=A, row_count=A, prefix_len=A, page_table=A, requests=3, max_pages=40, rows=12, max_rows=4)
    f.update(kw)
    return P._PagedBatch(*(f[n] for n, _ in P._PagedBatch._fields_))


def append(**kw):
    f = dict(q=A, k=A, v=A, q_out=A, q_stride=4096, k_stride=1024, v_stride=1024, q_out_stride=4096, q_norm=A,
             k_norm=A, rope=A, position=A, eps=1e-6, q_heads=32, rot_dim=128, positions=100, interleaved=0)
    f.update(kw)
    return P._Append(*(f[n] for n, _ in P._Append._fields_))


def do_append(c=None, b=None, a=None):
    return P.lib().pctree_append_paged(ctypes.byref(c or cache()), ctypes.byref(b or batch()),
                                       ctypes.byref(a or append()), None)


def do_attention(c=None, b=None, q=A, heads=32, scale=0.1, mask=None, budget=0, out=A, ws=A, nb=1 << 40):
    return P.lib().pctree_paged_attention(ctypes.byref(c or cache()), ctypes.byref(b or batch()), q, heads, scale,
                                          mask, budget, out, ws, nb, None)


BAD_CACHES = [(dict(pages=0), 1), (dict(page_size=0), 1), (dict(kv_heads=0), 1), (dict(head_dim=0), 1),
              (dict(dtype=P.F32), 1), (dict(dtype=9), 1), (dict(page_stride=8 * 16 * 128 - 8), 1),
              (dict(page_stride=8 * 16 * 128 + 4), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(k=A + 8), 1),
              (dict(head_dim=96), 2), (dict(page_size=24), 2), (dict(page_size=2048), 2),
              (dict(page_stride=1 << 36), 2)]
BAD_BATCHES = [(dict(requests=0), 1), (dict(max_pages=0), 1), (dict(rows=0), 1), (dict(max_rows=0), 1),
               (dict(max_rows=13), 1), (dict(row_start=None), 1), (dict(row_count=None), 1),
               (dict(prefix_len=None), 1), (dict(page_table=None), 1), (dict(page_table=A + 2), 1),
               (dict(requests=70000), 2), (dict(max_pages=(1 << 30) // 16 + 1), 2)]
BAD_APPENDS = [(dict(k=None), 1), (dict(v=None), 1), (dict(q=None), 1), (dict(q_out=None), 1),
               (dict(q=None, q_out=None), 1),  # q_heads stays 32
               (dict(q_heads=0), 1), (dict(k_stride=1016), 1), (dict(v_stride=1028), 1), (dict(q_stride=4088), 1),
               (dict(q_out_stride=4100), 1), (dict(k=A + 8), 1), (dict(q_norm=A + 2), 1), (dict(rope=A + 4), 1),
               (dict(position=A + 1), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
               (dict(eps=float("inf")), 1), (dict(rot_dim=0), 1), (dict(rot_dim=24), 1), (dict(rot_dim=144), 1),
               (dict(positions=0), 1), (dict(interleaved=2), 1), (dict(q_heads=70000, q_stride=70000 * 128,
                                                                       q_out_stride=70000 * 128), 2)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches_that_are_refused(kw, code):
    assert do_append(c=cache(**kw)) == code
    assert do_attention(c=cache(**kw)) == code
    if kw.get("k", 1) and kw.get("v", 1) and "k" not in kw:
        assert P.lib().pctree_paged_attention_workspace_bytes(ctypes.byref(cache(**kw)), ctypes.byref(batch()),
                                                              32) == 0


@pytest.mark.parametrize("kw,code", BAD_BATCHES)
def test_batches_that_are_refused(kw, code):
    assert do_append(b=batch(**kw)) == code
    assert do_attention(b=batch(**kw)) == code


@pytest.mark.parametrize("kw,code", BAD_APPENDS)
def test_appends_that_are_refused(kw, code):
    assert do_append(a=append(**kw)) == code


def test_null_structs():
    c, b, a = cache(), batch(), append()
    f, g = P.lib().pctree_append_paged, P.lib().pctree_paged_attention
    for args in ((None, b, a), (c, None, a), (c, b, None)):
        assert f(*(ctypes.byref(x) if x is not None else None for x in args), None) == P.ERR_INVALID_ARGUMENT
    assert g(None, ctypes.byref(b), A, 32, 0.1, None, 0, A, A, 1 << 40, None) == P.ERR_INVALID_ARGUMENT
    assert g(ctypes.byref(c), None, A, 32, 0.1, None, 0, A, A, 1 << 40, None) == P.ERR_INVALID_ARGUMENT


def test_attention_refusals():
    for kw in (dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 4), dict(heads=0), dict(heads=12),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(mask=A, budget=0), dict(mask=A + 1, budget=4)):
        assert do_attention(**kw) == P.ERR_INVALID_ARGUMENT, kw
    assert do_attention(mask=A, budget=1025) == P.ERR_UNSUPPORTED
    need = P.lib().pctree_paged_attention_workspace_bytes(ctypes.byref(cache()), ctypes.byref(batch()), 32)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=A + 64), dict(nb=need - 1)):
        assert do_attention(**kw) == P.ERR_WORKSPACE, kw
    big = batch(rows=1 << 30, max_rows=1 << 30, requests=60000)
    assert do_attention(b=big) == P.ERR_UNSUPPORTED


def test_compact_refusals():
    f = P.lib().pctree_compact_paged
    names = ["pool", "group_stride", "page_stride", "groups", "pages", "heads", "page_size", "slot_bytes",
             "page_table", "max_pages", "prefix_len", "accept_node", "accept_len", "requests", "budget", "max_depth"]
    ok = dict(zip(names, [A, 1 << 20, 8 * 16 * 256, 4, 10, 8, 16, 256, A, 20, A, A, A, 2, 64, 16]))

    def call(**kw):
        return f(*({**ok, **kw}[n] for n in names), None)

    for kw in (dict(pool=None), dict(page_table=None), dict(prefix_len=None), dict(accept_node=None),
               dict(accept_len=None), dict(pool=A + 8), dict(accept_node=A + 2), dict(groups=0), dict(pages=0),
               dict(heads=0), dict(page_size=0), dict(slot_bytes=8), dict(slot_bytes=24), dict(max_pages=0),
               dict(requests=0), dict(budget=0), dict(max_depth=-1), dict(group_stride=8), dict(group_stride=-16),
               dict(page_stride=8 * 16 * 256 - 16), dict(page_stride=8 * 16 * 256 + 8)):
        assert call(**kw) == P.ERR_INVALID_ARGUMENT, kw
    for kw in (dict(max_depth=64), dict(requests=70000), dict(budget=1025), dict(page_size=24, page_stride=1 << 20),
               dict(page_size=2048, page_stride=1 << 30), dict(max_pages=1 << 28), dict(groups=1 << 30)):
        assert call(**kw) == P.ERR_UNSUPPORTED, kw


def test_workspace_follows_the_split():
    ws = lambda b, h=32, c=None: P.lib().pctree_paged_attention_workspace_bytes(  # noqa: E731
        ctypes.byref(c or cache()), ctypes.byref(b), h)
    assert ws(batch(rows=1, max_rows=1, requests=1)) > 0
    assert ws(batch(rows=1 << 16, max_rows=1 << 16, requests=1)) == 0  # enough row blocks
    assert ws(batch(rows=1, max_rows=1, requests=1, max_pages=1)) == 0  # nothing to split


def test_binding_refuses_host_tensors_and_wrong_shapes():
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        P.PagedBatch(i, i, i, torch.zeros(3, 4, dtype=torch.int32), 5)
    with pytest.raises(ValueError):
        P.PagedBatch(i, i, i, i, 5)
    with pytest.raises(TypeError):
        P.PagedBatch(i, i, i, torch.zeros(3, 4), 5)
    with pytest.raises(ValueError):
        P.rope_table(10, 24, device="cpu")
    k = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        P._paged_cache(k, k, 0)
    with pytest.raises(TypeError):
        P._paged_cache(k.float(), k.float(), 0)
    with pytest.raises(ValueError):
        P.compact_paged(torch.zeros(2, 4, 2, 16, 64), i, i, torch.zeros(3, 5, dtype=torch.int32), i, 8)


def test_calls_past_a_launch_are_refused():
    wide = dict(rows=1 << 24, max_rows=1 << 24)
    assert do_append(b=batch(**wide)) == P.ERR_UNSUPPORTED
    assert do_attention(b=batch(**wide)) == P.ERR_UNSUPPORTED
    # few rows, but blocks for every request, head and run
    assert do_attention(c=cache(kv_heads=4096), b=batch(rows=8192, max_rows=8192, requests=60000),
                        heads=4096) == P.ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(group_stride=0), dict(group_stride=4096), dict(group_stride=1 << 15),
                                dict(group_stride=9 * (1 << 15)), dict(group_stride=1 << 15, page_stride=1 << 16)])
def test_compaction_refuses_groups_that_overlap(kw):
    block = 8 * 16 * 256
    a = {**dict(group_stride=10 * block, page_stride=block), **kw}
    st = P.lib().pctree_compact_paged(A, a["group_stride"], a["page_stride"], 4, 10, 8, 16, 256, A, 20, A, A, A, 2,
                                      64, 16, None)
    assert st == P.ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("x", [(1 << 32) + 2, 1 << 31, -(1 << 32) + 2])
def test_binding_refuses_sizes_past_31_bits(x):
    """A size that the C interface cannot hold is not cut to its low bits."""
    i, table = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 4, dtype=torch.int32)
    pool = torch.zeros(1, 4, 2, 16, 64)

    class Batch:
        sizes, idx, _ref = (3, 4, 2, 2), 0, ctypes.byref(batch())
    for call in (lambda: P.PagedBatch(i, i, i, table, x), lambda: P.PagedBatch(i, i, i, table, 2, x),
                 lambda: P.PagedAttention(Batch, x, 2, 128, 16), lambda: P.PagedAttention(Batch, 2, x, 128, 16),
                 lambda: P.PagedAttention(Batch, 2, 2, x, 16), lambda: P.PagedAttention(Batch, 2, 2, 128, x),
                 lambda: P.compact_paged(pool, table, i, i[:, None], i, x), lambda: P.Sampler(x, 100, device="cpu"),
                 lambda: P.Sampler(2, x, device="cpu")):
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_binding_refuses_sizes_that_are_no_integers():
    class Batch:
        sizes, idx, _ref = (3, 4, 2, 2), 0, ctypes.byref(batch())
    for call in (lambda: P.PagedAttention(Batch, 2.5, 2, 128, 16), lambda: P.Sampler(2.5, 100, device="cpu"),
                 lambda: P.compact_paged(torch.zeros(1, 4, 2, 16, 64), None, None, None, None, 8.5)):
        with pytest.raises(TypeError):
            call()


def test_pages_of_more_elements_than_64_bits_hold():
    """2^64 elements a page: larger than any page stride."""
    big = dict(kv_heads=1 << 24, page_size=1 << 20, head_dim=1 << 20, page_stride=1 << 20)
    assert do_append(c=cache(**big)) == P.ERR_INVALID_ARGUMENT
    assert do_attention(c=cache(**big)) == P.ERR_INVALID_ARGUMENT
