"""GPU parity of the verification step over a paged cache against the float64
oracle: appended rows, attention over pages, compaction in pages.

Tolerances, with u the 16-bit type's half step (2^-8 bfloat16, 2^-11 float16):

* append: float32 arithmetic and one rounding to 16 bits.  The mean of D squares,
  its root and three products are off by less than (D / 2 + 8) 2^-24 <= 72 * 2^-24
  relative, the rotation adds two products (another 3 * 2^-24), each relative to the
  magnitudes that are added: |err| <= u |z| + 2^-17 (|a| + |b|), and float16's
  smallest half step 2^-25.
* attention: each weight is rounded to 16 bits before the weighted sum, which moves
  the output by at most u * sum w |v|; the output is rounded, u |o|; scores are
  sums of D float32 products, off by at most D 2^-24 sum |q k| scale < 2^-11 for the
  sizes here (|q k| sums below 64), which moves a weight by that factor:
  |err| <= u (sum w |v| + |o|) + 2^-10 sum w |v|, and float16's 2^-25.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import pctree_paged as PO
from paper_2608_02123_amd import pctree as P
from paper_2608_02123_amd import synth

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = [torch.bfloat16, torch.float16]


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _np(t):
    return t.detach().cpu().double().numpy()


def make_batch(rng, rows, prefix, page, *, gap=0, width=None, spare=3):
    """Host arrays of a batch: rows one after the other with `gap` rows between."""
    rows, prefix = np.asarray(rows, np.int32), np.asarray(prefix, np.int32)
    need = -(-(np.maximum(rows, 0) + prefix) // page)
    W = width or max(int(need.max()), 1)
    order = rng.permutation(int(need.sum()) + spare).astype(np.int32)
    table = np.full((len(rows), W), -1, np.int32)
    at = 0
    for r, n in enumerate(np.minimum(need, W)):
        table[r, :n] = order[at:at + n]
        at += n
    start = np.cumsum(rows + gap) - rows - gap
    return {"row_start": start.astype(np.int32), "row_count": rows, "prefix_len": prefix,
            "page_table": table, "rows": max(int((rows + gap).sum()), 1),
            "max_rows": max(int(rows.max()), 1), "pages": len(order)}


def dev_batch(b):
    def up(x):
        return torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return P.PagedBatch(up(b["row_start"]), up(b["row_count"]), up(b["prefix_len"]),
                        up(b["page_table"]), b["rows"], b["max_rows"])


def tree_masks(rng, R, N, counts):
    par = np.full((R, N), -1, np.int32)
    for r in range(R):
        if counts[r] > 0:
            _, par[r], _ = synth.random_tree(rng, N, int(min(counts[r], N)), 16, 151936)
    mask = P.build_mask(torch.from_numpy(par).cuda(),
                        torch.from_numpy(np.minimum(counts, N).astype(np.int32)).cuda())
    return mask


def check_attention(b, q, k, v, out, scale, mask=None, budget=None):
    dt = out.dtype
    ref = PO.attention(b, _np(q), _np(k), _np(v), scale,
                       None if mask is None else mask.cpu().numpy(), budget)
    got = _np(out)
    u = HALF[dt]
    worst = 0.0
    for t, (o, mag) in ref.items():
        nan = ~np.isfinite(o)
        assert np.array_equal(nan, ~np.isfinite(got[t])), f"row {t}: non-finite elsewhere"
        tol = u * (mag + np.abs(o)) + 2.0 ** -10 * mag + 2.0 ** -25
        err = np.abs(got[t] - o)
        assert (err[~nan] <= tol[~nan]).all(), \
            f"row {t}: {np.nanmax((err / tol)[~nan]):.3g} of the tolerance"
        if (~nan).any():
            worst = max(worst, float((err / tol)[~nan].max()))
    return ref, worst


def run_attention(b, Hq, Hkv, D, page, dt, seed=0, tree=False, poison=True, q_scale=1.0, view=None,
                  scale=None):
    g = _gen(seed)
    rng = np.random.default_rng((seed, 5))
    T = b["rows"]

    def normal(*shape):
        return torch.randn(*shape, generator=g).to(dt).cuda()

    q = (normal(T, Hq, D).float() * q_scale).to(dt)
    shape = (b["pages"], Hkv, page, D)
    if view == "interleaved":  # pages of K and V in one pool
        pool = normal(b["pages"], 2, Hkv, page, D)
        k, v = pool[:, 0], pool[:, 1]
    else:
        k, v = normal(*shape), normal(*shape)
    if poison:  # what no request's slot holds must not matter
        used = torch.zeros(b["pages"], page, dtype=torch.bool)
        for r, t, i, prefix, n in PO.live_rows(b, page):
            for s in range(prefix + n):
                at = PO.place(b, r, s, page, b["pages"])
                if at:
                    used[at] = True
        idx = (~used).cuda()
        k.transpose(1, 2)[idx] = float("nan")
        v.transpose(1, 2)[idx] = float("nan")
    mask = budget = None
    if tree:
        budget = max(b["max_rows"], 1)
        mask = tree_masks(rng, len(b["row_count"]), budget, b["row_count"])
    marker = 3.5
    out = torch.full((T, Hq, D), marker, dtype=dt, device="cuda")
    scale = D ** -0.5 if scale is None else scale
    layer = P.PagedAttention(dev_batch(b), Hq, Hkv, D, page, scale)
    layer.workspace.fill_(0xA5)
    got = layer(q, k, v, dev_batch(b), mask=mask, out=out)
    torch.cuda.synchronize()
    assert got is out
    ref, worst = check_attention(b, q, k, v, out, scale, mask, budget)
    rest = [t for t in range(T) if t not in ref]
    if rest:
        assert (out[rest] == marker).all(), "rows of no request were written"
    print(f"[paged attention] worst {worst:.3f} of the tolerance, ws {layer.ws_bytes}", flush=True)
    return q, k, v, mask, out


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 4, 4), (128, 5, 1), (64, 14, 2)])
@pytest.mark.parametrize("page", [1, 16, 64, 256])
def test_causal_rows(dt, D, Hq, Hkv, page):
    """One token, short and odd chunks, contexts of nothing to several chunks."""
    rng = np.random.default_rng((D, Hq, page))
    b = make_batch(rng, [1, 3, 0, 33, 70, 1, 17], [0, 0, 40, 5, 63, 200, 129], page, gap=1)
    run_attention(b, Hq, Hkv, D, page, dt)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("ctx", [0, 1, 62, 63, 64, 65, 127, 128, 511, 1000, 2047])
def test_single_tokens(dt, ctx):
    rng = np.random.default_rng(ctx)
    b = make_batch(rng, [1, 1], [ctx, ctx // 2], 16)
    run_attention(b, 8, 2, 128, 16, dt, seed=ctx)


@pytest.mark.parametrize("D,Hq,Hkv,N,R", [(128, 8, 2, 64, 2), (64, 8, 8, 45, 3), (128, 5, 1, 128, 1),
                                          (128, 2, 2, 16, 5)])
@pytest.mark.parametrize("page", [16, 128])
def test_tree_rows(D, Hq, Hkv, N, R, page):
    rng = np.random.default_rng((D, N, page))
    prefix = rng.integers(0, 400, R)
    b = make_batch(rng, [N] * R, prefix, page)
    run_attention(b, Hq, Hkv, D, page, torch.bfloat16, tree=True)


@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 128), (8, 2, 64), (5, 1, 128)])
@pytest.mark.parametrize("N,counts", [(1024, [1024, 5, 701]), (1000, [31, 1000, 999])])
def test_tree_rows_of_wide_masks(Hq, Hkv, D, N, counts):
    """Masks of up to 32 words a row, counts below the budget, prefixes of no whole word."""
    rng = np.random.default_rng((N, Hq))
    b = make_batch(rng, [N] * 3, [37, 130, 3], 32)
    b["row_count"] = np.array(counts, np.int32)
    run_attention(b, Hq, Hkv, D, 32, torch.bfloat16, tree=True)


@pytest.mark.parametrize("Hq,Hkv,D,dt", [(4, 2, 128, torch.bfloat16), (6, 1, 64, torch.float16)])
def test_trees_of_few_rows_beside_many(Hq, Hkv, D, dt):
    """One masked call whose requests go to both kernels, whole and cut into runs."""
    rng = np.random.default_rng(Hq)
    rows = [1, 200, 3, 5, 0, 90, 2, 1]
    b = make_batch(rng, rows, [50, 129, 0, 2100, 10, 1700, 300, 1], 16)
    run_attention(b, Hq, Hkv, D, 16, dt, tree=True, poison=False)


def test_trees_in_padded_rows():
    """Trees of fewer nodes than the budget, in the builder's [R][N] layout."""
    rng = np.random.default_rng(3)
    N, counts = 40, np.array([40, 1, 17, 0], np.int32)
    b = make_batch(rng, [N] * 4, [100, 3, 64, 9], 16)
    b["row_count"] = counts
    run_attention(b, 8, 2, 128, 16, torch.bfloat16, tree=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,ctx", [(300, 0), (257, 321), (1, 3000), (5, 2500), (130, 1500)])
def test_longer_chunks(D, rows, ctx):
    rng = np.random.default_rng((rows, ctx))
    b = make_batch(rng, [rows], [ctx], 64)
    run_attention(b, 4, 2, D, 64, torch.bfloat16, poison=ctx < 1000)


@pytest.mark.parametrize("rows,ctx", [([1], [70001]), ([1, 1], [33000, 20]), ([40], [20000])])
def test_long_contexts(rows, ctx):
    """Runs of thousands of slots."""
    rng = np.random.default_rng(ctx[0])
    b = make_batch(rng, rows, ctx, 64)
    run_attention(b, 2, 1, 64, 64, torch.bfloat16, poison=False)


def test_mixed_rows():
    rng = np.random.default_rng(8)
    rows = [1, 1, 1, 200, 1, 1, 90, 1, 4, 1]
    b = make_batch(rng, rows, rng.integers(0, 700, len(rows)), 32)
    run_attention(b, 14, 2, 64, 32, torch.float16)


@pytest.mark.parametrize("R,Hq,Hkv,D", [(70, 4, 2, 64), (130, 2, 1, 128), (64, 6, 3, 64), (65, 5, 5, 128)])
def test_many_requests(R, Hq, Hkv, D):
    """More requests than a wave has lanes, and kv heads that do not divide the XCDs."""
    rng = np.random.default_rng((R, Hkv))
    rows = rng.choice([0, 1, 1, 1, 2, 5], R)
    rows[3] = 40
    b = make_batch(rng, rows, rng.integers(0, 300, R), 16)
    run_attention(b, Hq, Hkv, D, 16, torch.bfloat16)


@pytest.mark.parametrize("R", [64, 65, 129])
def test_many_trees(R):
    """Masked rows of more requests than a wave has lanes, in both kernels."""
    rng = np.random.default_rng(R)
    rows = rng.choice([0, 1, 4, 7], R)
    rows[R - 2] = 60
    b = make_batch(rng, rows, rng.integers(0, 200, R), 16)
    run_attention(b, 4, 2, 64, 16, torch.bfloat16, tree=True)


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (6, 3, 64), (8, 4, 128)])
def test_long_runs_beside_single_tokens(Hq, Hkv, D):
    """A mixed batch whose long requests are cut into runs, in both kernels."""
    rng = np.random.default_rng(Hkv)
    rows = [1, 40, 1, 1, 150, 2, 1, 1, 30, 1, 1]
    ctx = [2900, 2100, 3, 700, 1500, 1030, 0, 64, 10, 1999, 128]
    b = make_batch(rng, rows, ctx, 32)
    run_attention(b, Hq, Hkv, D, 32, torch.bfloat16, poison=False)


@pytest.mark.parametrize("page", [2, 4, 8, 32])
def test_long_chunk_in_small_pages(page):
    rng = np.random.default_rng(page)
    b = make_batch(rng, [200], [600], page)
    b["page_table"][0, 40 // page] = -1
    run_attention(b, 4, 2, 128, page, torch.bfloat16, poison=False)


def test_growing_scores():
    """Keys ordered so that a row's scores grow all along: the softmax reference has to
    follow, by small and by large steps."""
    rng = np.random.default_rng(31)
    for dt in DTYPES:
        for step in (0.002, 0.05, 0.5):
            b = make_batch(rng, [40], [700], 64)
            g = _gen(1)
            q = torch.ones(40, 2, 128, dtype=dt, device="cuda")
            k = torch.zeros(b["pages"], 2, 64, 128, dtype=dt, device="cuda")
            for s in range(740):
                p, o = PO.place(b, 0, s, 64, b["pages"])
                k[p, :, o] = s * step / 128
            v = torch.randn(b["pages"], 2, 64, 128, generator=g).to(dt).cuda()
            out = P.paged_attention(q, k, v, dev_batch(b), scale=1.0)
            # (|q k| sums up to 370 here: the score bound of the file's head, times 8)
            ref = PO.attention(b, _np(q), _np(k), _np(v), 1.0)
            for t, (o, mag) in ref.items():
                tol = HALF[dt] * (mag + np.abs(o)) + 2.0 ** -7 * mag + 2.0 ** -25
                assert (np.abs(_np(out[t]) - o) <= tol).all(), (dt, step, t)


def test_rows_that_admit_nothing_are_zero():
    """An empty mask row without a prefix, and a request whose pages are all missing."""
    rng = np.random.default_rng(4)
    N = 20
    b = make_batch(rng, [N, N, N], [0, 50, 30], 16)
    b["page_table"][2] = -1
    q, k, v, mask, _ = run_attention(b, 4, 2, 128, 16, torch.bfloat16, tree=True)
    mask = mask.clone()
    mask[0, 5:9] = 0
    mask[1, 3] = 0
    bt = dev_batch(b)
    out = P.paged_attention(q, k, v, bt, mask=mask)
    check_attention(b, q, k, v, out, 128 ** -0.5, mask, N)
    t0 = int(b["row_start"][0])
    assert (out[t0 + 5:t0 + 9] == 0).all() and (out[int(b["row_start"][2]):] == 0).all()


@pytest.mark.parametrize("rows", [1, 7, 40])
@pytest.mark.parametrize("what", [-1, -7, 10 ** 6])
def test_missing_pages(rows, what):
    """Pages that do not exist, in the prefix and among the new rows: their slots are
    admitted by nobody, and what the pool's first page holds does not leak in."""
    rng = np.random.default_rng((rows, abs(what)))
    b = make_batch(rng, [rows, rows], [200, 90], 16)
    b["page_table"][0, 3] = what
    b["page_table"][1, 0] = what
    b["page_table"][1, -1] = what
    q, k, v, _, _ = run_attention(b, 8, 2, 128, 16, torch.bfloat16)
    first = [p for p in range(b["pages"]) if p not in b["page_table"]][0]
    assert first >= 0
    b2 = {**b, "page_table": np.where(b["page_table"] == 0, what, b["page_table"])}
    k[0], v[0] = float("inf"), float("nan")  # page 0 belongs to nobody now
    out = P.paged_attention(q, k, v, dev_batch(b2))
    check_attention(b2, q, k, v, out, 128 ** -0.5)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_masked_slots_hold(dt, bad):
    """Infinite and NaN keys and values at slots that only some rows admit reach those
    rows only."""
    rng = np.random.default_rng(11)
    N, D, page = 50, 128, 16
    b = make_batch(rng, [N, N], [70, 0], page)
    for tree in (False, True):
        q, k, v, mask, _ = run_attention(b, 4, 2, D, page, dt, tree=tree, poison=False)
        at = PO.place(b, 0, 70 + 20, page, b["pages"])
        v[at[0], 1, at[1], 37] = bad
        at = PO.place(b, 1, 33, page, b["pages"])
        v[at[0], 0, at[1]] = bad
        k2 = k.clone()
        k2[at[0], 0, at[1], 5] = float("nan")  # (its row is NaN for whoever admits it)
        for kk in (k, k2):
            out = P.paged_attention(q, kk, v, dev_batch(b), mask=mask)
            ref = PO.attention(b, _np(q), _np(kk), _np(v), D ** -0.5,
                               None if mask is None else mask.cpu().numpy(), N)
            got = _np(out)
            for t, (o, _) in ref.items():
                assert np.array_equal(np.isfinite(o), np.isfinite(got[t])), t
                ok = np.isfinite(o)
                assert np.abs(got[t] - o)[ok].max(initial=0) < 0.05


@pytest.mark.parametrize("n", [6, 50])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_masked_slots_hold_to_the_tolerance(n, bad):
    """As above, in requests of few rows and of many, to the tolerance of the file's head:
    nothing of such a slot reaches the rows that do not admit it."""
    rng = np.random.default_rng(n)
    D, page, prefix = 128, 16, 70
    b = make_batch(rng, [n, n, n], [prefix, 0, 300], page)
    for dt in DTYPES:
        for tree in (False, True):
            q, k, v, mask, _ = run_attention(b, 4, 2, D, page, dt, tree=tree, poison=False)
            for j in (1, n // 2, n - 1):
                at = PO.place(b, 0, prefix + j, page, b["pages"])
                v[at[0], 1, at[1], 5 * j:] = bad
            at = PO.place(b, 1, n // 2, page, b["pages"])
            v[at[0], 0, at[1]] = bad
            k[at[0], 1, at[1], 7] = bad
            at = PO.place(b, 2, 300 + n - 1, page, b["pages"])
            k[at[0], :, at[1]] = float("nan")
            v[at[0], :, at[1]] = bad
            out = P.paged_attention(q, k, v, dev_batch(b), mask=mask)
            check_attention(b, q, k, v, out, D ** -0.5, mask, n)


def test_clamped_batches():
    """Starts, counts and prefixes out of range, and rows past the cache's capacity."""
    rng = np.random.default_rng(12)
    b = make_batch(rng, [10, 10, 10, 10, 10], [20, 20, 20, 20, 20], 16, width=2)
    b["row_start"][0] = -1
    b["row_count"][1] = 400      # clamped to max_rows
    b["row_start"][2] = b["rows"]
    b["row_count"][3] = -5
    b["prefix_len"][4] = 27      # the last five rows have no slot
    b["row_start"][1] = 0        # (rows 0.. 9, the first request has none)
    run_attention(b, 4, 2, 128, 16, torch.bfloat16)
    b["prefix_len"][4] = 1 << 30
    b["prefix_len"][1] = -3
    run_attention(b, 4, 2, 128, 16, torch.bfloat16)


def test_flat_scores():
    rng = np.random.default_rng(14)
    b = make_batch(rng, [30, 1], [500, 800], 64)
    for dt in DTYPES:
        run_attention(b, 4, 2, 128, 64, dt, scale=0.01, poison=False)


def test_pages_of_a_larger_pool():
    rng = np.random.default_rng(15)
    b = make_batch(rng, [20, 1], [100, 300], 16)
    run_attention(b, 8, 2, 128, 16, torch.bfloat16, view="interleaved")


def test_offsets_past_32_bits():
    """A pool of more than 2^32 elements; the request's pages lie at its end."""
    pages, Hkv, page, D = 34000, 8, 128, 128
    k = torch.empty(pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty(pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 1 << 32
    g = _gen(1)
    table = np.array([[pages - 1, pages - 2, 7]], np.int32)
    b = {"row_start": np.zeros(1, np.int32), "row_count": np.array([5], np.int32),
         "prefix_len": np.array([290], np.int32), "page_table": table, "rows": 5, "max_rows": 5,
         "pages": pages}
    new = [torch.randn(5, h, D, generator=g).to(torch.bfloat16).cuda() for h in (16, 8, 8)]
    for c in (k, v):
        for p in table[0]:
            c[int(p)] = torch.randn(Hkv, page, D, generator=g).to(torch.bfloat16).cuda()
    bt = dev_batch(b)
    q = P.append_paged(bt, k, v, new[1], new[2], q=new[0])
    assert torch.equal(q, new[0])  # (neither norm nor rotation)
    out = P.paged_attention(q, k, v, bt)
    small = {p: i for i, p in enumerate(table[0])}
    ks, vs = (torch.stack([c[int(p)] for p in table[0]]) for c in (k, v))
    for i in range(5):
        s = 290 + i
        assert torch.equal(ks[s // page, :, s % page], new[1][i])
    b2 = {**b, "page_table": np.array([[small[p] for p in table[0]]], np.int32), "pages": 3}
    check_attention(b2, q, ks, vs, out, D ** -0.5)


# ---------------------------------------------------------------------------
# appended rows
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("D,rot,Hq,Hkv,page", [(128, 128, 8, 2, 16), (64, 64, 3, 3, 1), (128, 64, 5, 1, 64),
                                               (64, 16, 14, 2, 32), (128, 0, 4, 4, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_append(dt, D, rot, Hq, Hkv, page, interleaved, norm):
    rng = np.random.default_rng((D, rot, Hq))
    g = _gen(D + rot)
    b = make_batch(rng, [1, 5, 0, 33, 2], [0, 7, 3, 100, 31], page, gap=2)
    b["page_table"][3, 1] = -1 if page < 64 else b["page_table"][3, 1]
    T = b["rows"]
    fused = (torch.randn(T, (Hq + 2 * Hkv) * D, generator=g) * 3).to(dt).cuda()
    q, k, v = (x.unflatten(1, (-1, D)) for x in fused.split([Hq * D, Hkv * D, Hkv * D], 1))
    kc = torch.full((b["pages"], Hkv, page, D), 9.0, dtype=dt, device="cuda")
    vc = torch.full_like(kc, -9.0)
    wq, wk = ((1 + 0.3 * torch.randn(D, generator=g)).to(dt).cuda() if norm else None for _ in "qk")
    rope = P.rope_table(150, rot, theta=1e4) if rot else None
    pos = torch.from_numpy(rng.integers(-3, 160, T).astype(np.int32)).cuda()
    for position in (None, pos):
        q_out = torch.full((T, Hq, D), 5.0, dtype=dt, device="cuda")
        kc.fill_(9.0), vc.fill_(-9.0)
        got = P.append_paged(dev_batch(b), kc, vc, k, v, q=q, q_norm=wq, k_norm=wk, eps=1e-5, rope=rope,
                             interleaved=interleaved, position=position, q_out=q_out)
        assert got is q_out
        qo, ko, vo = PO.append(b, _np(kc), _np(vc), _np(q), _np(k), _np(v),
                               None if wq is None else _np(wq), None if wk is None else _np(wk), 1e-5,
                               None if rope is None else _np(rope), interleaved,
                               None if position is None else position.cpu().numpy())
        u = HALF[dt]

        def near(x, refs):
            for h, (z, mag) in enumerate(refs):
                assert (np.abs(x[h] - z) <= u * np.abs(z) + 2.0 ** -17 * mag + 2.0 ** -25).all()

        gq, gk, gv = _np(q_out), _np(kc), _np(vc)
        for t in range(T):
            if t in qo:
                near(gq[t], qo[t])
            else:
                assert (gq[t] == 5.0).all()
        for p in range(b["pages"]):
            for o in range(page):
                if (p, o) in ko:
                    near(gk[p, :, o], ko[(p, o)])
                    assert np.array_equal(gv[p, :, o], vo[(p, o)])
                else:
                    assert (gk[p, :, o] == 9.0).all() and (gv[p, :, o] == -9.0).all()


def test_append_rows_of_many_requests():
    """Every row finds its request among more than a wave has lanes."""
    rng = np.random.default_rng(6)
    R, page, D = 150, 16, 64
    b = make_batch(rng, rng.choice([0, 1, 3], R), rng.integers(0, 60, R), page, gap=1)
    k, v = (torch.randn(b["rows"], 2, D, generator=_gen(i)).to(torch.bfloat16).cuda() for i in (1, 2))
    kc, vc = (torch.full((b["pages"], 2, page, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    P.append_paged(dev_batch(b), kc, vc, k, v)
    kw, vw = torch.full_like(kc, 9.0), torch.full_like(vc, 9.0)
    for r, t, i, prefix, n in PO.live_rows(b, page):
        p, o = PO.place(b, r, prefix + i, page, b["pages"])
        kw[p, :, o], vw[p, :, o] = k[t], v[t]
    assert torch.equal(kc, kw) and torch.equal(vc, vw)


def test_append_many_rows_in_place():
    """Enough rows for one wave each, q written over itself, keys only."""
    rng = np.random.default_rng(2)
    b = make_batch(rng, [2100, 300], [10, 700], 64)
    g = _gen(9)
    D, Hq, Hkv = 128, 6, 2
    q, k, v = ((torch.randn(b["rows"], h, D, generator=g) * 2).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
    w = (1 + 0.2 * torch.randn(D, generator=g)).to(torch.bfloat16).cuda()
    rope = P.rope_table(3000, D, theta=1e6)
    caches = [torch.zeros(b["pages"], Hkv, 64, D, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    a = P.append_paged(dev_batch(b), caches[0], caches[1], k, v, q=q, q_norm=w, k_norm=w, rope=rope)
    q2 = q.clone()
    P.append_paged(dev_batch(b), caches[2], caches[3], k, v, q=q2, q_norm=w, k_norm=w, rope=rope, q_out=q2)
    assert torch.equal(a, q2) and torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
    caches[2].zero_(), caches[3].zero_()
    assert P.append_paged(dev_batch(b), caches[2], caches[3], k, v, k_norm=w, rope=rope) is None
    assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
    qo, ko, _ = PO.append({**b, "row_count": np.array([40, 0], np.int32)}, _np(caches[0]), _np(caches[1]), _np(q),
                          _np(k), _np(v), _np(w), _np(w), 1e-6, _np(rope), False, None)
    for t in qo:
        for h in range(Hq):
            z, mag = qo[t][h]
            assert (np.abs(_np(a[t, h]) - z) <= 2.0 ** -8 * np.abs(z) + 2.0 ** -17 * mag).all()


@pytest.mark.parametrize("T", [1300, 3500, 9000])
@pytest.mark.parametrize("D", [64, 128])
def test_append_of_many_rows_is_that_of_few(T, D):
    """However many waves share a row: the same bits as 100 rows a call."""
    Hq, Hkv, page = 12, 4, 32
    g = _gen(T + D)
    b = make_batch(np.random.default_rng(T), [T], [17], page)
    q, k, v = ((torch.randn(T, h, D, generator=g) * 2).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
    w = (1 + 0.2 * torch.randn(D, generator=g)).to(torch.bfloat16).cuda()
    rope = P.rope_table(T + 20, D)
    caches = [torch.zeros(b["pages"], Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    out = P.append_paged(dev_batch(b), caches[0], caches[1], k, v, q=q, q_norm=w, k_norm=w, rope=rope)
    for t0 in range(0, T, 100):
        n = min(100, T - t0)
        few = dev_batch({**b, "rows": n, "row_count": np.array([n], np.int32),
                         "prefix_len": np.array([17 + t0], np.int32), "max_rows": n})
        part = P.append_paged(few, caches[2], caches[3], k[t0:t0 + n], v[t0:t0 + n], q=q[t0:t0 + n], q_norm=w,
                              k_norm=w, rope=rope)
        assert torch.equal(out[t0:t0 + n], part), t0
    assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])


def test_far_positions():
    """Rotation angles of positions past 2^20 keep their fractions of a turn."""
    rope = P.rope_table((1 << 20) + 5, 64, theta=1e4)
    i = np.arange(32)
    angle = np.float64((1 << 20) + 3) * 1e4 ** (-2.0 * i / 64)
    want = np.concatenate([np.cos(angle), np.sin(angle)])
    assert np.abs(_np(rope[(1 << 20) + 3]) - want).max() < 1e-7


# ---------------------------------------------------------------------------
# compaction
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("page", [1, 16, 64])
def test_compact(page):
    rng = np.random.default_rng(page)
    R, N, W = 9, 40, 17
    prefix = rng.integers(0, 90, R).astype(np.int32)
    b = make_batch(rng, [N] * R, prefix, page)
    table = b["page_table"]
    node = np.full((R, W), -1, np.int32)
    alen = np.zeros(R, np.int32)
    for r in range(R):
        n = int(rng.integers(1, W + 1))
        node[r, :n] = np.concatenate([[0], np.sort(rng.choice(np.arange(1, N), n - 1, replace=False))])
        alen[r] = n - 1
    alen[1] = -1
    alen[2] = W
    node[3, 0], alen[3] = N, 0
    node[4, :3], alen[4] = (0, 7, 7), 2
    node[5, :3], alen[5] = (0, 2, 5), 2
    table[5, (prefix[5] + 5) // page] = -2
    prefix[6] = table.shape[1] * page - 1
    node[7, :4], alen[7] = (0, 1, 2, 3), 3
    pool = torch.randn(3, b["pages"], 2, page, 64, generator=_gen(3)).to(torch.bfloat16).cuda()
    want = PO.compact(_np(pool), table, prefix, node, alen, N)

    def up(x):
        return torch.from_numpy(x).cuda()
    got = P.compact_paged(pool, up(table), up(prefix), up(node), up(alen), N)
    assert got is pool and np.array_equal(_np(pool), want)


@pytest.mark.parametrize("n", [1, 2, 9, 17, 63])
def test_compact_of_groups_inside_pages(n):
    """Keys and values of a page side by side, paths of one batch of moves and of several."""
    rng = np.random.default_rng(n)
    R, N, page = 3, 80, 16
    prefix = rng.integers(0, 50, R).astype(np.int32)
    b = make_batch(rng, [N] * R, prefix, page)
    node = np.stack([np.concatenate([[0], np.sort(rng.choice(np.arange(1, N), n, replace=False))])
                     for _ in range(R)]).astype(np.int32)
    alen = np.array([n, n, n - 1], np.int32)
    pool = torch.randn(b["pages"], 2, 2, page, 8, generator=_gen(n)).to(torch.bfloat16).cuda().transpose(0, 1)
    want = PO.compact(_np(pool), b["page_table"], prefix, node, alen, N)

    def up(x):
        return torch.from_numpy(x).cuda()
    P.compact_paged(pool, up(b["page_table"]), up(prefix), up(node), up(alen), N)
    assert np.array_equal(_np(pool), want)


def test_compact_checks_the_nodes_that_stay():
    """An accepted node that would stay where it is, on a page that does not exist: its
    request is left untouched."""
    page, N, W = 4, 12, 6
    table = np.array([[0, 1, 2, 3], [4, -1, 5, 6], [9, 7, 8, 99]], np.int32)
    prefix = np.array([3, 4, 0], np.int32)
    node = np.array([[0, 1, 4, 6, 9, -1], [0, 1, 4, 6, 7, -1], [0, 1, 2, 3, 9, -1]], np.int32)
    alen = np.array([4, 4, 4], np.int32)
    table[2, 0] = 10  # (of 10 pages: none)
    pool = torch.randn(2, 10, 3, page, 8, generator=_gen(4)).to(torch.bfloat16).cuda()
    before = pool.clone()
    want = PO.compact(_np(pool), table, prefix, node, alen, N)

    def up(x):
        return torch.from_numpy(x).cuda()
    P.compact_paged(pool, up(table), up(prefix), up(node), up(alen), N)
    assert np.array_equal(_np(pool), want)
    assert torch.equal(pool[:, 4:], before[:, 4:]) and not torch.equal(pool, before)


# ---------------------------------------------------------------------------
# streams, graphs
# ---------------------------------------------------------------------------

def _small_step():
    rng = np.random.default_rng(21)
    N, page = 32, 16
    b = make_batch(rng, [N, N], [300, 45], page)
    g = _gen(5)
    t = {n: (torch.randn(b["rows"], h, 128, generator=g)).to(torch.bfloat16).cuda()
         for n, h in (("q", 8), ("k", 2), ("v", 2))}
    kc = torch.randn(b["pages"], 2, page, 128, generator=g).to(torch.bfloat16).cuda()
    vc = torch.randn(b["pages"], 2, page, 128, generator=g).to(torch.bfloat16).cuda()
    mask = tree_masks(rng, 2, N, np.array([N, N]))
    rope = P.rope_table(500, 128)
    bt = dev_batch(b)
    layer = P.PagedAttention(bt, 8, 2, 128, page)
    assert layer.ws_bytes > 0  # (split runs: the workspace is in play)
    q_out, out = torch.empty_like(t["q"]), torch.empty_like(t["q"])

    def step(stream=None):
        P.append_paged(bt, kc, vc, t["k"], t["v"], q=t["q"], rope=rope, q_out=q_out, stream=stream)
        layer(q_out, kc, vc, bt, mask=mask, out=out, stream=stream)

    return step, t, kc, vc, out, bt


def test_another_stream():
    step, t, kc, vc, out, _ = _small_step()
    step()
    torch.cuda.synchronize()
    want = out.clone()
    out.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("passed", [True, False])
def test_a_workspace_outlives_its_object_on_another_stream(passed):
    """Freed while another stream's call is still queued, it has no new owner yet."""
    b = make_batch(np.random.default_rng(3), [1, 1], [2000, 900], 16)
    q = torch.randn(2, 8, 128).to(torch.bfloat16).cuda()
    kc = torch.randn(b["pages"], 2, 16, 128).to(torch.bfloat16).cuda()
    x, u = torch.randn(2, 30000).cuda(), torch.rand(2).cuda()
    bt, s = dev_batch(b), torch.cuda.Stream()
    torch.cuda.synchronize()
    for make in (lambda: P.PagedAttention(bt, 8, 2, 128, 16), lambda: P.Sampler(2, 30000)):
        layer = make()
        ptr, n = layer.workspace.data_ptr(), layer.workspace.numel()
        s.wait_stream(torch.cuda.current_stream())
        args = (q, kc, kc, bt) if isinstance(layer, P.PagedAttention) else (x, u)
        with torch.cuda.stream(s):
            torch.cuda._sleep(200_000_000)  # about 0.1 s
            if not passed:
                layer(*args)
        if passed:
            layer(*args, stream=s)
        del layer
        again = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(3)]
        assert not s.query(), "the other stream's work has ended"
        assert ptr not in [t.data_ptr() for t in again]
        s.synchronize()


def test_graph_replays():
    """A captured step, replayed with other inputs, lengths and work between."""
    step, t, kc, vc, out, bt = _small_step()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    prefix = bt._keep[2]
    for i in range(4):
        t["q"].mul_(-0.5), t["k"].neg_()
        prefix.sub_(7 * i)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, kc, vc)]
        out.zero_()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, kc, vc)):
            assert torch.equal(a, b), f"replay {i}"


def test_a_verification_step_as_it_is_used():
    """A drafted tree through the target's step and on: rows appended with norm and
    rotation, tree attention over pages, a token sampled at every node, greedy walk,
    compaction; then the next token's row over the compacted pages.  The pages must
    then be those of a plain decoding of the accepted tokens."""
    from paper_2608_02123_amd.synth import CONFIGS, make_inputs
    w = CONFIGS["tiny"]
    builder = P.TreeBuilder(w.V, w.B, w.N, w.k, w.r, w.R, P.F32)
    inp = P.device_inputs(make_inputs(w))
    tree = builder.run(**inp, check=True)
    N, Hq, Hkv, D, page = w.N, 8, 2, 128, 16
    g = _gen(77)
    emb = torch.randn(w.V, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16).cuda()
    head = (torch.randn(Hq * D, w.V, generator=g) * 0.3).cuda()
    wn = (1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16).cuda()
    rope = P.rope_table(1200, D)
    prefix = int(inp["prefix_len"][0])
    pages = (prefix + N + page) // page + 2
    table = torch.randperm(pages, generator=g).to(torch.int32)[None].cuda()
    pool = torch.randn(2, pages, Hkv, page, D, generator=g).to(torch.bfloat16).cuda()

    def one(x):
        return torch.tensor([x], dtype=torch.int32, device="cuda")

    def rows(tokens):
        q, k, v = emb[tokens.long()].split([Hq * D, Hkv * D, Hkv * D], 1)
        return [x.unflatten(1, (-1, D)) for x in (q, k, v)]

    bt = P.PagedBatch(one(0), tree["count"], inp["prefix_len"], table, N)
    q, k, v = rows(tree["token"][0])
    q = P.append_paged(bt, pool[0], pool[1], k, v, q=q, q_norm=wn, k_norm=wn, rope=rope, position=tree["position"][0])
    out = P.PagedAttention(bt, Hq, Hkv, D, page)(q, pool[0], pool[1], bt, mask=tree["mask"])
    logits = out.float().flatten(1) @ head
    # (so that something is accepted: each node's target likes one of its children)
    par = tree["parent"][0].cpu().numpy()
    for i in range(1, N):
        logits[par[i], int(tree["token"][0, i])] += 40.0 + i
    u = torch.rand(N, generator=g).cuda()
    target, _ = P.sample(logits, u, top_k=torch.full((N,), 20, dtype=torch.int32, device="cuda"))
    rws, nrows = P.build_retrieve(tree["parent"], tree["count"], w.B)
    acc = P.accept_greedy(tree["token"], rws, nrows, target[None])
    P.compact_paged(pool, table, inp["prefix_len"], acc["accept_node"], acc["accept_len"], N)
    n = int(acc["accept_len"][0])
    assert n > 0
    nodes = acc["accept_node"][0, :n + 1].long()
    tokens = tree["token"][0][nodes]
    # the accepted tokens, decoded one after the other into fresh pages
    plain = pool.clone()
    for s in range(n + 1):
        p, o = int(table[0, (prefix + s) // page]), (prefix + s) % page
        plain[:, p, :, o] = 0
    for s in range(n + 1):
        b1 = P.PagedBatch(one(0), one(1), one(prefix + s), table, 1)
        _, k, v = rows(tokens[s:s + 1])
        P.append_paged(b1, plain[0], plain[1], k, v, k_norm=wn, rope=rope)
    assert torch.equal(plain, pool)
    # the bonus token's row
    b1 = P.PagedBatch(one(0), one(1), one(prefix + n + 1), table, 1)
    q, k, v = rows(acc["bonus"])
    q = P.append_paged(b1, pool[0], pool[1], k, v, q=q, q_norm=wn, k_norm=wn, rope=rope)
    out = P.paged_attention(q, pool[0], pool[1], b1)
    host = {"row_start": np.array([0]), "row_count": np.array([1]), "prefix_len": np.array([prefix + n + 1]),
            "page_table": table.cpu().numpy(), "rows": 1, "max_rows": 1, "pages": pages}
    check_attention(host, q, pool[0], pool[1], out, D ** -0.5)


def test_results_repeat():
    step, t, kc, vc, out, _ = _small_step()
    step()
    want = out.clone()
    for _ in range(3):
        step()
        assert torch.equal(out, want)
