"""GPU parity of a paged cache in 8 bits against the float64 oracle: appended rows, attention
over held values, compaction.

Tolerances:

* values, scales of values, rescaled rows and compaction: every step is exact but the one
  rounding to e4m3, so bytes are equal (but for the two that are NaN, whose sign is nothing).
* keys: float32 arithmetic before the rounding, off by d = 2^-17 (|a| + |b|) (the append of
  16-bit pages), then half a step of e4m3: |err| <= d + max(2^-4 (|z| + d), 2^-10 scale), 2^-10
  of the scale being half a step under its normal numbers.  A block's scale is that of a largest
  magnitude within d of the exact one.
* attention: as over 16-bit pages (weights and output rounded to 16 bits); held values are
  exact in bfloat16, and in float16 within 2^-25, of which a weighted mean keeps no more.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import pctree_held as HO
from oracle import pctree_paged as PO
from paper_2608_02123_amd import pctree as P
from test_gpu_paged import DTYPES, HALF, _gen, _np, check_attention, dev_batch, make_batch, tree_masks

pytestmark = pytest.mark.gpu

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy()


def same(a, b):
    """Whether held bytes stand for the same numbers, NaN for NaN."""
    return bool(((a == b) | ((a & 127 == 127) & (b & 127 == 127))).all())


def _held(pages, scale):
    """Device tensors of host bytes."""
    def up(a):
        return torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return up(pages).view(E4M3), up(scale).view(E8M0)


def random_pages(rng, *shape, block, low=118, high=124):
    """Held bytes of normal values [..., slots, D] under random scales of blocks."""
    scale = rng.integers(low, high + 1, (*shape[:-2], shape[-2] // block)).astype(np.uint8)
    z = np.clip(rng.standard_normal(shape) * 128.0, -448, 448)
    return HO.hold(z, 127), scale


def random_held(rng, pages, Hkv, page, D, block, scale=None):
    k, ks = random_pages(rng, pages, Hkv, page, D, block=block, low=119, high=121)
    v, vs = random_pages(rng, pages, Hkv, page, D, block=block)
    return k, ks, v, vs


def run_attention(b, Hq, Hkv, D, page, block, dt, seed=0, tree=False, poison=True, budget=None, mask=None, spoil=None):
    rng = np.random.default_rng((seed, 5))
    T = b["rows"]
    q = torch.randn(T, Hq, D, generator=_gen(seed)).to(dt).cuda()
    k, ks, v, vs = random_held(rng, b["pages"], Hkv, page, D, block)
    if poison:  # what no request's slot holds must not matter
        used = np.zeros((b["pages"], page), bool)
        for r, t, i, prefix, n in PO.live_rows(b, page):
            for s in range(prefix + n):
                at = PO.place(b, r, s, page, b["pages"])
                if at:
                    used[at] = True
        idx = ~used
        k.transpose(0, 2, 1, 3)[idx] = 0x7f
        v.transpose(0, 2, 1, 3)[idx] = 0xff
        whole = idx.reshape(b["pages"], page // block, block).all(-1)
        ks.transpose(0, 2, 1)[whole] = 255
        vs.transpose(0, 2, 1)[whole] = 255
    if spoil:
        spoil(k, ks, v, vs)
    if tree and mask is None:
        budget = max(b["max_rows"], 1)
        mask = tree_masks(rng, len(b["row_count"]), budget, b["row_count"])
    kd, ksd = _held(k, ks)
    vd, vsd = _held(v, vs)
    out = torch.full((T, Hq, D), 3.5, dtype=dt, device="cuda")
    layer = P.PagedAttention(dev_batch(b), Hq, Hkv, D, page)
    layer.workspace.fill_(0xA5)
    assert layer(q, kd, vd, dev_batch(b), mask=mask, out=out, k_scale=ksd, v_scale=vsd) is out
    torch.cuda.synchronize()
    kv, vv = (torch.from_numpy(HO.values(x, s)) for x, s in ((k, ks), (v, vs)))
    ref, worst = check_attention(b, q, kv, vv, out, D ** -0.5, mask, budget)
    rest = [t for t in range(T) if t not in ref]
    if rest:
        assert (out[rest] == 3.5).all(), "rows of no request were written"
    print(f"[held attention] worst {worst:.3f} of the tolerance", flush=True)
    return q, kd, ksd, vd, vsd, mask, out


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 4, 4), (128, 5, 1), (64, 14, 2)])
@pytest.mark.parametrize("page,block", [(8, 8), (16, 16), (64, 8), (64, 64), (256, 32)])
def test_causal_rows(dt, D, Hq, Hkv, page, block):
    """One token, short and odd chunks, contexts of nothing to several chunks."""
    rng = np.random.default_rng((D, Hq, page))
    b = make_batch(rng, [1, 3, 0, 33, 70, 1, 17], [0, 0, 40, 5, 63, 200, 129], page, gap=1)
    run_attention(b, Hq, Hkv, D, page, block, dt)


@pytest.mark.parametrize("dt,D", [(torch.bfloat16, 128), (torch.float16, 64)])
@pytest.mark.parametrize("ctx", [0, 1, 7, 8, 62, 63, 64, 65, 127, 128, 255, 256, 257, 511, 1000, 2047])
def test_single_tokens(dt, D, ctx):
    rng = np.random.default_rng(ctx)
    b = make_batch(rng, [1, 1], [ctx, ctx // 2], 16)
    run_attention(b, 8, 2, D, 16, 8, dt, seed=ctx)


@pytest.mark.parametrize("D,Hq,Hkv,N,R", [(128, 8, 2, 64, 2), (64, 8, 8, 45, 3), (128, 5, 1, 128, 1), (128, 2, 2, 16, 5)])
@pytest.mark.parametrize("page,block", [(16, 8), (128, 64)])
def test_tree_rows(D, Hq, Hkv, N, R, page, block):
    rng = np.random.default_rng((D, N, page))
    b = make_batch(rng, [N] * R, rng.integers(0, 400, R), page)
    run_attention(b, Hq, Hkv, D, page, block, torch.bfloat16, tree=True)


@pytest.mark.parametrize("Hq,Hkv,D,dt", [(4, 2, 128, torch.bfloat16), (6, 1, 64, torch.float16)])
def test_trees_of_few_rows_beside_many(Hq, Hkv, D, dt):
    """One masked call whose requests go to both kernels, whole and cut into runs."""
    rng = np.random.default_rng(Hq)
    b = make_batch(rng, [1, 200, 3, 5, 0, 90, 2, 1], [50, 129, 0, 2100, 10, 1700, 300, 1], 16)
    run_attention(b, Hq, Hkv, D, 16, 16, dt, tree=True, poison=False)


def test_wide_masks_and_padded_rows():
    rng = np.random.default_rng(3)
    b = make_batch(rng, [1000] * 3, [37, 130, 3], 32)
    b["row_count"] = np.array([31, 1000, 0], np.int32)
    run_attention(b, 4, 2, 64, 32, 32, torch.bfloat16, tree=True)


@pytest.mark.parametrize("D,dt", [(64, torch.float16), (128, torch.bfloat16)])
@pytest.mark.parametrize("rows,ctx", [(300, 0), (257, 321), (1, 3000), (5, 2500), (130, 1500)])
def test_longer_chunks(D, dt, rows, ctx):
    b = make_batch(np.random.default_rng((rows, ctx)), [rows], [ctx], 64)
    run_attention(b, 6, 2, D, 64, 32, dt, poison=False)


@pytest.mark.parametrize("Hq,Hkv,D", [(64, 1, 128), (40, 1, 64), (16, 1, 128), (33, 3, 64), (7, 7, 128)])
def test_groups_of_heads(Hq, Hkv, D):
    """Single tokens and short chunks whose heads alone are more rows than the small kernel's."""
    rng = np.random.default_rng(Hq)
    b = make_batch(rng, [1, 2, 1, 9], [700, 90, 0, 31], 32)
    run_attention(b, Hq, Hkv, D, 32, 32, torch.bfloat16)


def test_large_pages():
    rng = np.random.default_rng(77)
    b = make_batch(rng, [1, 100, 3], [1500, 1000, 5], 1024)
    run_attention(b, 4, 2, 64, 1024, 64, torch.float16)
    run_append(b, 4, 3, 64, 1024, 64, torch.float16)


def test_many_requests():
    """More than 64, which are not ordered by length."""
    rng = np.random.default_rng(8)
    rows = rng.integers(0, 5, 90)
    rows[3], rows[77] = 60, 41
    b = make_batch(rng, rows, rng.integers(0, 300, 90), 16, gap=1)
    run_attention(b, 4, 2, 64, 16, 16, torch.bfloat16, poison=False)


@pytest.mark.parametrize("rows,ctx", [(1, 700), (90, 300)])
def test_pages_that_are_none(rows, ctx):
    """Entries of the table outside the pool, inside a run and at a request's start; one request
    of nothing else, whose rows are zero."""
    rng = np.random.default_rng(rows)
    b = make_batch(rng, [rows, rows, rows], [ctx, ctx, ctx], 16)
    b["page_table"][0, ::3] = -1
    b["page_table"][1, :9] = b["pages"]
    b["page_table"][2] = -5
    out = run_attention(b, 8, 2, 128, 16, 16, torch.bfloat16)[-1]
    assert (out[2 * rows:] == 0).all()


def test_rows_whose_mask_leaves_nothing():
    rng = np.random.default_rng(1)
    for N in (8, 100):
        b = make_batch(rng, [N, N], [0, 20], 16)
        mask = tree_masks(rng, 2, N, b["row_count"])
        mask[:, 3] = 0
        out = run_attention(b, 8, 2, 128, 16, 8, torch.bfloat16, mask=mask, budget=N)[-1]
        assert (out[3] == 0).all() and (out[N + 3] != 0).any()


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("rows,ctx,tree", [(1, 200, False), (3, 200, False), (100, 70, False), (60, 150, True)])
def test_nan_values_reach_the_rows_that_admit_them(dt, rows, ctx, tree):
    """NaN among the held values of the prefix and of the new rows; and scales that take
    float16's values past its range."""
    rng = np.random.default_rng(rows)
    b = make_batch(rng, [rows, rows], [ctx, ctx], 16)

    def spoil(k, ks, v, vs):
        for s, d in ((5, 3), (ctx + rows - 1, 17), (ctx + rows // 2, 64)):
            page, off = PO.place(b, 0, s, 16, b["pages"])
            v[page, 1, off, d] = 0x7f
        if dt == torch.float16 and rows > 1:
            page, off = PO.place(b, 1, ctx + rows - 1, 16, b["pages"])
            v[page, 0, off, 9], vs[page, 0, off // 8] = 0x7e, 140  # 448 * 2^13
            v[page, 0, off - off % 8:off, :] = 0
            v[page, 0, off, :9] = v[page, 0, off, 10:] = 0
    if dt == torch.float16 and rows > 1:
        # (what float16 rounds to infinity counts as infinite)
        orig = HO.values
        try:
            HO.values = lambda x, s: _half_range(orig(x, s))
            run_attention(b, 8, 2, 128, 16, 8, dt, tree=tree, spoil=spoil, poison=False)
        finally:
            HO.values = orig
    else:
        run_attention(b, 8, 2, 128, 16, 8, dt, tree=tree, spoil=spoil, poison=False)


def _half_range(v):
    return np.where(np.abs(v) > 65519.0, np.copysign(np.inf, v), v)


def test_scales_at_their_ends():
    """The smallest and the largest scales that are written: every value is there in bfloat16."""
    b = make_batch(np.random.default_rng(0), [1, 70], [90, 20], 16)

    def spoil(k, ks, v, vs):
        vs[:, 0], vs[:, 1] = 16, 20
    run_attention(b, 4, 2, 128, 16, 16, torch.bfloat16, spoil=spoil)

    def spoil2(k, ks, v, vs):
        vs[:] = 230
    run_attention(b, 4, 2, 128, 16, 16, torch.bfloat16, spoil=spoil2, poison=False)


def test_pages_past_32_bits():
    """A pool whose pages lie so far apart that offsets pass 2^32 bytes."""
    stride = (5 << 30) // 40
    raw = torch.zeros(40 * stride, dtype=torch.uint8, device="cuda")
    b = make_batch(np.random.default_rng(0), [1, 40], [200, 260], 16)
    assert b["pages"] <= 40
    rng = np.random.default_rng(2)
    k, ks, v, vs = random_held(rng, b["pages"], 2, 16, 128, 16)
    page = 2 * 16 * 128

    def far(x, at):
        t = raw.as_strided((b["pages"], 2, 16, 128), (stride, 16 * 128, 128, 1), at)
        t.copy_(torch.from_numpy(x))
        return t.view(E4M3)
    kd, vd = far(k, 0), far(v, page)
    _, ksd = _held(k, ks)
    _, vsd = _held(v, vs)
    q = torch.randn(b["rows"], 4, 128, generator=_gen(3)).bfloat16().cuda()
    layer = P.PagedAttention(dev_batch(b), 4, 2, 128, 16)
    got = layer(q, kd, vd, dev_batch(b), k_scale=ksd, v_scale=vsd)
    same = layer(q, *(_held(x, x[..., 0])[0] for x in (k, v)), dev_batch(b), k_scale=ksd, v_scale=vsd)
    assert torch.equal(got, same)
    new = torch.randn(b["rows"], 2, 128, generator=_gen(4)).bfloat16().cuda()
    P.append_paged(dev_batch(b), kd, vd, new, new, k_scale=ksd, v_scale=vsd)
    check_append(b, 16, 16, k, ks, v, vs, kd, ksd, vd, vsd, new, new, {})


# ---------------------------------------------------------------------------
# appended rows
# ---------------------------------------------------------------------------

def check_append(b, page, block, k0, ks0, v0, vs0, kd, ksd, vd, vsd, k, v, opts, q=None, q_out=None):
    """Bytes before (host) and after (device) an append of rows k and v."""
    pages = k0.shape[0]
    norm = {n: None if opts.get(n) is None else _np(opts[n]) for n in ("q_norm", "k_norm", "rope")}
    pos = None if opts.get("position") is None else opts["position"].cpu().numpy()
    eps, inter = opts.get("eps", 1e-6), opts.get("interleaved", False)
    P_, Hkv, G = page, k0.shape[1], block
    kn, vn = _np(k), _np(v)
    slot = {t: prefix + i for _, t, i, prefix, _ in PO.live_rows(b, page)}

    def row(x, t, weight):
        cs = None
        if norm["rope"] is not None:
            p = slot[t] if pos is None else int(pos[t])
            cs = norm["rope"][min(max(p, 0), len(norm["rope"]) - 1)]
        with np.errstate(invalid="ignore", over="ignore"):
            return PO.norm_rotate(x, weight, eps, cs, inter)

    kg, ksg, vg, vsg = (_bytes(x) for x in (kd, ksd, vd, vsd))
    want_k, want_ks, want_v, want_vs = (x.copy() for x in (k0, ks0, v0, vs0))
    worst = 0.0
    for r, pg, first, old, rows in HO.touched_blocks(b, page, pages, G):
        for h in range(Hkv):
            kept = slice(first, first + old)
            # values: exact
            was = int(np.clip(vs0[pg, h, first // G], 16, 246))
            now = max(HO.scale_byte(HO.largest(np.stack([vn[t, h] for t, _ in rows]))), was if old else 0)
            want_vs[pg, h, first // G] = now
            want_v[pg, h, kept] = HO.rescale(v0[pg, h, kept], was, now)
            for t, o in rows:
                want_v[pg, h, first + o] = HO.hold(vn[t, h], now)
            # keys: a scale of a largest magnitude nearby, values within half a step
            z = {o: row(kn[t, h], t, norm["k_norm"]) for t, o in rows}
            most = [HO.largest(np.stack([y + s * 2.0 ** -17 * m for y, m in z.values()])) for s in (-1, 1)]
            most += [HO.largest(np.stack([y for y, _ in z.values()]))]
            was = int(np.clip(ks0[pg, h, first // G], 16, 246))
            lo, hi = (max(HO.scale_byte(f(most)), was if old else 0) for f in (min, max))
            s = int(ksg[pg, h, first // G])
            assert lo <= s <= hi, f"request {r} page {pg} head {h}: scale {s}, {lo} to {hi} wanted"
            want_ks[pg, h, first // G] = s
            want_k[pg, h, kept] = HO.rescale(k0[pg, h, kept], was, s)
            for o, (y, m) in z.items():
                got = HO.NUMBERS[kg[pg, h, first + o]] * 2.0 ** (s - 127)
                fine = np.isfinite(y)
                assert np.array_equal(~fine, np.isnan(got))
                d = 2.0 ** -17 * m[fine]
                tol = d + np.maximum(2.0 ** -4 * (np.abs(y[fine]) + d), 2.0 ** (s - 127 - 10))
                e = np.abs(got[fine] - y[fine]) / tol
                if e.size:
                    worst = max(worst, float(e.max()))
                want_k[pg, h, first + o] = kg[pg, h, first + o]
    assert worst <= 1.0, worst
    assert np.array_equal(vsg, want_vs) and same(vg, want_v)
    assert np.array_equal(ksg, want_ks) and same(kg, want_k), "slots of no new row changed"
    if q is not None:
        u, qn, got = HALF[q.dtype], _np(q), _np(q_out)
        for t in slot:
            for h in range(qn.shape[1]):
                y, m = row(qn[t, h], t, norm["q_norm"])
                assert (np.abs(got[t, h] - y) <= u * np.abs(y) + 2.0 ** -17 * m + 2.0 ** -25).all()
    return worst


def run_append(b, Hq, Hkv, D, page, block, dt, seed=0, norm=True, rope=True, rot=None, inter=False, position=True,
               amplitude=None, spoil=None, low=100, high=124):
    rng = np.random.default_rng((seed, 9))
    T, g = b["rows"], _gen(seed)
    k0, ks0 = random_pages(rng, b["pages"], Hkv, page, D, block=block, low=low, high=high)
    v0, vs0 = random_pages(rng, b["pages"], Hkv, page, D, block=block, low=low, high=high)
    k0[0, 0, :2] = 0x7f  # (NaN that lies there stays)
    qkv = torch.randn(T, (Hq + 2 * Hkv) * D, generator=g)
    if amplitude is not None:
        qkv *= torch.from_numpy(amplitude)[:, None].float()
    if spoil:
        spoil(qkv)
    qkv = qkv.to(dt).cuda()
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
    kd, ksd = _held(k0, ks0)
    vd, vsd = _held(v0, vs0)
    o = {"interleaved": inter}
    if norm:
        o["q_norm"], o["k_norm"] = ((1 + 0.2 * torch.randn(D, generator=g)).to(dt).cuda() for _ in range(2))
    if rope:
        o["rope"] = P.rope_table(4000, rot or D)
        if position:
            o["position"] = torch.randint(0, 4000, (T,), generator=g, dtype=torch.int32).cuda()
    out = torch.full((T, Hq, D), 7.0, dtype=dt, device="cuda")
    P.append_paged(dev_batch(b), kd, vd, k, v, q=q, q_out=out, k_scale=ksd, v_scale=vsd, **o)
    torch.cuda.synchronize()
    w = check_append(b, page, block, k0, ks0, v0, vs0, kd, ksd, vd, vsd, k, v, o, q, out)
    print(f"[held append] keys: worst {w:.3f} of the tolerance", flush=True)
    live = {t for _, t, *_ in PO.live_rows(b, page)}
    rest = [t for t in range(T) if t not in live]
    assert (out[rest] == 7.0).all()


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,block", [(8, 8), (16, 16), (64, 16), (32, 32), (128, 64)])
def test_append(dt, D, page, block):
    """Requests that begin inside a block, at its edges and in its last slot, and end anywhere."""
    rng = np.random.default_rng((page, block))
    b = make_batch(rng, [1, 5, 0, 70, 1, 33, 2], [0, 3, 9, block - 1, 2 * block, 63, block + 7], page, gap=1)
    run_append(b, 4, 2, D, page, block, dt)


@pytest.mark.parametrize("Hkv", [1, 3, 5])
@pytest.mark.parametrize("D,page,block", [(64, 8, 8), (64, 32, 16), (128, 16, 8), (128, 64, 64)])
def test_append_of_odd_heads(Hkv, D, page, block):
    """Heads that do not fill a workgroup."""
    b = make_batch(np.random.default_rng((Hkv, block)), [9, 1, 40, 2], [3, 8, 30, 0], page)
    run_append(b, 3, Hkv, D, page, block, torch.bfloat16)


@pytest.mark.parametrize("kw", [dict(norm=False, rope=False), dict(rope=False), dict(norm=False, inter=True),
                                dict(rot=32), dict(rot=16, inter=True), dict(position=False)])
def test_append_options(kw):
    b = make_batch(np.random.default_rng(4), [3, 40, 1], [13, 5, 31], 32)
    run_append(b, 3, 1, 128, 32, 16, torch.bfloat16, **kw)


def test_append_scales_of_all_sizes():
    """Rows of very unequal size: scales that grow far past the block's (whose rows go under),
    stay below it, and sit at both ends; all zeros."""
    b = make_batch(np.random.default_rng(5), [2] * 8 + [20], [5] * 8 + [40], 16)
    amp = np.repeat([1e-30, 1e-6, 0.01, 1.0, 100.0, 1e6, 1e30, 0.0, 3.0], [2] * 8 + [20])
    run_append(b, 2, 2, 128, 16, 16, torch.bfloat16, norm=False, amplitude=amp)
    run_append(b, 2, 2, 64, 16, 8, torch.bfloat16, norm=False, rope=False, amplitude=amp * 1e3, low=16, high=246)


def test_append_infinities_and_nan():
    """They are held as NaN, by themselves, and do not reach the scale."""
    b = make_batch(np.random.default_rng(6), [20, 3], [5, 30], 16)

    def spoil(qkv):
        qkv[2, -5], qkv[7, -9], qkv[21, 130] = float("inf"), float("nan"), float("-inf")
        qkv[11, :] = 0
    run_append(b, 1, 2, 128, 16, 16, torch.bfloat16, norm=False, rope=False, spoil=spoil)


@pytest.mark.parametrize("Hkv,T", [(8, 1100), (1, 9000)])
def test_append_of_many_rows(Hkv, T):
    """Calls whose waves go over windows of rows: requests that begin and end inside one."""
    rng = np.random.default_rng(Hkv)
    cuts = np.sort(rng.choice(np.arange(1, T), 30, replace=False))
    rows = np.diff(np.concatenate([[0], cuts, [T - 40]])) if cuts[-1] < T - 40 else np.diff(np.concatenate([[0], cuts, [T]]))
    b = make_batch(rng, rows, rng.integers(0, 50, len(rows)), 16, gap=1)
    assert b["rows"] * 2 * Hkv > 16384
    run_append(b, 2, Hkv, 64, 16, 8, torch.bfloat16)


@pytest.mark.parametrize("D,Hkv,page,block,T", [(64, 47, 16, 8, 900), (128, 25, 8, 8, 900), (128, 25, 32, 16, 900),
                                                (128, 50, 64, 32, 850), (64, 200, 64, 64, 450)])
def test_append_of_rows_that_fill_the_card(D, Hkv, page, block, T):
    """Keys and values by the same workgroups, also where their heads do not fill the last."""
    rng = np.random.default_rng((D, Hkv, block))
    cuts = np.sort(rng.choice(np.arange(1, T), 9, replace=False))
    b = make_batch(rng, np.diff(np.concatenate([[0], cuts, [T]])), rng.integers(0, 90, 10), page, gap=1)
    run_append(b, 3, Hkv, D, page, block, torch.bfloat16, low=110)


def test_append_of_many_requests_one_row_each():
    rng = np.random.default_rng(11)
    b = make_batch(rng, [1] * 300, rng.integers(0, 40, 300), 16)
    run_append(b, 2, 2, 64, 16, 16, torch.float16)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 3, 1), (128, 32, 8), (128, 5, 3)])
@pytest.mark.parametrize("page,block", [(8, 8), (64, 16), (64, 64)])
def test_append_of_single_tokens(dt, D, Hq, Hkv, page, block):
    """Every place of a block, scales that stay and grow, requests without a row or a page."""
    rng = np.random.default_rng((D, page, block))
    prefix = np.concatenate([np.arange(block + 1), [200, 5, 77]])
    b = make_batch(rng, [1] * len(prefix), prefix, page, gap=1)
    b["row_count"][2], b["page_table"][5, 0] = 0, -1
    amp = np.exp(rng.standard_normal(b["rows"]) * 4)
    run_append(b, Hq, Hkv, D, page, block, dt, amplitude=np.clip(amp, 0, 3000), norm=bool(block % 64))


def test_append_of_a_single_token_with_infinities():
    b = make_batch(np.random.default_rng(3), [1, 1, 1], [5, 16, 0], 16)

    def spoil(qkv):
        qkv[0, 130], qkv[1, -3], qkv[2] = float("inf"), float("nan"), 0.0
    run_append(b, 1, 2, 128, 16, 16, torch.bfloat16, norm=False, rope=False, spoil=spoil)


def test_append_without_queries_and_slots_that_do_not_exist():
    """Rows past the table's end or on no page leave every byte as it was."""
    rng = np.random.default_rng(12)
    b = make_batch(rng, [10, 40, 12], [20, 10, 3], 16, width=2)
    b["page_table"][2, 0] = -1
    k0, ks0 = random_pages(rng, b["pages"], 2, 16, 64, block=8, low=110)
    v0, vs0 = random_pages(rng, b["pages"], 2, 16, 64, block=8, low=110)
    kd, ksd = _held(k0, ks0)
    vd, vsd = _held(v0, vs0)
    k, v = (torch.randn(b["rows"], 2, 64, generator=_gen(s)).bfloat16().cuda() for s in (1, 2))
    assert P.append_paged(dev_batch(b), kd, vd, k, v, k_scale=ksd, v_scale=vsd) is None
    check_append(b, 16, 8, k0, ks0, v0, vs0, kd, ksd, vd, vsd, k, v, {})


def test_append_beside_other_data():
    """Pages and scales inside larger pools: what lies between is left as it was."""
    rng = np.random.default_rng(13)
    b = make_batch(rng, [9, 30], [12, 1], 16)
    n, Hkv, D = b["pages"], 2, 64
    k0, ks0 = random_pages(rng, n, 2, Hkv, 16, D, block=8, low=110)
    pool, scales = torch.from_numpy(k0).cuda(), torch.from_numpy(ks0).cuda()
    kd, vd = pool[:, 0].view(E4M3), pool[:, 1].view(E4M3)
    ksd, vsd = scales[:, 0].view(E8M0), scales[:, 1].view(E8M0)
    k, v = (torch.randn(b["rows"], Hkv, D, generator=_gen(s)).bfloat16().cuda() for s in (1, 2))
    P.append_paged(dev_batch(b), kd, vd, k, v, k_scale=ksd, v_scale=vsd)
    check_append(b, 16, 8, k0[:, 0], ks0[:, 0], k0[:, 1], ks0[:, 1], kd, ksd, vd, vsd, k, v, {})


# ---------------------------------------------------------------------------
# compaction
# ---------------------------------------------------------------------------

def run_compact(rng, R, N, W, page, block, groups, heads, D, pmax, paths=None, prefix=None, change=None, spread=12):
    prefix = rng.integers(0, pmax + 1, R).astype(np.int32) if prefix is None else np.asarray(prefix, np.int32)
    R = len(prefix)
    b = make_batch(rng, [N] * R, np.clip(prefix, 0, None), page)
    node, alen = np.full((R, W), -1, np.int32), np.zeros(R, np.int32)
    for r in range(R):
        n = int(rng.integers(1, min(W, N) + 1))
        path = np.sort(rng.choice(N, n, replace=False)) if paths is None else np.asarray(paths[r])
        node[r, :len(path)], alen[r] = path, len(path) - 1
    pool, scale = random_pages(rng, groups, b["pages"], heads, page, D, block=block, low=120 - spread, high=120)
    pool[:, :, 0, 0, 3] = 0x7f
    table = b["page_table"]
    if change:
        change(table, node, alen, prefix)
    pd, sd = _held(pool, scale)

    def up(x):
        return torch.from_numpy(np.ascontiguousarray(x)).cuda()
    assert P.compact_paged(pd, up(table), up(prefix), up(node), up(alen), N, scale=sd) is pd
    wp, ws = HO.compact(pool, scale, table, prefix, node, alen, N)
    assert np.array_equal(_bytes(sd), ws)
    assert same(_bytes(pd), wp)
    return wp, pool


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,block", [(8, 8), (16, 16), (64, 16), (64, 64), (256, 32)])
@pytest.mark.parametrize("R,N,W", [(1, 16, 5), (5, 64, 17), (3, 200, 64)])
def test_compact(D, page, block, R, N, W):
    rng = np.random.default_rng((D, page, N))
    wp, before = run_compact(rng, R, N, W, page, block, 3, 2, D, 100)
    assert not np.array_equal(wp, before)


def test_compact_paths():
    """Rows that stay beside rows that move, in blocks whose scale grows and in one that does
    not; whole paths in place; the root alone; the longest path."""
    rng = np.random.default_rng(2)
    paths = [[0, 1, 2, 9], [0, 1, 2], [0], [5], list(range(64)), list(range(1, 65)), [0, 3, 4, 5, 20, 40]]
    for block in (8, 32):
        run_compact(rng, 0, 70, 64, 32, block, 2, 3, 128, 0, paths=paths, prefix=[3, 13, 0, 7, 5, 30, 16])


def test_compact_past_32_bits():
    """A pool whose second group lies 5 GiB behind the first, pages between."""
    rng = np.random.default_rng(21)
    b = make_batch(rng, [20], [11], 16)
    raw = torch.zeros(6 << 30, dtype=torch.uint8, device="cuda")
    pool, scale = random_pages(rng, 2, b["pages"], 2, 16, 64, block=8, low=110)
    far = raw.as_strided(pool.shape, (5 << 30, 1 << 20, 1024, 64, 1))
    far.copy_(torch.from_numpy(pool))
    _, sd = _held(pool, scale)
    node = np.array([[2, 7, 8, 19]], np.int32)

    def up(x):
        return torch.from_numpy(np.ascontiguousarray(x)).cuda()
    P.compact_paged(far.view(E4M3), up(b["page_table"]), up(np.array([11], np.int32)), up(node),
                    up(np.array([3], np.int32)), 20, scale=sd)
    wp, ws = HO.compact(pool, scale, b["page_table"], [11], node, [3], 20)
    assert same(far.cpu().numpy(), wp) and np.array_equal(_bytes(sd), ws)


def test_compact_leaves_refused_requests_untouched():
    rng = np.random.default_rng(4)

    def change(table, node, alen, prefix):
        node[0, 1] = node[0, 0]          # not increasing
        alen[0] = 1
        node[1, 0] = 16                  # not below the budget
        table[2] = -1                    # on no page
        prefix[3] = 2 ** 31 - 3          # past the capacity
        prefix[4] = -1
        alen[5] = 7                      # past the path's width
    wp, before = run_compact(rng, 7, 16, 6, 16, 16, 2, 2, 64, 40, change=change)


def test_compact_many_groups_and_strides():
    """Groups between a page's own and others' data (K and V of a layer in one pool)."""
    rng = np.random.default_rng(9)
    run_compact(rng, 4, 64, 17, 16, 16, 72, 8, 128, 200)
    b = make_batch(rng, [20], [11], 16)
    raw, rs = random_pages(rng, b["pages"], 3, 2, 16, 64, block=8, low=110)
    pool, scale = torch.from_numpy(raw).cuda(), torch.from_numpy(rs).cuda()
    node = np.array([[2, 7, 8, 19]], np.int32)
    pd, sd = pool[:, :2].transpose(0, 1).view(E4M3), scale[:, :2].transpose(0, 1).view(E8M0)

    def up(x):
        return torch.from_numpy(np.ascontiguousarray(x)).cuda()
    P.compact_paged(pd, up(b["page_table"]), up(np.array([11], np.int32)), up(node), up(np.array([3], np.int32)), 20,
                    scale=sd)
    wp, ws = HO.compact(raw[:, :2].swapaxes(0, 1), rs[:, :2].swapaxes(0, 1), b["page_table"], [11], node, [3], 20)
    want, wants = raw.copy(), rs.copy()
    want[:, :2], wants[:, :2] = wp.swapaxes(0, 1), ws.swapaxes(0, 1)
    assert same(pool.cpu().numpy(), want) and np.array_equal(scale.cpu().numpy(), wants)


def _time(call, n=20):
    """The least of five times of a call among others, in us."""
    begin, end, best = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True), float("inf")
    for _ in range(6):
        begin.record()
        for _ in range(n):
            call()
        end.record()
        torch.cuda.synchronize()
        best = min(best, begin.elapsed_time(end) / n * 1e3)
    return best


@pytest.mark.parametrize("dt,D", [(torch.bfloat16, 128), (torch.float16, 64)])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("rows,hole", [(1, False), (1, True), (300, False), (300, True)])
def test_slots_that_hold_nothing_cost_no_time(dt, D, page, rows, hole):
    """NaN (memory that nothing was written to) behind the last row of a request, and in the pages that
    no request has, leaves the output's bits and the call's time (walking a run for such values
    slot by slot takes ten times as long and more)."""
    ctx, Hq, Hkv = 4001, 8, 2
    rng = np.random.default_rng(page)
    b = make_batch(rng, [rows] * (8 if rows == 1 else 1), [ctx] * (8 if rows == 1 else 1), page)
    table = b["page_table"]
    table[table == 0] = np.setdiff1d(np.arange(b["pages"]), table)[-1]  # (which an entry of no page could be read as)
    if hole:
        table[:, 5] = -1
    k, ks, v, vs = random_held(rng, b["pages"], Hkv, page, D, 8)
    dead = np.ones((b["pages"], page), bool)
    for r in range(len(table)):
        for s in range(ctx + rows):
            at = PO.place(b, r, s, page, b["pages"])
            if at:
                dead[at] = False
    assert dead[0].all()
    kn, vn = k.copy(), v.copy()
    for a in (kn, vn):
        a.transpose(0, 2, 1, 3)[dead] = 0x7f
    q = torch.randn(b["rows"], Hq, D, generator=_gen(1)).to(dt).cuda()
    batch = dev_batch(b)
    layer = P.PagedAttention(batch, Hq, Hkv, D, page)
    got, us = [], []
    for kk, vv in ((k, v), (kn, vn)):
        (kd, ksd), (vd, vsd) = _held(kk, ks), _held(vv, vs)
        out = torch.zeros(b["rows"], Hq, D, dtype=dt, device="cuda")
        us.append(_time(lambda: layer(q, kd, vd, batch, out=out, k_scale=ksd, v_scale=vsd)))
        got.append(out)
    print(f"[held attention] {us[0]:.1f} us, with NaN {us[1]:.1f}", flush=True)
    assert torch.equal(got[0].view(torch.int16), got[1].view(torch.int16))
    assert us[1] < 3 * us[0] + 20


def test_errors_name_the_call():
    """Blocks of four slots, which the pages' shapes allow and the library does not have."""
    b = dev_batch(make_batch(np.random.default_rng(0), [1], [5], 16))
    k = torch.zeros(4, 2, 16, 128, dtype=torch.uint8, device="cuda").view(E4M3)
    s = torch.zeros(4, 2, 4, dtype=torch.uint8, device="cuda").view(E8M0)
    row = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(P.PCTreeError, match="^pctree_append_paged8:"):
        P.append_paged(b, k, k, row, row, k_scale=s, v_scale=s)
    with pytest.raises(P.PCTreeError, match="^pctree_paged_attention8:"):
        P.PagedAttention(b, 2, 2, 128, 16)(row, k, k, b, k_scale=s, v_scale=s)
    pages = torch.zeros(4, 2, 3, 128, dtype=torch.bfloat16, device="cuda")  # (three slots: no power of two)
    with pytest.raises(P.PCTreeError, match="^pctree_append_paged:"):
        P.append_paged(b, pages, pages, row, row)
