"""The operators of a step with 8-bit storage as they are used together, on other streams, in
graphs and beside calls of the 16-bit ones.

A step: norm, projection, append, attention, penalties and masks, a token for every row,
acceptance, compaction.  Each call is compared with its own oracle in its own file; here the
chain's bookkeeping is: what a step leaves in the cache is what the next one reads.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import pctree_held as HO
from paper_2608_02123_amd import pctree as P
from paper_2608_02123_amd import synth
from test_gpu_held import E8M0, _bytes, _held, random_held
from test_gpu_paged import check_attention, dev_batch, make_batch

pytestmark = pytest.mark.gpu

R, N, HQ, HKV, D, PAGE, BLOCK, H, V = 3, 24, 4, 2, 64, 16, 8, 256, 700


def up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Model:
    """One layer of a small target: random weights, an 8-bit cache, penalties and a grammar."""

    def __init__(self, seed, prefix, dt=torch.bfloat16):
        rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)

        def rand(*shape, a=1.0):
            return (torch.randn(*shape, generator=g) * a).to(dt).cuda()
        self.dt = dt
        self.b = make_batch(rng, [N] * R, prefix, PAGE, width=10)
        for r in range(R):  # (room for what the requests grow by)
            self.b["page_table"][r] = np.arange(10) * R + r
        self.pages = 10 * R
        self.rows = (up(self.b["row_start"]), up(self.b["row_count"]))
        self.prefix = up(self.b["prefix_len"])
        self.table = up(self.b["page_table"])
        self.batch = P.PagedBatch(*self.rows, self.prefix, self.table, R * N, N)
        k, ks, v, vs = random_held(rng, self.pages, HKV, PAGE, D, BLOCK)
        self.pool, self.scale = _held(np.stack([k, v]), np.stack([ks, vs]))
        self.embed, self.w = rand(V, H), rand(H)
        self.qkv = rand(H, (HQ + 2 * HKV) * D, a=H ** -0.5)
        self.o, self.head = rand(HQ * D, H, a=0.05), rand(H, V, a=0.3)
        self.rope = P.rope_table(512, D)
        self.layer, self.sampler = P.PagedAttention(self.batch, HQ, HKV, D, PAGE), P.Sampler(R * N, V)
        token, parent, depth = zip(*(synth.random_tree(rng, N, N, 6, V) for _ in range(R)))
        self.token, self.parent, self.depth = up(np.stack(token)), np.stack(parent), up(np.stack(depth))
        self.count = torch.full((R,), N, dtype=torch.int32, device="cuda")
        self.mask = P.build_mask(up(self.parent), self.count)
        self.tree_rows, self.nrows = P.build_retrieve(up(self.parent), self.count, 6)
        self.history = torch.randint(0, V, (90,), generator=g, dtype=torch.int32).cuda()
        self.h0 = up(np.array([0, 30, 70], np.int32))
        self.hn = up(np.array([30, 40, 20], np.int32))
        self.half = torch.full((R,), 0.5, device="cuda")
        self.rep = torch.full((R,), 1.2, device="cuda")
        self.allowed = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, (V + 31) // 32), generator=g, dtype=torch.int64).int().cuda()
        self.which = up((np.arange(R * N) % 3 - 1).astype(np.int32))
        self.uniform = torch.rand(R * N, generator=g).cuda()

    def project(self, y, s):
        """y times its scales, then the projection (a library product of 16 bits)."""
        return ((y.float() * s.repeat_interleave(64, 1)).to(self.dt) @ self.qkv)

    def step(self):
        x = self.embed[self.token.flatten().long()]
        residual = x * 0.5
        y, s = P.rms_norm(x, self.w, residual, group=64)
        qkv = self.project(y, s)
        q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([HQ * D, HKV * D, HKV * D], 1))
        pos = (self.prefix[:, None] + self.depth).flatten().contiguous()
        q = P.append_paged(self.batch, self.pool[0], self.pool[1], k, v, q=q, rope=self.rope, position=pos,
                           k_scale=self.scale[0], v_scale=self.scale[1])
        out = self.layer(q, self.pool[0], self.pool[1], self.batch, mask=self.mask, k_scale=self.scale[0],
                         v_scale=self.scale[1])
        z = out.flatten(1) @ self.o
        z = P.rms_norm(z, self.w, residual)
        logits = z @ self.head
        raw = logits.clone()
        P.adjust_logits(logits, *self.rows, max_rows=N, history=self.history, history_start=self.h0,
                        history_count=self.hn, repetition=self.rep, presence=self.half, token=self.token,
                        mask=self.mask, allowed=self.allowed, allowed_row=self.which)
        token, logprob = self.sampler(logits, self.uniform)
        acc = P.accept_greedy(self.token, self.tree_rows, self.nrows, token.view(R, N))
        return {"q": q, "out": out, "raw": raw, "logits": logits, "token": token, "logprob": logprob, **acc}

    def compact(self, acc):
        P.compact_paged(self.pool, self.table, self.prefix, acc["accept_node"], acc["accept_len"], N, scale=self.scale)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_two_steps(dt):
    """The attention of each step reads what the append before it, and the compaction of the step
    before, left in the cache; tokens are never forbidden ones."""
    m = Model(1, [20, 33, 7], dt)
    for _ in range(2):
        b = {**m.b, "prefix_len": m.prefix.cpu().numpy(), "page_table": m.table.cpu().numpy()}
        got = m.step()
        torch.cuda.synchronize()
        kv = [torch.from_numpy(HO.values(_bytes(m.pool[i]), _bytes(m.scale[i]))) for i in (0, 1)]
        check_attention(b, got["q"], *kv, got["out"], D ** -0.5, m.mask, N)
        token, which = got["token"].long(), m.which.long()
        bit = (m.allowed[which.clamp_min(0), token // 32] >> (token % 32).int()) & 1
        assert ((bit == 1) | (which < 0) | (which >= 2)).all()
        assert (got["logits"] != got["raw"]).any()
        before, scales = _bytes(m.pool), _bytes(m.scale)
        # a path that the greedy acceptance need not have found, so that slots move
        acc = {"accept_node": up(np.array([[0, 3, 5, 9], [0, 2, -1, -1], [0, 1, 2, 20]], np.int32)),
               "accept_len": up(np.array([3, 1, 3], np.int32))}
        m.compact(acc)
        wp, ws = HO.compact(before, scales, b["page_table"], b["prefix_len"], acc["accept_node"].cpu().numpy(),
                            acc["accept_len"].cpu().numpy(), N)
        assert np.array_equal(_bytes(m.scale), ws)
        same = _bytes(m.pool) == wp
        assert (same | ((wp & 127) == 127)).all()
        m.prefix += acc["accept_len"] + 1


def test_a_captured_step_follows_its_arrays():
    """A graph of the whole step, replayed with new prefixes, tokens and histories, between eager
    work, gives what eager calls give; two graphs hold an attention object each."""
    m = Model(2, [20, 33, 7])
    start = (m.pool.view(torch.uint8).clone(), m.scale.view(torch.uint8).clone())

    def reset():
        m.pool.view(torch.uint8).copy_(start[0])
        m.scale.view(torch.uint8).copy_(start[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = m.step()
        m.compact(got)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = m.step()
        m.compact(kept)
    gen = torch.Generator().manual_seed(5)
    for k in range(3):
        m.prefix.copy_(torch.tensor([[20, 33, 7], [1, 90, 16], [50, 0, 31]][k], dtype=torch.int32))
        m.token.copy_(torch.randint(0, V, (R, N), generator=gen, dtype=torch.int32))
        m.history.copy_(torch.randint(0, V, (90,), generator=gen, dtype=torch.int32))
        reset()
        want = {n: t.clone() for n, t in (lambda g: (m.compact(g), g)[1])(m.step()).items()}
        pool, scale = m.pool.view(torch.uint8).clone(), m.scale.view(torch.uint8).clone()
        (torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in want.items():
            assert torch.equal(t.view(torch.uint8) if t.dtype.is_floating_point else t,
                               kept[n].view(torch.uint8) if t.dtype.is_floating_point else kept[n]), (k, n)
        assert torch.equal(m.pool.view(torch.uint8), pool) and torch.equal(m.scale.view(torch.uint8), scale)


def test_calls_on_another_stream():
    """Each call takes the stream that it is given, and allocates there."""
    m = Model(3, [20, 33, 7])
    want = m.step()
    torch.cuda.synchronize()
    m2 = Model(3, [20, 33, 7])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    x = m2.embed[m2.token.flatten().long()]
    residual = x * 0.5
    s.wait_stream(torch.cuda.current_stream())
    y, sc = P.rms_norm(x, m2.w, residual, group=64, stream=s)
    with torch.cuda.stream(s):
        qkv = m2.project(y, sc)
        q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([HQ * D, HKV * D, HKV * D], 1))
        pos = (m2.prefix[:, None] + m2.depth).flatten().contiguous()
    kw = dict(k_scale=m2.scale[0], v_scale=m2.scale[1], stream=s)
    q = P.append_paged(m2.batch, m2.pool[0], m2.pool[1], k, v, q=q, rope=m2.rope, position=pos, **kw)
    out = m2.layer(q, m2.pool[0], m2.pool[1], m2.batch, mask=m2.mask, **kw)
    raw = want["raw"].clone()
    s.wait_stream(torch.cuda.current_stream())
    P.adjust_logits(raw, *m2.rows, max_rows=N, history=m2.history, history_start=m2.h0, history_count=m2.hn,
                    repetition=m2.rep, presence=m2.half, token=m2.token, mask=m2.mask, allowed=m2.allowed,
                    allowed_row=m2.which, stream=s)
    s.synchronize()
    for name, t in (("q", q), ("out", out), ("logits", raw)):
        assert torch.equal(t, want[name]), name
    assert torch.equal(m2.pool.view(torch.uint8), m.pool.view(torch.uint8))
    acc = {"accept_node": want["accept_node"], "accept_len": want["accept_len"]}
    P.compact_paged(m2.pool, m2.table, m2.prefix, acc["accept_node"], acc["accept_len"], N, s, scale=m2.scale)
    s.synchronize()
    m.compact(acc)
    torch.cuda.synchronize()
    assert torch.equal(m2.pool.view(torch.uint8), m.pool.view(torch.uint8))


def test_one_object_for_both_kinds_of_pages():
    """An attention object serves 16-bit pages and pages in 8 bits in turn; values that both can
    hold give the same rows within the rounding of weights to 16 bits."""
    rng = np.random.default_rng(4)
    b = make_batch(rng, [1, 60, 2], [300, 100, 5], 16)
    k, ks, v, vs = random_held(rng, b["pages"], 2, 16, 128, 16)
    kd, ksd = _held(k, ks)
    vd, vsd = _held(v, vs)
    k16, v16 = (torch.from_numpy(HO.values(x, s)).bfloat16().cuda() for x, s in ((k, ks), (v, vs)))
    q = torch.randn(b["rows"], 8, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    batch = dev_batch(b)
    layer = P.PagedAttention(batch, 8, 2, 128, 16)
    first = layer(q, k16, v16, batch).clone()
    held = layer(q, kd, vd, batch, k_scale=ksd, v_scale=vsd).clone()
    again = layer(q, k16, v16, batch)
    assert torch.equal(first, again)
    ref = check_attention(b, q, k16.double().cpu(), v16.double().cpu(), held, 128 ** -0.5)[0]
    assert len(ref) == 63
    one = P.paged_attention(q, kd, vd, batch, k_scale=ksd, v_scale=vsd)
    assert torch.equal(one, held)


def test_the_same_calls_give_the_same_bits():
    for seed in (6, 7):
        runs = []
        for _ in range(2):
            m = Model(seed, [64, 2, 15])
            got = m.step()
            m.compact(got)
            torch.cuda.synchronize()
            runs.append((got, _bytes(m.pool), _bytes(m.scale)))
        (a, p0, s0), (b, p1, s1) = runs
        assert all(torch.equal(a[n], b[n]) for n in a) and np.array_equal(p0, p1) and np.array_equal(s0, s1)


def test_held_refusals():
    m = Model(8, [4, 5, 6])
    q = torch.zeros(R * N, HQ, D, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(R * N, HKV, D, dtype=torch.bfloat16, device="cuda")
    kc, vc, ks, vs = m.pool[0], m.pool[1], m.scale[0], m.scale[1]
    for bad, error in ((dict(k_scale=ks), TypeError), (dict(v_scale=vs), TypeError),
                       (dict(k_scale=ks, v_scale=vs.view(torch.uint8)), TypeError),
                       (dict(k_scale=ks[:-1], v_scale=vs[:-1]), ValueError),
                       (dict(k_scale=ks[:, :, :1], v_scale=vs), ValueError),
                       (dict(k_scale=ks.cpu(), v_scale=vs.cpu()), ValueError)):
        with pytest.raises(error):
            m.layer(q, kc, vc, m.batch, **bad)
        with pytest.raises(error):
            P.append_paged(m.batch, kc, vc, k, k, **bad)
    with pytest.raises(TypeError):  # pages in 8 bits without scales
        m.layer(q, kc, vc, m.batch)
    with pytest.raises(TypeError):
        m.layer(q.float(), kc, vc, m.batch, k_scale=ks, v_scale=vs)
    fine = torch.zeros(m.pages, HKV, 4, dtype=torch.uint8, device="cuda").view(E8M0)
    with pytest.raises(P.PCTreeError):  # blocks of four slots
        m.layer(q, kc, vc, m.batch, k_scale=fine, v_scale=fine)
    node, n = up(np.zeros((R, 4), np.int32)), up(np.zeros(R, np.int32))
    for pool, scale, error in ((m.pool, m.scale[:1], ValueError), (m.pool, m.scale.view(torch.uint8), TypeError),
                               (m.pool.view(torch.uint8), m.scale, ValueError),
                               (m.pool.to(torch.bfloat16), m.scale, ValueError)):
        with pytest.raises(error):
            P.compact_paged(pool, m.table, m.prefix, node, n, N, scale=scale)
    # a pool of bytes with a scale of its own moves as before, without scales
    P.compact_paged(m.pool, m.table, m.prefix, node, n, N)
