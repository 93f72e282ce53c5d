"""Rotation of queries and keys on their way into the paged cache, against 64 bits: layouts, parts of a head, scalings, far positions, strides,
idle rows, bad pages."""
import math

import pytest
import torch

import paper_2502_11880_b200 as bn
from helpers import Guarded

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = {F32: 2.0 ** -24, BF: 2.0 ** -8, HF: 2.0 ** -11}


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, low=1.0, high=4.0, context=8192, freqs=None, **_):
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)] if freqs is None else list(freqs)
    if freqs is None and scaling == "linear":
        f = [x / factor for x in f]
    if freqs is None and scaling == "bands":
        s = [min(1.0, max(0.0, (x * context / (2 * math.pi) - low) / (high - low))) for x in f]
        f = [(1 - b) * x / factor + b * x for x, b in zip(f, s)]
    return torch.tensor(f, dtype=torch.float64)


def rotated(x, pos, layout="half", magnitude=1.0, **rope):
    """(values, bounds of their binary32 error) in 64 bits: x [tokens][heads][dim]."""
    rot = rope["rot"]
    x = x.double().cpu()
    out, err = x.clone(), torch.zeros_like(x)
    angle = torch.tensor(pos, dtype=torch.float64)[:, None] * frequencies(**rope)
    c, s = ((f(angle) * magnitude)[:, None] for f in (torch.cos, torch.sin))
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    # sines and cosines to 2^-22 (the angle in half turns to 2^-25 = 2^-23 radians, the function 2 steps), two products and a sum
    err[..., a] = err[..., b] = (x[..., a].abs() + x[..., b].abs()) * (2.0 ** -22 + 3 * 2.0 ** -24) * max(abs(magnitude), 1e-30)
    return out, err


def close(got, want, err):
    bound = err + want.abs() * HALF_STEP[got.dtype] * 1.001 + (2.0 ** -25 if got.dtype == HF else 1e-37)
    worst = ((got.double().cpu() - want).abs() / bound).max()
    assert worst <= 1, float(worst)


class Case:
    def __init__(self, spans, heads, kv_heads, dim, page, dtype, io, seed=0, far=0, nhd=False):
        """spans: (cached, new) tokens of each sequence; only the pages of new tokens exist."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.spans, self.heads = spans, heads
        first = [b // page for b, _ in spans]
        count = [-(-(b + n) // page) - f for (b, n), f in zip(spans, first)]
        pages = sum(count) + 3
        dp = -(-dim // 8) * 8
        shape = (2, pages, page, kv_heads, dp) if nhd else (2, pages, kv_heads, page, dp)
        self.k, self.v = (torch.full(shape, 7.0, dtype=dtype, device="cuda") for _ in range(2))
        if nhd:
            self.k, self.v = self.k.permute(0, 1, 3, 2, 4), self.v.permute(0, 1, 3, 2, 4)
        self.padded = self.k, self.v
        self.k, self.v = self.k[..., :dim], self.v[..., :dim]
        self.cache = bn.KvCache(self.k, self.v)
        order = torch.randperm(pages, generator=g, device="cuda").cpu().int()
        self.table = torch.full((len(spans), max(f + c for f, c in zip(first, count)) + 1), -1, dtype=torch.int32)
        at = 0
        for i, (f, c) in enumerate(zip(first, count)):
            self.table[i, f:f + c] = order[at:at + c]
            at += c
        self.table = self.table.cuda()
        self.len = torch.tensor([b + n for b, n in spans], dtype=torch.int32, device="cuda")
        start = [0]
        for _, n in spans:
            start.append(start[-1] + n)
        self.start = torch.tensor(start, dtype=torch.int32, device="cuda")
        self.pos = [b + j for b, n in spans for j in range(n)]
        self.seq = [i for i, (_, n) in enumerate(spans) for _ in range(n)]
        t = start[-1]
        fused = torch.randn(t, heads + 2 * kv_heads, dim, generator=g, device="cuda").to(io)
        self.q, self.k_new, self.v_new = fused[:, :heads], fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:]

    def run(self, rope, out_type, layer=1, start=True, **kw):
        out = Guarded(self.q.shape, out_type)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = bn.bitnet_kv_append_rope(self.cache, layer, rope, self.q, self.k_new, self.v_new, self.table, self.len, self.start if start else None,
                                       q_out=out.t, dev_status=status, **kw)
        torch.cuda.synchronize()
        assert out.intact() and int(status) == 0 and got.data_ptr() == out.t.data_ptr()
        return got

    def check(self, got, layer=1, **rope):
        close(got, *rotated(self.q, self.pos, **rope))
        k, err = rotated(self.k_new, self.pos, **rope)
        page = self.cache.page_size
        at = self.table.cpu()[self.seq, [p // page for p in self.pos]].long().cuda()
        inside = torch.tensor([p % page for p in self.pos], device="cuda")
        close(self.k[layer][at, :, inside], k, err)
        assert torch.equal(self.v[layer][at, :, inside], self.v_new.to(self.v.dtype))
        # nothing else was written, but the padding of the rows
        for t in self.padded:
            t = t.clone()
            assert bool((t[layer][at, :, inside][..., self.cache.head_dim:] == 0).all())
            t[layer][at, :, inside] = 7.0
            t[layer, at, :, inside] = 7.0
            assert bool((t == 7.0).all())


CASES = [
    # spans, heads, kv_heads, dim, page, cache, in, out, rope
    ([(0, 1)], 1, 1, 64, 16, BF, F32, F32, dict(rot=64)),
    ([(5, 1), (100000, 1), (0, 1)], 64, 8, 128, 16, BF, F32, BF, dict(rot=128, base=500000.0)),
    ([(0, 77), (30, 0), (40, 200)], 8, 2, 128, 8, BF, BF, BF, dict(rot=64)),
    ([(9, 33)], 32, 32, 100, 32, HF, F32, HF, dict(rot=100)),
    ([(9, 33)], 4, 4, 100, 32, HF, HF, F32, dict(rot=100, layout="interleaved")),
    ([(0, 40)], 6, 3, 96, 64, HF, F32, F32, dict(rot=48, layout="interleaved")),
    ([(0, 9)], 3, 1, 4, 8, BF, F32, BF, dict(rot=2)),
    ([(0, 9)], 3, 1, 4, 8, BF, BF, F32, dict(rot=4, layout="interleaved")),
    ([(70, 50)], 5, 5, 72, 128, BF, F32, BF, dict(rot=6)),
    ([(70, 50)], 5, 5, 72, 128, HF, HF, HF, dict(rot=70, layout="interleaved")),
    ([(70, 20)], 4, 2, 120, 16, BF, F32, F32, dict(rot=20)),
    ([(70, 20)], 4, 2, 124, 16, BF, BF, BF, dict(rot=122)),
    ([(3, 300)] * 3, 12, 4, 64, 16, BF, F32, BF, dict(rot=32, scaling="linear", factor=3.5)),
    ([(20000, 65), (3, 5)], 8, 2, 128, 32, HF, F32, F32, dict(rot=128, scaling="bands", factor=8.0, base=500000.0, context=8192)),
    ([(0, 20)], 2, 2, 32, 16, BF, F32, F32, dict(rot=8, freqs=[1.0, -0.3, 7.5, 0.0], magnitude=1.25)),
]


@pytest.mark.parametrize("spans,heads,kv_heads,dim,page,dtype,io,out,rope", CASES)
def test_matches_64_bits(spans, heads, kv_heads, dim, page, dtype, io, out, rope):
    c = Case(spans, heads, kv_heads, dim, page, dtype, io, seed=dim + heads)
    c.check(c.run(bn.Rope(**rope), out), **rope)


def test_agrees_with_append_where_nothing_turns():
    """Position 0 and frequency 0: the rows of a plain append, bit for bit."""
    c = Case([(0, 1), (0, 1)], 4, 2, 96, 16, BF, F32)
    got = c.run(bn.Rope(96), F32)
    assert torch.equal(got, c.q)
    k, v = c.k.clone(), c.v.clone()
    c.k.fill_(7.0), c.v.fill_(7.0)
    bn.bitnet_kv_append(c.cache, 1, c.k_new, c.v_new, c.table, c.len, c.start)
    assert torch.equal(c.k, k) and torch.equal(c.v, v)
    c = Case([(50, 9)], 4, 2, 96, 16, BF, BF)
    assert torch.equal(c.run(bn.Rope(96, freqs=[0.0] * 48), BF), c.q)


def test_elements_beyond_the_pairs_move_as_they_are():
    c = Case([(50, 9)], 4, 2, 64, 16, HF, F32)
    c.q[..., 10] = float("inf")
    c.q[..., 63] = float("nan")
    for layout in ("half", "interleaved"):
        got = c.run(bn.Rope(10, layout=layout), F32)
        assert torch.equal(got[..., 10:63], c.q[..., 10:63]) and torch.isnan(got[..., 63]).all() and torch.isfinite(got[..., :10]).all()


def test_far_positions():
    """Near 2^31: the angle's product wraps around exactly."""
    page = 1 << 20
    n = 2 ** 31 - 3 * page
    c = Case([(0, 1), (0, 1)], 2, 1, 32, 16, BF, F32)
    k = torch.zeros(1, 2, 1, page, 32, dtype=BF, device="cuda")
    cache = bn.KvCache(k, k.clone())
    table = torch.full((2, 2048), -1, dtype=torch.int32, device="cuda")
    lens = [n, 131072 * 8 + 3]
    for i, x in enumerate(lens):
        table[i, (x - 1) // page] = i
    rope = dict(rot=32, base=500000.0)
    got = bn.bitnet_kv_append_rope(cache, 0, bn.Rope(**rope), c.q, c.k_new, c.v_new, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    want, err = rotated(c.q, [x - 1 for x in lens], **rope)
    # (the reference's own angles: 64-bit products of up to 2^31)
    close(got, want, err + 2.0 ** 31 * 2.0 ** -52 * c.q.double().abs().amax().cpu())


def test_strides_layouts_and_stream():
    c = Case([(3, 70), (0, 5)], 8, 2, 64, 16, BF, F32, nhd=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.run(bn.Rope(64), F32)
    c.check(got, rot=64)
    # odd strides and addresses: every width of a vector
    for shift, cut in ((1, 63), (2, 62), (4, 60)):
        for io in (F32, BF):
            c = Case([(3, 70), (0, 5)], 8, 2, 60, 16, BF, io)
            wide = torch.zeros(75, 12, 64, dtype=io, device="cuda")
            wide[:, :, shift:shift + 60][:, :8] = c.q
            if shift + 60 <= 64:
                view = wide.view(-1)[shift:][:75 * 12 * 64 - 64].as_strided((75, 8, 60), (12 * 64, 64, 1))
                c.q = view
            c.check(c.run(bn.Rope(40), F32), rot=40)


def test_queries_in_place_and_without_queries():
    c = Case([(11, 40)], 8, 2, 128, 16, BF, BF)
    want = c.run(bn.Rope(128), BF).clone()
    c.q = c.q.contiguous()
    got = bn.bitnet_kv_append_rope(c.cache, 0, bn.Rope(128), c.q, c.k_new, c.v_new, c.table, c.len, c.start, q_out=c.q)
    assert got.data_ptr() == c.q.data_ptr() and torch.equal(got, want)
    k = c.k.clone()
    c.k.fill_(7.0)
    assert bn.bitnet_kv_append_rope(c.cache, 0, bn.Rope(128), None, c.k_new, c.v_new, c.table, c.len, c.start) is None
    assert torch.equal(c.k[0], k[0])
    got = bn.bitnet_kv_append_rope(c.cache, 0, bn.Rope(128), c.q, c.k_new, c.v_new, c.table, c.len, c.start, q_dtype=F32)
    assert got.dtype == F32 and got.shape == c.q.shape


def test_idle_rows_and_bad_pages():
    """Rows before the start are left alone; a token without a page is reported, its query is written."""
    c = Case([(5, 1), (40, 1), (9, 1), (33, 1)], 4, 2, 64, 16, BF, F32)
    good = c.run(bn.Rope(64), F32, start=False).clone()
    k = c.k.clone()
    c.len[2] = 0
    out = torch.full_like(good, 9.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.k.fill_(7.0)
    bn.bitnet_kv_append_rope(c.cache, 1, bn.Rope(64), c.q, c.k_new, c.v_new, c.table, c.len, q_out=out, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and bool((out[2] == 9.0).all()) and all(torch.equal(out[i], good[i]) for i in (0, 1, 3))
    page = int(c.table[2, 0])
    assert bool((c.k[1, page] == 7.0).all())
    for bad in (-1, c.cache.num_pages, 2 ** 31 - 1, -2 ** 31):
        table = c.table.clone()
        table[1, 2] = bad
        c.len[2] = 10
        c.k.fill_(7.0)
        status.zero_()
        bn.bitnet_kv_append_rope(c.cache, 1, bn.Rope(64), c.q, c.k_new, c.v_new, table, c.len, q_out=out, dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == 7 and torch.equal(out, good)
        want = k.clone()
        want[1, int(c.table[1, 2]), :, 40 % 16] = 7.0
        assert torch.equal(c.k, want)
    c.len[0] = 2 ** 31 - 1                       # beyond the table
    status.zero_()
    bn.bitnet_kv_append_rope(c.cache, 1, bn.Rope(64), c.q, c.k_new, c.v_new, c.table, c.len, q_out=out, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 7


def test_tokens_behind_the_last_sequence():
    """A padded batch: rows that belong to no sequence are left as they were, and write nothing."""
    c = Case([(5, 3), (40, 2), (7, 4)], 4, 2, 64, 16, BF, F32)
    good = c.run(bn.Rope(64), F32).clone()
    k, v = c.k.clone(), c.v.clone()
    c.k.fill_(7.0), c.v.fill_(7.0)
    pad = lambda t: torch.cat([t, torch.full((6, *t.shape[1:]), 3.0, device="cuda")])
    out, status = torch.full((15, 4, 64), 9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    bn.bitnet_kv_append_rope(c.cache, 1, bn.Rope(64), pad(c.q), pad(c.k_new), pad(c.v_new), c.table, c.len, c.start, q_out=out, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(out[:9], good) and bool((out[9:] == 9.0).all())
    assert torch.equal(c.k, k) and torch.equal(c.v, v)
    c.k.fill_(7.0)
    start = torch.tensor([2, 3, 5, 9], dtype=torch.int32, device="cuda")       # two ahead of the first
    out.fill_(9.0)
    bn.bitnet_kv_append_rope(c.cache, 1, bn.Rope(64), c.q, c.k_new, c.v_new, c.table, c.len, start, q_out=out[:9], dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and bool((out[:2] == 9.0).all()) and torch.equal(out[2:9], good[2:9])


def test_graph():
    c = Case([(5, 1), (40, 1)], 4, 2, 64, 16, BF, F32)
    rope, out = bn.Rope(64), torch.empty(2, 4, 64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bn.bitnet_kv_append_rope(c.cache, 1, rope, c.q, c.k_new, c.v_new, c.table, c.len, q_out=out)
    del rope                                     # (its values are in the graph)
    c.len.add_(1)
    c.pos = [p + 1 for p in c.pos]
    graph.replay()
    torch.cuda.synchronize()
    c.check(out, rot=64)


def test_refusals():
    c = Case([(5, 1)], 4, 2, 64, 16, BF, F32)
    ok = dict(cache=c.cache, layer=0, rope=bn.Rope(64), q=c.q, k=c.k_new, v=c.v_new, table=c.table, kv_len=c.len)
    for bad in (dict(layer=2), dict(rope=bn.Rope(128)), dict(q=c.q.to(BF)), dict(q=c.q[..., :32]), dict(k=c.q), dict(v=c.v_new.to(BF)), dict(k=c.k_new.to(HF), v=c.v_new.to(HF), q=c.q.to(HF)),
                dict(table=c.table.long()), dict(kv_len=c.len[:0]), dict(q_out=torch.empty(1, 4, 64, dtype=HF, device="cuda")),
                dict(q_out=torch.empty(2, 4, 64, device="cuda")), dict(q=torch.cat([c.q, c.q]))):
        with pytest.raises(bn.BitnetError):
            bn.bitnet_kv_append_rope(**dict(ok, **bad))
    empty = torch.empty(0, 4, 64, device="cuda")
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    got = bn.bitnet_kv_append_rope(c.cache, 0, bn.Rope(64), empty, empty[:, :2], empty[:, :2], c.table, c.len, none)
    assert got.shape == (0, 4, 64)
