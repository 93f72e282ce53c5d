"""Attention of single tokens and of prompts over the paged cache against a 64-bit implementation: head layouts, odd head sizes,
page sizes, pages that end inside a tile, windows and sinks, empty sequences, poisoned unused memory, strides, streams."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from helpers import Guarded
from kv_ref import attn_ref, check_attn

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
# relative rounding of the probabilities: decode carries two 16-bit pieces (three for fp32 io over bf16)
DECODE_P = {(BF, False): 2.0 ** -16, (BF, True): 2.0 ** -23, (HF, False): 2.0 ** -21, (HF, True): 2.0 ** -21}
PROMPT_P = {BF: 2.0 ** -8, HF: 2.0 ** -11}


class Paged:
    """A pool full of NaN whose visible rows hold values, with pages in shuffled order."""

    def __init__(self, lens, kv_heads, dim, page, dtype, seed=0, layers=2, layer=1, nhd=False, extra=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        width = max(1, -(-max(lens) // page)) + 1
        counts = [-(-max(0, n) // page) for n in lens]
        pages = sum(counts) + extra
        dp = -(-dim // 8) * 8
        shape = (layers, pages, page, kv_heads, dp) if nhd else (layers, pages, kv_heads, page, dp)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        if nhd:
            self.k, self.v = self.k.permute(0, 1, 3, 2, 4), self.v.permute(0, 1, 3, 2, 4)
        self.k, self.v = self.k[..., :dim], self.v[..., :dim]
        order = torch.randperm(pages, generator=g, device="cuda").cpu()
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32)
        at = 0
        for i, n in enumerate(lens):
            self.table[i, :counts[i]] = order[at:at + counts[i]].int()
            at += counts[i]
            for e in range(counts[i]):
                rows, p = min(page, n - e * page), int(self.table[i, e])
                for t in (self.k, self.v):
                    t[layer, p, :, :rows] = torch.randn(kv_heads, rows, dim, generator=g, device="cuda").to(dtype)
        self.table = self.table.cuda()
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.cache, self.layer = bn.KvCache(self.k, self.v), layer
        self.g = g

    def queries(self, n, heads, dim, dtype, scale=1.0):
        return (torch.randn(n, heads, dim, generator=self.g, device="cuda") * scale).to(dtype)

    def ref(self, q, pos, seq, scale, window, sinks):
        return attn_ref(self.k[self.layer], self.v[self.layer], q, self.table, pos, seq, scale, window, sinks)


def run_decode(p, q, **kw):
    out = Guarded(q.shape, q.dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = bn.new_attn_workspace(q.shape[0], q.shape[1], p.cache.kv_heads, p.cache.head_dim)
    for _ in range(2):                       # the workspace is left as it was found
        bn.bitnet_attn_decode(p.cache, p.layer, q, p.table, p.len, out=out.t, workspace=ws, dev_status=status, **kw)
    torch.cuda.synchronize()
    assert out.intact() and int(status) == 0 and bn.bitnet_device_status() == 0
    return out.t


DECODE = [
    # lens, q_heads, kv_heads, dim, page, dtype, io, window, sinks
    ([1], 1, 1, 64, 16, BF, BF, 0, 0),
    ([0], 4, 4, 64, 16, BF, BF, 0, 0),                         # nothing visible: zeros
    ([0, 1, 2, 63, 64, 65], 8, 2, 128, 8, BF, F32, 0, 0),
    ([5, 0, 300, 129], 32, 8, 128, 16, BF, BF, 0, 0),
    ([517], 32, 8, 128, 16, BF, F32, 0, 0),
    ([700, 33], 64, 8, 128, 64, HF, HF, 0, 0),
    ([1030], 12, 12, 100, 32, HF, F32, 0, 0),
    ([260, 77], 16, 16, 96, 128, BF, BF, 0, 0),
    ([90, 19], 6, 2, 4, 8, HF, HF, 0, 0),                      # smallest head
    ([150], 5, 1, 36, 1024, BF, F32, 0, 0),                    # page larger than the context
    ([200, 70], 20, 2, 112, 16, BF, BF, 0, 0),                 # 10 heads per kv head: two blocks
    ([130], 33, 1, 128, 16, HF, F32, 0, 0),                    # 33 heads per kv head: five blocks, the last of one
    ([1000, 64, 3, 66], 8, 2, 128, 16, BF, BF, 64, 0),
    ([1000, 64, 3, 66, 0], 8, 2, 128, 16, BF, F32, 1, 0),      # a window of one: itself
    ([1000, 640, 3, 66], 8, 8, 100, 16, HF, F32, 100, 4),
    ([900, 130, 80], 8, 2, 64, 32, HF, HF, 63, 70),            # sinks over more than a tile
    ([900, 130, 80], 4, 2, 128, 8, BF, BF, 5, 2000),           # sinks beyond the context: everything
    ([300, 70, 9], 6, 3, 72, 8, BF, F32, 0, 0),                # rows of an odd number of 16-byte pieces
    ([300, 70, 1], 4, 4, 120, 256, HF, HF, 90, 3),
    ([500, 64], 8, 1, 88, 32, BF, BF, 0, 0),
    ([400], 8, 2, 128, 8, BF, BF, 390, 9),                     # sinks meet the window's first tile
]


@pytest.mark.parametrize("lens,hq,hkv,dim,page,dtype,io,window,sinks", DECODE)
def test_decode_matches_64_bits(lens, hq, hkv, dim, page, dtype, io, window, sinks):
    p = Paged(lens, hkv, dim, page, dtype, seed=len(lens) + dim)
    q = p.queries(len(lens), hq, dim, io)
    scale = dim ** -0.5
    out = run_decode(p, q, window=window, sinks=sinks)
    check_attn(out, p.ref(q, [n - 1 for n in lens], range(len(lens)), scale, window, sinks), DECODE_P[dtype, io == F32])
    assert all(bool((out[i] == 0).all()) for i, n in enumerate(lens) if n == 0)


@pytest.mark.parametrize("io", [BF, F32])
def test_decode_long_row_over_many_parts(io):
    """One row's tiles on every SM: parts meet in the workspace; the same call again gives the same bits."""
    p = Paged([40003], 1, 128, 64, BF, seed=3, layers=1, layer=0)
    q = p.queries(1, 8, 128, io)
    out = run_decode(p, q)
    check_attn(out, p.ref(q, [40002], [0], 128 ** -0.5, 0, 0), DECODE_P[BF, io == F32])
    for _ in range(5):
        assert torch.equal(out, run_decode(p, q))


def test_decode_more_sequences_than_threads():
    lens = [(7 * i) % 90 for i in range(700)]
    p = Paged(lens, 1, 64, 8, HF, seed=5, layers=1, layer=0)
    q = p.queries(700, 2, 64, HF)
    check_attn(run_decode(p, q), p.ref(q, [n - 1 for n in lens], range(700), 0.125, 0, 0), DECODE_P[HF, False])


def test_decode_large_scores_and_negative_scale():
    p = Paged([300, 90], 2, 64, 16, HF, seed=6)
    for s, scale in ((30.0, 0.125), (3.0, -0.5), (1.0, 0.0), (1e4, 0.125)):
        q = p.queries(2, 8, 64, F32, s)
        check_attn(run_decode(p, q, scale=scale), p.ref(q, [299, 89], [0, 1], scale, 0, 0), DECODE_P[HF, True])


def test_decode_strided_queries_other_pool_order_and_stream():
    """q as a slice of fused fp32 rows, pools in [page][token][head] order, everything on another stream."""
    p = Paged([333, 40, 7], 4, 100, 16, BF, seed=7, nhd=True)
    fused = p.queries(3, 24, 100, F32).view(3, 2400)
    q = fused[:, :1600].view(3, 16, 100)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = run_decode(p, q)
    check_attn(out, p.ref(q, [332, 39, 6], range(3), 0.1, 0, 0), DECODE_P[BF, True])


@pytest.mark.parametrize("dim", [64, 100, 128])
def test_decode_bad_pages_are_reported_and_not_read(dim):
    p = Paged([100, 50], 2, dim, 16, BF, seed=8)
    q = p.queries(2, 4, dim, BF)
    good = run_decode(p, q)
    for bad in (-1, p.cache.num_pages, 2 ** 31 - 1, -2 ** 31):
        table = p.table.clone()
        table[0, 2] = bad
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = bn.bitnet_attn_decode(p.cache, p.layer, q, table, p.len, dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == 7 and torch.equal(out[1], good[1]) and torch.isfinite(out[0]).all()


def test_decode_length_beyond_the_table_stops_at_its_end():
    p = Paged([64], 1, 64, 16, BF, seed=9)
    p.table = p.table[:, :4].contiguous()
    q = p.queries(1, 1, 64, BF)
    want = run_decode(p, q)
    p.len[0] = 2 ** 31 - 1
    assert torch.equal(run_decode(p, q), want)


def test_decode_offsets_beyond_32_bits():
    """Pools of more than 2^32 bytes each: the last pages."""
    pages, page, heads, dim = 70000, 64, 4, 128
    k, v = (torch.empty(1, pages, heads, page, dim, dtype=BF, device="cuda") for _ in range(2))
    assert k.numel() * 2 > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = [pages - 1, 3, pages - 2, pages // 2 + 7]
    for t in (k, v):
        for i in ids:
            t[0, i] = torch.randn(heads, page, dim, generator=g, device="cuda").to(BF)
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    ln = torch.tensor([4 * page - 5], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 8, dim, generator=g, device="cuda")
    out = bn.bitnet_attn_decode(bn.KvCache(k, v), 0, q, table, ln)
    small = torch.tensor([[0, 1, 2, 3]])
    ref = attn_ref(k[0, ids], v[0, ids], q, small, [4 * page - 6], [0], dim ** -0.5)
    check_attn(out, ref, DECODE_P[BF, True])


PROMPT = [
    # (cached before, new) per sequence, q_heads, kv_heads, dim, page, dtype, window, sinks
    ([(0, 1)], 2, 2, 64, 16, BF, 0, 0),
    ([(0, 77)], 16, 16, 96, 16, HF, 0, 0),
    ([(0, 200), (30, 0), (5, 3), (130, 129)], 8, 2, 128, 8, BF, 0, 0),
    ([(0, 300)], 4, 1, 100, 32, HF, 40, 4),
    ([(500, 65), (0, 64)], 8, 1, 128, 64, BF, 128, 16),
    ([(90, 150)], 6, 2, 64, 128, HF, 1, 0),
    ([(0, 140)], 10, 1, 128, 16, BF, 17, 1),
    ([(0, 260)], 1, 1, 4, 8, BF, 0, 0),
    ([(700, 30)], 12, 4, 112, 16, BF, 64, 200),
    ([(0, 513)], 3, 3, 128, 256, HF, 100, 130),
    ([(3, 20)], 40, 1, 36, 8, BF, 0, 0),
    ([(0, 9)], 144, 1, 32, 8, HF, 0, 0),
]


def prompt_args(spans):
    start = [0]
    for _, new in spans:
        start.append(start[-1] + new)
    seq = [i for i, (_, new) in enumerate(spans) for _ in range(new)]
    pos = [b + j for b, new in spans for j in range(new)]
    return torch.tensor(start, dtype=torch.int32, device="cuda"), seq, pos


def run_prompt(p, q, start, max_new, **kw):
    out = Guarded(q.shape, q.dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = bn.new_attn_workspace(q.shape[0], q.shape[1], p.cache.kv_heads, p.cache.head_dim)
    for _ in range(2):
        bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, start, max_new, out=out.t, workspace=ws, dev_status=status, **kw)
    torch.cuda.synchronize()
    assert out.intact() and int(status) == 0 and bn.bitnet_device_status() == 0
    return out.t


@pytest.mark.parametrize("spans,hq,hkv,dim,page,dtype,window,sinks", PROMPT)
def test_prompt_matches_64_bits(spans, hq, hkv, dim, page, dtype, window, sinks):
    p = Paged([b + n for b, n in spans], hkv, dim, page, dtype, seed=dim + len(spans))
    start, seq, pos = prompt_args(spans)
    q = p.queries(len(seq), hq, dim, dtype)
    out = run_prompt(p, q, start, max(n for _, n in spans), window=window, sinks=sinks)
    check_attn(out, p.ref(q, pos, seq, dim ** -0.5, window, sinks), PROMPT_P[dtype])


def test_prompt_single_tokens_agree_with_decode():
    p = Paged([90, 300, 31], 2, 128, 16, BF, seed=11)
    q = p.queries(3, 8, 128, BF)
    start = torch.arange(4, dtype=torch.int32, device="cuda")
    a, b = run_prompt(p, q, start, 1, window=50, sinks=3), run_decode(p, q, window=50, sinks=3)
    assert torch.allclose(a.float(), b.float(), rtol=2 ** -7, atol=2 ** -7)


SPLIT = [
    # few rows over long contexts: the blocks of a tile go to several CTAs and are joined
    ([(5000, 3)], 8, 2, 128, 64, BF, 0, 0),
    ([(2000, 40), (0, 5), (700, 1), (3, 130)], 8, 2, 128, 16, HF, 0, 0),
    ([(4100, 20)], 6, 1, 100, 32, HF, 1500, 7),
    ([(1500, 60)], 4, 4, 64, 128, BF, 0, 0),
    ([(1100, 9), (900, 3)], 160, 80, 32, 16, HF, 0, 0),        # 160 items: one for each SM, and some that are cut
]


@pytest.mark.parametrize("room", [True, False])
@pytest.mark.parametrize("spans,hq,hkv,dim,page,dtype,window,sinks", SPLIT)
def test_prompt_parts(spans, hq, hkv, dim, page, dtype, window, sinks, room):
    """With room for parts in the workspace and without; the workspace then serves decode, and the prompt again."""
    p = Paged([b + n for b, n in spans], hkv, dim, page, dtype, seed=dim + 3)
    start, seq, pos = prompt_args(spans)
    q = p.queries(len(seq), hq, dim, dtype)
    ws = bn.new_attn_workspace(len(seq) if room else 0, hq, hkv, dim)
    most = max(n for _, n in spans)
    call = lambda: bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, start, most, window=window, sinks=sinks, workspace=ws)
    out = call()
    check_attn(out, p.ref(q, pos, seq, dim ** -0.5, window, sinks), PROMPT_P[dtype])
    last = q[start[1:].long() - 1].contiguous()
    d = bn.bitnet_attn_decode(p.cache, p.layer, last, p.table, p.len, window=window, sinks=sinks, workspace=ws)
    assert torch.equal(d, run_decode(p, last, window=window, sinks=sinks))
    for _ in range(4):
        assert torch.equal(call(), out)
    assert int(ws[:bn.ATTN_WORKSPACE_HEAD].sum()) == 0


ROUNDS = [
    # more items than SMs, several times over: CTAs draw them, or take them in rounds when there is no workspace
    ([(100, 200), (0, 150), (637, 90)], 256, 64, 32, 32, BF, 120, 5),
    ([(3 * i, 1 + i % 9) for i in range(70)], 8, 8, 16, 8, HF, 0, 0),      # sequences beyond the 32 that are kept at hand
]


@pytest.mark.parametrize("room", [True, False])
@pytest.mark.parametrize("spans,hq,hkv,dim,page,dtype,window,sinks", ROUNDS)
def test_prompt_many_items(spans, hq, hkv, dim, page, dtype, window, sinks, room):
    p = Paged([b + n for b, n in spans], hkv, dim, page, dtype, seed=dim + 5)
    start, seq, pos = prompt_args(spans)
    q = p.queries(len(seq), hq, dim, dtype)
    ws = bn.new_attn_workspace(len(seq) if room else 0, hq, hkv, dim)
    most = max(n for _, n in spans)
    call = lambda: bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, start, most, window=window, sinks=sinks, workspace=ws)
    out = call()
    check_attn(out, p.ref(q, pos, seq, dim ** -0.5, window, sinks), PROMPT_P[dtype])
    for _ in range(4):
        assert torch.equal(call(), out)
    assert int(ws[:bn.ATTN_WORKSPACE_HEAD].sum()) == 0


def test_decode_one_workspace_for_calls_of_all_sizes():
    big = Paged([900 + 7 * i for i in range(40)], 4, 64, 16, BF, seed=21)
    small = Paged([30000], 1, 128, 64, HF, seed=22)
    ws = bn.new_attn_workspace(0, 16, 4, 64)
    qb, qs = big.queries(40, 16, 64, BF), small.queries(1, 4, 128, F32)
    wb, wsm = run_decode(big, qb), run_decode(small, qs)
    for _ in range(3):
        assert torch.equal(bn.bitnet_attn_decode(small.cache, 1, qs, small.table, small.len, workspace=ws), wsm)
        assert torch.equal(bn.bitnet_attn_decode(big.cache, 1, qb, big.table, big.len, workspace=ws), wb)
    assert int(ws[:bn.ATTN_WORKSPACE_HEAD].sum()) == 0


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_prompt_scales(scale):
    """Negative scales (the largest exponent belongs to the smallest product), 0 (all alike) and sharp ones."""
    p = Paged([150, 40], 2, 64, 16, BF, seed=14)
    start, seq, pos = prompt_args([(30, 120), (0, 40)])
    q = p.queries(160, 4, 64, BF)
    out = run_prompt(p, q, start, 120, scale=scale, window=77, sinks=2)
    check_attn(out, p.ref(q, pos, seq, scale, 77, 2), PROMPT_P[BF])


def test_prompt_rising_maxima():
    """Scores that grow along the context, so that the running maximum rises block after block."""
    p = Paged([1500], 1, 64, 64, BF, seed=15)
    grow = torch.linspace(0.2, 12.0, 1500, device="cuda")
    ids = p.table[0].long()
    for e in range(-(-1500 // 64)):
        rows = min(64, 1500 - e * 64)
        p.k[p.layer, ids[e], 0, :rows] = (p.k[p.layer, ids[e], 0, :rows].float().abs() * grow[e * 64:e * 64 + rows, None]).to(BF)
    start, seq, pos = prompt_args([(1300, 200)])
    q = p.queries(200, 2, 64, BF).abs()
    out = run_prompt(p, q, start, 200)
    check_attn(out, p.ref(q, pos, seq, 0.125, 0, 0), PROMPT_P[BF])
    d = run_decode(p, q[-1:].contiguous())
    check_attn(d, p.ref(q[-1:], [1499], [0], 0.125, 0, 0), DECODE_P[BF, False])


def test_prompt_strided_queries_negative_positions_and_stream():
    """Tokens before the start of the context (kv_len smaller than the number of new tokens) see nothing."""
    p = Paged([5, 60], 2, 64, 16, HF, seed=12, nhd=True)
    start = torch.tensor([0, 9, 40], dtype=torch.int32, device="cuda")
    pos = [5 - 9 + j for j in range(9)] + [60 - 31 + j for j in range(31)]
    fused = p.queries(40, 12, 64, HF).view(40, 768)
    q = fused[:, 256:].view(40, 8, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = run_prompt(p, q, start, 31)
    assert bool((out[:4] == 0).all())
    check_attn(out, p.ref(q, pos, [0] * 9 + [1] * 31, 0.125, 0, 0), PROMPT_P[HF])


def test_calls_without_workspace_on_another_stream():
    """The result and the workspace that the call makes belong to the stream that it runs on."""
    p = Paged([3000], 2, 128, 16, BF, seed=16)
    q = p.queries(1, 8, 128, BF)
    start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    want, side = run_decode(p, q), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        out = bn.bitnet_attn_decode(p.cache, p.layer, q, p.table, p.len, stream=side)
        junk = torch.full((1 << 22,), 7, dtype=torch.int32, device="cuda")     # would land in memory given back too early
        out2 = bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, start, 1, stream=side)
        side.synchronize()
        assert torch.equal(out, want) and torch.equal(out2, want)
        del junk, out, out2


def test_refusals():
    p = Paged([20], 2, 64, 16, BF, seed=13)
    q = p.queries(1, 4, 64, BF)
    ok = dict(table=p.table, kv_len=p.len)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_decode(p.cache, 2, q, **ok)                                   # no such layer
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_decode(p.cache, 0, p.queries(1, 3, 64, BF), **ok)             # heads not a multiple of kv heads
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_decode(p.cache, 0, q.to(HF), **ok)                            # another 16-bit type
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_decode(p.cache, 0, q, p.table.long(), p.len)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_decode(p.cache, 0, q, p.table[:0], p.len)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_decode(p.cache, 0, q, window=-1, **ok)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_decode(p.cache, 0, q, scale=float("nan"), **ok)
    with pytest.raises(bn.BitnetError, match="workspace"):
        bn.bitnet_attn_decode(p.cache, 0, q, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"), **ok)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_decode(p.cache, 0, q, out=torch.empty(1, 4, 64, device="cuda"), **ok)
    start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_prompt(p.cache, 0, q.float(), p.table, p.len, start, 1)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_attn_prompt(p.cache, 0, q, p.table, p.len, start, 2)               # max_new beyond the tokens
    with pytest.raises(bn.BitnetError):
        bn.KvCache(p.k, p.v[..., :32])
    with pytest.raises(bn.BitnetError):
        bn.KvCache(p.k.float(), p.v.float())
    x = torch.zeros(1, 4, 2, 24, 64, dtype=BF, device="cuda")
    with pytest.raises(bn.BitnetError, match="shape"):
        bn.KvCache(x, x.clone())                                                     # page size not a power of two
    x = torch.zeros(1, 4, 2, 16, 130, dtype=BF, device="cuda")
    with pytest.raises(bn.BitnetError):
        bn.KvCache(x, x.clone())
    x = torch.zeros(1, 4, 2, 16, 100, dtype=BF, device="cuda")
    with pytest.raises(bn.BitnetError):
        bn.KvCache(x, x.clone())                                                     # rows of 200 bytes
    assert bn.bitnet_attn_decode(p.cache, 0, q[:0], p.table[:0], p.len[:0]).shape == (0, 4, 64)
    empty = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert bn.bitnet_attn_prompt(p.cache, 0, empty, p.table, p.len, none, 0).shape == (0, 4, 64)
