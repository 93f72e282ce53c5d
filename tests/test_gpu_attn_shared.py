"""Attention of sequences that share prefixes against a 64-bit implementation and against the decode kernel: group and head layouts, prefixes that end
inside a page or a tile, sequences shorter than their prefix, windows and sinks, idle rows, bad pages, calls that give up."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from helpers import Guarded
from kv_ref import attn_ref, check_attn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=["as it goes", "always shared"])
def path(request):
    """Calls of these sizes are mostly ones that the decode kernel takes: every test runs a second time without it."""
    bn.bitnet_debug_attn_shared(request.param == "always shared")
    yield request.param
    bn.bitnet_debug_attn_shared(False)

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
PROMPT_P = {BF: 2.0 ** -8, HF: 2.0 ** -11}       # relative rounding of the prefix's probabilities


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Groups:
    """groups: (prefix, tokens of each sequence).  Full pages of a prefix are shared, the page filled in part is copied; unused places of the pool are NaN."""

    def __init__(self, groups, kv_heads, dim, page, dtype, seed=0, nhd=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g, self.lens = g, [n for _, ns in groups for n in ns]
        rows, at = [], 0
        for prefix, ns in groups:
            full = min(prefix, max(ns, default=0)) // page
            shared, at = list(range(at, at + full)), at + full
            for n in ns:
                more = max(0, -(-n // page) - full)
                rows.append(shared + list(range(at, at + more)))
                at += more
        pages, dp = at + 3, -(-dim // 8) * 8
        shape = (2, pages, page, kv_heads, dp) if nhd else (2, pages, kv_heads, page, dp)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        if nhd:
            self.k, self.v = self.k.permute(0, 1, 3, 2, 4), self.v.permute(0, 1, 3, 2, 4)
        self.k, self.v = self.k[..., :dim], self.v[..., :dim]
        order = torch.randperm(pages, generator=g, device="cuda").cpu().int()
        self.table = torch.full((len(rows), max(map(len, rows)) + 1), -1, dtype=torch.int32)
        i = 0
        for prefix, ns in groups:
            of_first = None
            for j, n in enumerate(ns):
                r = rows[i]
                self.table[i, :len(r)] = order[r]
                for t in (self.k, self.v):
                    for e in range(-(-n // page)):
                        c = min(page, n - e * page)
                        x = torch.randn(kv_heads, c, dim, generator=g, device="cuda").to(dtype)
                        p = int(order[r[e]])
                        if j and (e + 1) * page <= prefix and bool(torch.isfinite(t[1, p, :, :c]).all()):
                            continue             # shared, and there
                        if j and e * page < prefix:
                            keep = min(prefix - e * page, c, of_first - e * page)
                            if keep > 0:
                                x[:, :keep] = t[1, int(order[first_row[e]]), :, :keep]
                        t[1, p, :, :c] = x
                if j == 0:
                    of_first, first_row = n, r
                i += 1
        self.table, self.len = self.table.cuda(), ints(self.lens)
        self.start = ints([sum(len(ns) for _, ns in groups[:k]) for k in range(len(groups) + 1)])
        self.prefix = ints([p for p, _ in groups])
        self.cache = bn.KvCache(self.k, self.v)

    def queries(self, heads, scale=1.0):
        return (torch.randn(len(self.lens), heads, self.cache.head_dim, generator=self.g, device="cuda") * scale).to(self.cache.dtype)

    def run(self, q, **kw):
        out, status = Guarded(q.shape, q.dtype), ints([0])
        ws = bn.new_attn_shared_workspace(q.shape[0], q.shape[1], self.cache.kv_heads, self.cache.head_dim)
        again = []
        for _ in range(3):                       # the workspace is left as it was found; the same bits every time
            bn.bitnet_attn_shared(self.cache, 1, q, self.table, self.len, self.start, self.prefix, out=out.t, workspace=ws, dev_status=status, **kw)
            again.append(out.t.clone())
        torch.cuda.synchronize()
        assert out.intact() and int(status) == 0 and bn.bitnet_device_status() == 0 and int(ws[:bn.ATTN_WORKSPACE_HEAD].sum()) == 0
        assert torch.equal(again[0], again[1]) and torch.equal(again[0], again[2])
        return out.t

    def check(self, q, scale=None, window=0, sinks=0):
        scale = self.cache.head_dim ** -0.5 if scale is None else scale
        out = self.run(q, scale=scale, window=window, sinks=sinks)
        ref = attn_ref(self.k[1], self.v[1], q, self.table, [n - 1 for n in self.lens], range(len(self.lens)), scale, window, sinks)
        check_attn(out, ref, PROMPT_P[self.cache.dtype])
        assert all(bool((out[i] == 0).all()) for i, n in enumerate(self.lens) if n == 0)
        return out


CASES = [
    # groups, q_heads, kv_heads, dim, page, dtype, window, sinks
    ([(64, [70])], 1, 1, 64, 16, BF, 0, 0),
    ([(128, [128, 129, 200])], 8, 2, 128, 16, BF, 0, 0),        # nothing of its own: the prefix alone
    ([(700, [720] * 8)], 32, 8, 128, 16, BF, 0, 0),
    ([(704, [710 + 9 * i for i in range(40)])], 16, 2, 128, 64, BF, 0, 0),     # 320 rows: two pairs of tiles
    ([(300, [310 + i for i in range(20)]), (0, [5, 77, 200]), (1, [2, 2])], 16, 16, 96, 32, HF, 0, 0),
    ([(333, [340, 345, 401])], 4, 4, 100, 32, HF, 0, 0),        # prefix ends inside a page; odd rows
    ([(77, [90, 99])] * 40, 8, 2, 64, 8, BF, 0, 0),             # more groups than are kept at hand
    ([(500, [500, 0, 300, 700, 20])], 8, 2, 128, 16, BF, 0, 0), # shorter than the prefix, idle
    ([(500, [0, 0]), (0, [0]), (30, [31])], 4, 2, 64, 16, HF, 0, 0),
    ([(900, [901, 1000, 1400, 990])], 8, 2, 128, 16, BF, 200, 0),
    ([(900, [901, 1000, 1400, 990])], 8, 2, 128, 16, BF, 200, 5),
    ([(900, [901, 950]), (640, [700, 640])], 8, 8, 64, 32, HF, 1000, 7),
    ([(900, [1500, 1400])], 8, 2, 128, 16, BF, 100, 70),        # windows beyond the prefix: its sinks alone
    ([(900, [1500, 1400])], 8, 2, 128, 16, BF, 100, 0),         # nothing of it
    ([(40, [600, 300])], 8, 2, 128, 16, BF, 100, 70),           # sinks beyond the prefix
    ([(300, [400, 350])], 8, 2, 128, 16, BF, 60, 5000),         # sinks beyond everything
    ([(150, [160, 170])], 160, 1, 32, 8, HF, 0, 0),             # more heads of a kv head than a tile has rows
    ([(260, [270, 300])], 6, 2, 4, 8, HF, 0, 0),                # smallest head
    ([(260, [270, 300, 261])], 20, 2, 112, 256, BF, 0, 0),
]


@pytest.mark.parametrize("groups,hq,hkv,dim,page,dtype,window,sinks", CASES)
def test_matches_64_bits(groups, hq, hkv, dim, page, dtype, window, sinks):
    s = Groups(groups, hkv, dim, page, dtype, seed=dim + len(groups))
    s.check(s.queries(hq), window=window, sinks=sinks)


def test_long_prefix_over_all_ctas():
    for n, hkv in ((3, 1), (50, 8)):
        s = Groups([(9000, [9001 + 37 * i for i in range(n)])], hkv, 128, 64, BF, seed=n)
        s.check(s.queries(4 * hkv))


def test_more_items_than_ctas():
    s = Groups([(130 + i, [200 + i, 300]) for i in range(70)], 8, 32, 16, HF, seed=3)
    s.check(s.queries(8))


def test_more_groups_and_sequences_than_threads():
    """More than are looked at at a time, some groups without sequences, or shorter than their prefix; with and without a window."""
    s = Groups([(37 * (i % 3), [40 + i % 90] * (i % 3)) for i in range(400)], 2, 16, 8, BF, seed=4)
    q = s.queries(4)
    for window, sinks in ((0, 0), (30, 2)):
        s.check(q, window=window, sinks=sinks)


def test_many_small_probabilities():
    """One token far ahead of many: each of those has a probability below fp16's normal numbers, together they have most of the weight."""
    s = Groups([(20032, [20040, 40000])], 1, 64, 64, HF, seed=16)
    s.k[1, :, :, :, 1:] = 0
    s.k[1, :, :, :, 0] = 0
    s.k[1, s.table[0, 0].long(), 0, 5, 0] = 9.5 * 8
    q = torch.zeros_like(s.queries(2))
    q[..., 0] = 1
    s.check(q)


def test_scales_and_rising_maxima():
    s = Groups([(300, [310, 420, 300])], 2, 64, 16, BF, seed=4)
    for scale in (-0.3, 0.0, 2.0):
        s.check(s.queries(8), scale=scale)
    s = Groups([(960, [1100, 1010])], 1, 64, 64, HF, seed=5)      # (full pages: a change in them is a change for both)
    for e in range(1100 // 64 + 1):
        page = s.table[0, e].long()
        s.k[1, page] = s.k[1, page].abs() * (0.2 + 0.3 * e)
    s.check(s.queries(4).abs())


def test_agrees_with_decode():
    s = Groups([(500, [510, 777, 640]), (64, [65, 90])], 4, 128, 16, BF, seed=6)
    q = s.queries(16)
    a = s.run(q, window=300, sinks=3)
    b = bn.bitnet_attn_decode(s.cache, 1, q, s.table, s.len, window=300, sinks=3)
    assert torch.allclose(a.float(), b.float(), rtol=2 ** -7, atol=2 ** -7)


def test_the_first_sequences_pages_are_read(path):
    """A prefix is read through the first sequence's row: where the decode kernel does not take the call, other rows' pages there are not looked at."""
    s = Groups([(320, [330, 400, 350])], 2, 64, 16, BF, seed=7)
    q = s.queries(8)
    want = s.run(q)
    if path == "always shared":
        s.table[1:, :320 // 16] = -1
        assert torch.equal(s.run(q), want)


def test_calls_go_by_what_there_is_to_save():
    """Few tokens, or groups of one or two: the decode kernel's results, bit for bit; many: not."""
    for groups, alike in (([(500, [510] * 4)], True), ([(4000, [4010, 4100])] * 3, True), ([(4096, [4100] * 24)], False)):
        s = Groups(groups, 8, 128, 16, BF, seed=18)
        q = s.queries(16)
        bn.bitnet_debug_attn_shared(False)
        a, b = s.run(q), bn.bitnet_attn_decode(s.cache, 1, q, s.table, s.len)
        assert torch.equal(a, b) == alike
        assert torch.allclose(a.float(), b.float(), rtol=2 ** -7, atol=2 ** -7)


def test_strides_other_pool_order_stream_and_one_workspace():
    s = Groups([(200, [210, 260, 333])], 4, 100, 16, BF, seed=8, nhd=True)
    wide = s.queries(24)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.check(wide[:, 8:24])
    big = Groups([(2000, [2100 + i for i in range(30)])], 2, 128, 16, HF, seed=9)
    ws = bn.new_attn_shared_workspace(30, 16, 4, 128)
    q, qb = s.queries(16), big.queries(8)
    a, b = s.run(q), big.run(qb)
    d = bn.bitnet_attn_decode(big.cache, 1, qb, big.table, big.len)
    for _ in range(3):
        assert torch.equal(bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, workspace=ws), a)
        assert torch.equal(bn.bitnet_attn_shared(big.cache, 1, qb, big.table, big.len, big.start, big.prefix, workspace=ws), b)
        assert torch.equal(bn.bitnet_attn_decode(big.cache, 1, qb, big.table, big.len, workspace=ws), d)
    torch.cuda.synchronize()
    out = bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, stream=side)
    side.synchronize()
    assert torch.equal(out, a)


def test_bad_pages_are_reported():
    s = Groups([(320, [330, 400]), (64, [70])], 2, 64, 16, BF, seed=10)
    q = s.queries(8)
    good = s.run(q)
    for row, entry in ((0, 3), (1, 22)):
        for bad in (-1, s.cache.num_pages, 2 ** 31 - 1, -2 ** 31):
            table, status = s.table.clone(), ints([0])
            table[row, entry] = bad
            out = bn.bitnet_attn_shared(s.cache, 1, q, table, s.len, s.start, s.prefix, dev_status=status)
            torch.cuda.synchronize()
            assert int(status) == 7 and torch.equal(out[2], good[2]) and torch.isfinite(out).all()


def test_a_first_sequence_without_the_prefixs_pages_is_reported(path):
    """The first sequence has 300 of the 500 tokens that the others have: their tokens from 300 on have no page to be read from."""
    s = Groups([(500, [300, 0, 500, 700, 20])], 2, 128, 16, BF, seed=129)
    s.table[0, -(-300 // 16):] = -1
    status = ints([0])
    out = bn.bitnet_attn_shared(s.cache, 1, s.queries(8), s.table, s.len, s.start, s.prefix, dev_status=status)
    torch.cuda.synchronize()
    assert (int(status) == 7 or path != "always shared") and torch.isfinite(out).all() and bool((out[1] == 0).all())


def test_arrays_of_groups_that_are_not_as_they_should():
    """Sequences in no group are taken by themselves; prefixes below 0 and beyond the table are cut; nothing outside is read."""
    s = Groups([(320, [330, 400, 350]), (64, [70, 90])], 2, 64, 16, BF, seed=11)
    q = s.queries(8)
    alone = bn.bitnet_attn_decode(s.cache, 1, q, s.table, s.len)
    run = lambda start, prefix: bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, ints(start), ints(prefix))
    for start, prefix in (([0, 5], [-7]), ([2, 2], [100]), ([9, 12], [100]), ([-5, -2], [100]), ([5, 0], [64]), ([0, 0, 0], [5, 5])):
        assert torch.allclose(run(start, prefix).float(), alone.float(), rtol=2 ** -7, atol=2 ** -7), start
    got = run([1, 3], [320])                     # sequences 0, 3, 4 in none
    assert torch.allclose(got.float(), alone.float(), rtol=2 ** -7, atol=2 ** -7)
    got = run([0, 1, 9], [2 ** 31 - 1, 0])       # the whole table is sequence 0's prefix; a group that ends beyond the sequences
    assert torch.allclose(got.float(), alone.float(), rtol=2 ** -7, atol=2 ** -7)


def test_length_beyond_the_table():
    s = Groups([(60, [64, 64])], 1, 64, 16, BF, seed=12)
    s.table = s.table[:, :4].contiguous()
    q = s.queries(2)
    want = s.run(q)
    s.len[1] = 2 ** 31 - 1
    assert torch.equal(s.run(q), want)


def test_lengths_below_zero():
    """Idle rows, however far below: they see nothing, and the others of their group what they see without them."""
    s = Groups([(200, [210, 260, 333])], 2, 64, 16, BF, seed=17)
    q = s.queries(8)
    for window in (0, 150):
        want = s.run(q, window=window)
        for n in (0, -1, -2 ** 31):
            s.len[1] = n
            out = s.run(q, window=window)
            assert bool((out[1] == 0).all()) and all(torch.allclose(out[i].float(), want[i].float(), rtol=2 ** -7, atol=2 ** -7) for i in (0, 2))
        s.len[1] = 260


def test_graph():
    s = Groups([(200, [210, 260, 333]), (0, [40])], 4, 128, 16, BF, seed=13)
    q = s.queries(16)
    ws, out = bn.new_attn_shared_workspace(4, 16, 4, 128), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, out=out, workspace=ws)
    q.mul_(-0.5)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, s.run(q))


@pytest.mark.parametrize("tile", [0, 1])
def test_calls_that_give_up(tile):
    """Every CTA's wait runs out: the call ends, the status says so, and the next call is whole again.  (Four blocks for each CTA.)"""
    s = Groups([(9000, [9200, 9300, 9250])], 8, 64, 64, BF, seed=14)
    q = s.queries(16)
    want = s.run(q)
    ws = bn.new_attn_shared_workspace(3, 16, 8, 64)
    bn.bitnet_debug_attn_give_up(tile)
    try:
        bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, workspace=ws)
        assert bn.bitnet_device_status() == 6
    finally:
        bn.bitnet_debug_attn_give_up(-1)
        bn.bitnet_device_status_clear()
    ws[:bn.ATTN_WORKSPACE_HEAD].zero_()
    assert torch.equal(bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, workspace=ws), want)


def test_refusals():
    s = Groups([(100, [110, 120])], 2, 64, 16, BF, seed=15)
    q = s.queries(4)
    ok = dict(cache=s.cache, layer=1, q=q, table=s.table, kv_len=s.len, group_start=s.start, prefix_len=s.prefix)
    for bad in (dict(q=q.float()), dict(q=q.to(HF)), dict(q=q[:, :3]), dict(layer=2), dict(group_start=s.start.long()), dict(group_start=s.start[:1]), dict(group_start=s.start[:0]),
                dict(prefix_len=s.prefix[:0]), dict(window=-1), dict(scale=float("inf")), dict(table=s.table[:1]),
                dict(workspace=bn.new_attn_workspace(0, 4, 2, 64)), dict(out=torch.empty(2, 4, 64, device="cuda"))):
        with pytest.raises(bn.BitnetError):
            bn.bitnet_attn_shared(**dict(ok, **bad))
    assert bn.bitnet_attn_shared(s.cache, 1, q[:0], s.table[:0], s.len[:0], ints([0]), ints([])).shape == (0, 4, 64)
