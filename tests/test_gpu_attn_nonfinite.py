"""NaN, infinities and huge values where queries see them and where they do not: a NaN that a query sees is in its result, by whichever
kernel serves the call, and what a query does not see leaves its result as it is."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from test_gpu_kv_attn import BF, HF, Paged, prompt_args

pytestmark = pytest.mark.gpu


def prompt(p, q, start, most, room=True, **kw):
    ws = bn.new_attn_workspace(q.shape[0] if room else 0, q.shape[1], p.cache.kv_heads, p.cache.head_dim)
    out = bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, start, most, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert bn.bitnet_device_status() == 0 and int(ws[:bn.ATTN_WORKSPACE_HEAD].sum()) == 0
    return out


def at(p, seq, token):
    """Page and row of a token."""
    return int(p.table[seq, token // p.cache.page_size]), token % p.cache.page_size


@pytest.mark.parametrize("column", list(range(64, 80)) + [(78, 79), (14, 30)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_prompt_nan_key_makes_nan_of_the_rows_that_see_it(dtype, column):
    """A key at every place of a group of 16 columns, whatever way that column's exponential is taken."""
    p = Paged([200], 2, 64, 16, dtype, seed=31)
    start, _, _ = prompt_args([(0, 200)])
    q = p.queries(200, 4, 64, dtype)
    clean = prompt(p, q, start, 200)
    columns = column if isinstance(column, tuple) else (column,)
    for c in columns:
        page, row = at(p, 0, c)
        p.k[p.layer, page, 0, row, 5] = float("nan")
    out = prompt(p, q, start, 200)
    first = min(columns)
    assert torch.equal(out[:first], clean[:first])                 # before the key
    assert torch.equal(out[:, 2:], clean[:, 2:])                   # heads of the other kv head
    assert bool(out[first:, :2].isnan().all())


@pytest.mark.parametrize("dtype", [BF, HF])
def test_prompt_hidden_tokens_have_no_weight(dtype):
    """Values as large as the type holds, beside queries that do not see them."""
    p = Paged([150], 1, 64, 16, dtype, seed=32)
    start, _, _ = prompt_args([(0, 150)])
    q = p.queries(150, 3, 64, dtype)
    for window, sinks in ((0, 0), (20, 2)):
        clean = prompt(p, q, start, 150, window=window, sinks=sinks)
        for column in (46, 47, 63, 78):
            page, row = at(p, 0, column)
            kept = p.v[p.layer, page, 0, row].clone()
            p.v[p.layer, page, 0, row] = torch.finfo(dtype).max
            out = prompt(p, q, start, 150, window=window, sinks=sinks)
            p.v[p.layer, page, 0, row] = kept
            assert torch.equal(out[:column], clean[:column])
            if window:
                assert torch.equal(out[column + window:], clean[column + window:])


SPANS = [
    ([(0, 200), (30, 5)], True),
    ([(0, 200), (30, 5)], False),
    ([(5000, 3)], True),                                           # blocks of the tile on several CTAs, joined
    ([(5000, 3)], False),
    ([(300, 2), (40, 1)], True),                                   # the kernel of single tokens
]


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("spans,room", SPANS)
def test_prompt_query_whose_scores_are_all_nan(spans, room, dtype, value):
    """A NaN in a query, or infinities whose products cancel: NaN for that query, and nothing else changes."""
    p = Paged([b + n for b, n in spans], 2, 64, 16, dtype, seed=33)
    start, seq, _ = prompt_args(spans)
    q, most = p.queries(len(seq), 8, 64, dtype), max(n for _, n in spans)
    clean = prompt(p, q, start, most, room)
    t = len(seq) // 2
    for heads in ([3], list(range(8))):
        bad = q.clone()
        bad[t, heads] = value
        out = prompt(p, bad, start, most, room)
        others = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
        others[t, heads] = False
        assert bool(out[~others].isnan().all())
        assert torch.equal(out[others], clean[others])


@pytest.mark.parametrize("room", [True, False])
def test_prompt_first_token_with_a_nan_key(room):
    """The first token sees itself alone: all that it sees is NaN."""
    p = Paged([40], 1, 64, 16, BF, seed=34)
    start, _, _ = prompt_args([(0, 40)])
    q = p.queries(40, 2, 64, BF)
    page, row = at(p, 0, 0)
    p.k[p.layer, page, 0, row] = float("nan")
    assert bool(prompt(p, q, start, 40, room).isnan().all())
    d = bn.bitnet_attn_decode(p.cache, p.layer, q[-1:].contiguous(), p.table, p.len)
    assert bool(d.isnan().all())


@pytest.mark.parametrize("room", [True, False])
def test_prompt_part_whose_keys_are_all_nan(room):
    """The first four blocks of 128 tokens, which one CTA has by itself where the row's blocks go to several."""
    p = Paged([6000], 1, 64, 64, BF, seed=35)
    start, _, _ = prompt_args([(5995, 5)])
    q = p.queries(5, 4, 64, BF)
    clean = prompt(p, q, start, 5, room, window=5000)
    for e in range(512 // 64):
        p.k[p.layer, int(p.table[0, e])] = float("nan")
    assert bool(prompt(p, q, start, 5, room).isnan().all())
    assert torch.equal(prompt(p, q, start, 5, room, window=5000), clean)      # those keys are outside the window
