"""NaN and huge values where queries see them and where they do not: a NaN that a query sees is in its result, by whichever
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
