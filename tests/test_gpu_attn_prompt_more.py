"""Prompts where whole items and items in parts meet, over pages that are missing, released or far into a large pool."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from kv_ref import attn_ref, check_attn
from test_gpu_kv_attn import BF, HF, PROMPT_P, Paged, prompt_args, run_prompt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF])
def test_prompt_whole_items_then_items_in_parts(dtype):
    """More items than SMs, of which those left over are cut: the boundary of the two, and the parts' places behind it."""
    sms, heads = torch.cuda.get_device_properties(0).multi_processor_count, 40
    # pairs of tiles (one per sequence) so that items = SMs + a few
    pairs = sms // heads + 1
    items, rest = pairs * heads, pairs * heads % sms
    spans = [(1500 - 90 * i, 3 + i) for i in range(pairs)]
    p = Paged([b + n for b, n in spans], heads, 16, 32, dtype, seed=51)
    start, seq, pos = prompt_args(spans)
    q = p.queries(len(seq), heads, 16, dtype)
    # the rest are the first sequence's (items go from the last one back), in at least two parts of four blocks of 128
    assert items > sms and 0 < rest < heads and sms // rest >= 2 and spans[0][0] >= 2 * 4 * 128
    ws = bn.new_attn_workspace(len(seq), heads, heads, 16)
    assert ws.numel() > bn.bitnet_attn_workspace_bytes(0, heads, heads, 16)
    call = lambda: bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, start, max(n for _, n in spans), workspace=ws)
    out = call()
    check_attn(out, p.ref(q, pos, seq, 0.25, 0, 0), PROMPT_P[dtype])
    for _ in range(4):
        assert torch.equal(call(), out)
    assert int(ws[:bn.ATTN_WORKSPACE_HEAD].sum()) == 0 and bn.bitnet_device_status() == 0


@pytest.mark.parametrize("dim,new", [(64, 60), (100, 60), (128, 3), (128, 2)])
def test_prompt_bad_pages_are_reported_and_not_read(dim, new):
    p = Paged([100, 90], 2, dim, 16, BF, seed=52)
    start, seq, pos = prompt_args([(100 - new, new), (90 - new, new)])
    q = p.queries(2 * new, 4, dim, BF)
    good = run_prompt(p, q, start, new)
    for bad in (-1, p.cache.num_pages, 2 ** 31 - 1, -2 ** 31):
        table = p.table.clone()
        table[0, 2] = bad
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = bn.bitnet_attn_prompt(p.cache, p.layer, q, table, p.len, start, new, dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == 7 and torch.equal(out[new:], good[new:]) and torch.isfinite(out[:new]).all()
        before = sum(x < 32 for x in pos[:new])                    # tokens before that page do not see it
        assert torch.equal(out[:before], good[:before])


@pytest.mark.parametrize("room", [True, False])
@pytest.mark.parametrize("sinks", [0, 20])
def test_prompt_over_released_pages(sinks, room):
    """Pages between the sinks and the first new token's window have been given up: not read, not reported."""
    window, spans = 150, [(900, 40), (30, 25)]
    p = Paged([b + n for b, n in spans], 2, 128, 16, HF, seed=53)
    start, seq, pos = prompt_args(spans)
    q = p.queries(len(seq), 8, 128, HF)
    refs = torch.zeros(p.cache.num_pages, dtype=torch.int32, device="cuda")
    refs[p.table[p.table >= 0].long()] = 1
    before = torch.tensor([b for b, _ in spans], dtype=torch.int32, device="cuda")
    whole = p.table.clone()
    bn.bitnet_kv_trim(refs, p.table, before + 1, 16, window, sinks)
    assert int((p.table < 0).sum()) > int((whole < 0).sum())
    out = run_prompt(p, q, start, 40, window=window, sinks=sinks)
    p.table = whole
    check_attn(out, p.ref(q, pos, seq, 128 ** -0.5, window, sinks), PROMPT_P[HF])
    ws = bn.new_attn_workspace(len(seq) if room else 0, 8, 2, 128)
    again = bn.bitnet_attn_prompt(p.cache, p.layer, q, whole, p.len, start, 40, window=window, sinks=sinks, workspace=ws)
    assert torch.equal(again, out) or not room
    check_attn(again, p.ref(q, pos, seq, 128 ** -0.5, window, sinks), PROMPT_P[HF])


def test_prompt_offsets_beyond_32_bits():
    """Pools of more than 2^32 bytes each: the last pages."""
    pages, page, heads, dim = 70000, 64, 4, 128
    k, v = (torch.empty(1, pages, heads, page, dim, dtype=BF, device="cuda") for _ in range(2))
    assert k.numel() * 2 > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(2)
    ids = [pages - 1, 3, pages - 2, pages // 2 + 7]
    for t in (k, v):
        for i in ids:
            t[0, i] = torch.randn(heads, page, dim, generator=g, device="cuda").to(BF)
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    n, new = 4 * page - 5, 9
    ln, start = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, new], dtype=torch.int32, device="cuda")
    q = torch.randn(new, 8, dim, generator=g, device="cuda").to(BF)
    out = bn.bitnet_attn_prompt(bn.KvCache(k, v), 0, q, table, ln, start, new)
    ref = attn_ref(k[0, ids], v[0, ids], q, torch.tensor([[0, 1, 2, 3]]), list(range(n - new, n)), [0] * new, dim ** -0.5)
    check_attn(out, ref, PROMPT_P[BF])
