"""Calls in which a wait is taken for one that has run out (on the host's order: nothing hangs, and every other wait is as it is):
they end, they are reported, and the next call is right."""
import time

import pytest
import torch

import paper_2502_11880_b200 as bn
from test_gpu_kv_attn import BF, F32, HF, Paged, prompt_args

pytestmark = pytest.mark.gpu


@pytest.fixture
def give_up():
    yield bn.bitnet_debug_attn_give_up
    bn.bitnet_debug_attn_give_up(-1)
    torch.cuda.synchronize()
    bn.bitnet_device_status_clear()


def gives_up(call):
    """The call ends within seconds (no wait was left that runs out by itself: those take a quarter of a minute) and is reported."""
    torch.cuda.synchronize()
    t = time.perf_counter()
    call()
    torch.cuda.synchronize()
    assert time.perf_counter() - t < 8
    assert bn.bitnet_device_status() == 6
    bn.bitnet_device_status_clear()
    assert bn.bitnet_device_status() == 0


DECODE = [
    ([3000, 70, 1900], 8, 2, 128, 16, BF, BF),
    ([40003], 8, 1, 128, 64, BF, F32),                     # one row on all SMs, joined
    ([2000, 900], 12, 12, 100, 32, HF, F32),               # rows by plain bulk copies
    ([500] * 90, 4, 4, 64, 8, HF, HF),                     # several rows to a CTA
]


@pytest.mark.parametrize("tile", [0, 1, 3, 7])
@pytest.mark.parametrize("lens,hq,hkv,dim,page,dtype,io", DECODE)
def test_decode_that_gives_up(give_up, lens, hq, hkv, dim, page, dtype, io, tile):
    p = Paged(lens, hkv, dim, page, dtype, seed=61)
    q = p.queries(len(lens), hq, dim, io)
    ws = bn.new_attn_workspace(0, hq, hkv, dim)
    call = lambda: bn.bitnet_attn_decode(p.cache, p.layer, q, p.table, p.len, workspace=ws)
    want = call()
    deepest = tile < 2 or sum(-(-n // 64) for n in lens) * hkv > 148 * tile     # does some CTA come to that tile?
    give_up(tile)
    if deepest:
        gives_up(call)
    give_up(-1)
    bn.bitnet_workspace_init(ws[:bn.ATTN_WORKSPACE_HEAD])
    assert torch.equal(call(), want) and bn.bitnet_device_status() == 0


PROMPT = [
    ([(0, 600), (300, 200)], 8, 2, 128, 16, BF, True),
    ([(0, 600), (300, 200)], 8, 2, 128, 16, BF, False),
    ([(9000, 20)], 4, 1, 64, 64, HF, True),                # an item in parts
    ([(100, 300)] * 5, 64, 32, 32, 32, BF, True),          # several items to a CTA
    ([(100, 300)] * 5, 64, 32, 32, 32, BF, False),
]


@pytest.mark.parametrize("block", [0, 1, 2, 3])                # every case has a CTA with four blocks
@pytest.mark.parametrize("spans,hq,hkv,dim,page,dtype,room", PROMPT)
def test_prompt_that_gives_up(give_up, spans, hq, hkv, dim, page, dtype, room, block):
    p = Paged([b + n for b, n in spans], hkv, dim, page, dtype, seed=62)
    start, seq, _ = prompt_args(spans)
    q, most = p.queries(len(seq), hq, dim, dtype), max(n for _, n in spans)
    ws = bn.new_attn_workspace(len(seq) if room else 0, hq, hkv, dim)
    call = lambda: bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, start, most, workspace=ws)
    want = call()
    give_up(block)
    gives_up(call)
    give_up(-1)
    bn.bitnet_workspace_init(ws[:bn.ATTN_WORKSPACE_HEAD])
    assert torch.equal(call(), want) and bn.bitnet_device_status() == 0
    assert int(ws[:bn.ATTN_WORKSPACE_HEAD].sum()) == 0
