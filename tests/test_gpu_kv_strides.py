"""Tensors with dimensions of one entry, whose strides say nothing: odd ones there are taken as they are."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from test_gpu_kv_attn import BF, Paged
from test_gpu_kv_pages import i32

pytestmark = pytest.mark.gpu


def odd(t, *dims):
    """The same values with strides of 3 in these dimensions, which have one entry."""
    stride = list(t.stride())
    for d in dims:
        assert t.shape[d] == 1
        stride[d] = 3
    return t.as_strided(t.shape, stride)


def test_one_token_and_one_head():
    p = Paged([70], 1, 64, 16, BF, seed=71)
    q, start = p.queries(1, 1, 64, BF), i32([0, 1])
    want = bn.bitnet_attn_decode(p.cache, p.layer, q, p.table, p.len)
    assert torch.equal(bn.bitnet_attn_decode(p.cache, p.layer, odd(q, 0, 1), p.table, p.len), want)
    assert torch.equal(bn.bitnet_attn_prompt(p.cache, p.layer, odd(q, 0, 1), p.table, p.len, start, 1), want)
    q = p.queries(5, 1, 64, BF)
    want = bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, i32([0, 5]), 5)
    assert torch.equal(bn.bitnet_attn_prompt(p.cache, p.layer, odd(q, 1), p.table, p.len, i32([0, 5]), 5), want)
    k, v = torch.randn(1, 1, 64, device="cuda"), torch.randn(1, 1, 64, device="cuda")
    bn.bitnet_kv_append(p.cache, p.layer, odd(k, 0, 1), v, p.table, p.len)       # k and v differ there
    page, row = int(p.table[0, 4]), 5
    assert torch.equal(p.k[p.layer, page, 0, row], k.view(64).to(BF)) and torch.equal(p.v[p.layer, page, 0, row], v.view(64).to(BF))


def test_one_layer_and_one_kv_head():
    k, v = (torch.randn(1, 6, 1, 8, 64, device="cuda").to(BF) for _ in range(2))
    q, table, length = torch.randn(1, 4, 64, device="cuda"), i32([[3, 1, 5]]), i32([20])
    want = bn.bitnet_attn_decode(bn.KvCache(k, v), 0, q, table, length)
    assert torch.equal(bn.bitnet_attn_decode(bn.KvCache(odd(k, 0, 2), v), 0, q, table, length), want)


def test_k_and_v_of_different_heads_are_refused():
    p = Paged([20], 2, 64, 16, BF, seed=72)
    k = torch.zeros(1, 2, 64, device="cuda")
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_append(p.cache, 0, k, k[:, :1], p.table, p.len)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_append(p.cache, 0, k.expand(3, 2, 64), torch.zeros(3, 2, 64, device="cuda"), p.table[:1].expand(3, -1).contiguous(),
                            p.len.expand(3).contiguous())                       # strides that differ
