"""The cache and the attention between the ternary linears of a layer, as the example runs them."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from paper_2502_11880_b200 import run_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("args", [
    [],                                                                                                 # 8B-shaped layer
    ["--hidden", "3200", "--heads", "32", "--kv-heads", "32", "--prompt", "77", "--steps", "9", "--samples", "2", "--window", "40", "--page", "8"],
    ["--hidden", "1536", "--heads", "16", "--kv-heads", "16", "--prompt", "1", "--steps", "3", "--samples", "1", "--window", "2", "--sinks", "0"],
])
def test_layer(args):
    worst, same, status = run_decode.main(args)
    # fp32 queries and outputs over bf16 pages: probabilities of 24 bits, scores and sums in fp32 over a few hundred tokens
    assert worst < 2e-6 and same and status == 0


def test_calls_between_framework_kernels_in_one_stream():
    """Append and attention right behind the linear that writes their inputs, many times, without a synchronisation between:
    every kernel waits for what it reads."""
    layer = run_decode.Layer(1536, 16, 16, seed=3)
    cache = bn.new_kv_cache(1, 40, 16, 16, 96)
    ints = dict(dtype=torch.int32, device="cuda")
    table = torch.arange(40, **ints).view(2, 20)
    length = torch.zeros(2, **ints)
    ws = bn.new_attn_workspace(0, 16, 16, 96)
    xs = [torch.randn(2, 1536, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda") for i in range(60)]

    def run(wait):
        length.zero_()
        outs = []
        for x in xs:
            length.add_(1)
            q, k, v = layer.qkv(x)
            if wait:
                torch.cuda.synchronize()
            bn.bitnet_kv_append(cache, 0, k, v, table, length)
            if wait:
                torch.cuda.synchronize()
            y = bn.bitnet_attn_decode(cache, 0, q, table, length, workspace=ws)
            outs.append(layer.linear(1, y.view(2, -1)))
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return outs

    want = run(True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(False), want))


def test_decode_step_in_a_graph():
    """A captured step follows the books that change between replays."""
    cache = bn.new_kv_cache(1, 32, 2, 16, 64)
    ints = dict(dtype=torch.int32, device="cuda")
    refs, table = torch.zeros(32, **ints), torch.full((2, 16), -1, **ints)
    old, length = torch.zeros(2, **ints), torch.zeros(2, **ints)
    q, k, v = (torch.zeros(2, h, 64, device="cuda") for h in (4, 2, 2))
    out, ws = torch.zeros(2, 4, 64, device="cuda"), bn.new_attn_workspace(0, 4, 2, 64)

    def step():
        old.copy_(length)
        length.add_(1)
        bn.bitnet_kv_reserve(refs, table, old, length, 16)
        bn.bitnet_kv_append(cache, 0, k, v, table, length)
        bn.bitnet_attn_decode(cache, 0, q, table, length, out=out, workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    refs.zero_()
    table.fill_(-1)
    length.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    keys, values = [], []
    for i in range(40):
        g = torch.Generator(device="cuda").manual_seed(i)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        keys.append(k.to(torch.bfloat16).double())
        values.append(v.to(torch.bfloat16).double())
        graph.replay()
        kk, vv = torch.stack(keys, 2), torch.stack(values, 2)                         # seqs, heads, tokens, dim
        s = torch.einsum("bhgd,bhtd->bhgt", q.double().view(2, 2, 2, 64), kk) / 8
        ref = torch.einsum("bhgt,bhtd->bhgd", torch.softmax(s, -1), vv).reshape(2, 4, 64)
        assert float((out.double() - ref).norm() / ref.norm()) < 2e-6
    assert int((refs > 0).sum()) == 2 * 3
