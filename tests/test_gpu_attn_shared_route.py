"""Which kernels take a call for shared prefixes: groups of one and empty groups beside a large one, and what the device finds of lengths and prefixes."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from test_gpu_attn_shared import BF, Groups, ints

pytestmark = pytest.mark.gpu


def three_ways(s, q, **kw):
    """As the rule has it, by the kernels of shared prefixes, by the decode kernel."""
    run = lambda: bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, **kw)
    a = run()
    bn.bitnet_debug_attn_shared(True)
    try:
        b = run()
    finally:
        bn.bitnet_debug_attn_shared(False)
    c = bn.bitnet_attn_decode(s.cache, 1, q, s.table, s.len, **kw)
    torch.cuda.synchronize()
    assert not torch.equal(b, c) and torch.allclose(b.float(), c.float(), rtol=2 ** -7, atol=2 ** -7)
    return a, b, c


def test_sequences_alone_do_not_cancel_a_large_group():
    s = Groups([(0, [40])] * 20 + [(4096, [4100 + i for i in range(24)])] + [(0, [30])] * 25, 8, 128, 128, BF, seed=41)
    a, b, _ = three_ways(s, s.queries(16))
    assert torch.equal(a, b)


def test_empty_groups_do_not_cancel_a_large_one():
    """Arrays of a fixed number of groups, padded at the end or in between."""
    s = Groups([(4096, [4100 + i for i in range(32)])], 8, 128, 128, BF, seed=42)
    q = s.queries(16)
    for start in ([0] + [32] * 64, [0] * 30 + [32] * 35, [0] * 64 + [32]):
        s.start = ints(start)
        s.prefix = ints([4096] * (len(start) - 1))
        a, b, _ = three_ways(s, q)
        assert torch.equal(a, b)


def test_groups_of_two():
    """Many over much: shared; few: not."""
    for count, shared in ((40, True), (2, False)):
        s = Groups([(4096, [4100, 4110])] * count, 8, 128, 128, BF, seed=43)
        a, b, c = three_ways(s, s.queries(16))
        assert torch.equal(a, b if shared else c)


def padded(s, groups):
    """Empty groups behind the others: the host cannot tell what is shared."""
    more = groups - s.prefix.numel()
    s.start, s.prefix = torch.cat([s.start, s.start[-1:].repeat(more)]), torch.cat([s.prefix, ints([0] * more)])


def test_nothing_shared_goes_to_the_decode_kernel():
    """Sequences alone, with prefixes of their own or without; rows of a group without tokens do not count; prefixes that left the window neither."""
    s = Groups([(4000, [4100])] * 48, 8, 128, 128, BF, seed=44)
    q = s.queries(16)
    a, _, c = three_ways(s, q)
    assert torch.equal(a, c)
    s.start, s.prefix = ints([0, 48] + [48] * 47), ints([0] * 48)
    a = bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix)
    assert torch.equal(a, c)
    s = Groups([(4000, [4100] * 40)] + [(0, [20])] * 40, 8, 128, 128, BF, seed=45)
    q = s.queries(16)
    s.len[1:40] = 0
    a, b, _ = three_ways(s, q)
    assert torch.equal(a, b)                     # (40 sequences in few groups: not asked)
    padded(s, 80)
    a, _, c = three_ways(s, q)
    assert torch.equal(a, c)
    s = Groups([(1000, [4100] * 40)] + [(0, [20])] * 40, 8, 128, 128, BF, seed=46)
    q = s.queries(16)
    padded(s, 80)
    a, _, c = three_ways(s, q, window=3000)
    assert torch.equal(a, c)
    # 40 x 65 + 40 tiles seen, 39 x 16 of them again: three times those are fewer
    a, _, c = three_ways(s, q)
    assert torch.equal(a, c)
    s.prefix[0] = 4096                           # (the sequences have these in common too, or not: it is only weighed)
    a = bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix)
    assert not torch.equal(a, c)


def test_a_captured_call_goes_by_the_lengths_at_its_replay():
    s = Groups([(4096, [4100 + i for i in range(24)])] + [(0, [30])] * 30, 8, 128, 128, BF, seed=47)
    q = s.queries(16)
    ws, out, status = bn.new_attn_shared_workspace(54, 16, 8, 128), torch.empty_like(q), ints([0])
    long = s.len.clone()
    s.len.fill_(25)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(2):
            bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, out=out, workspace=ws, dev_status=status)
    for lens, shared in ((s.len.clone(), False), (long, True), (s.len.clone(), False), (long, True)):
        s.len.copy_(lens)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        _, b, c = three_ways(s, q)
        assert torch.equal(out, b if shared else c)
    assert int(status) == 0 and bn.bitnet_device_status() == 0 and int(ws[:bn.ATTN_WORKSPACE_HEAD].sum()) == 0


def test_asked_calls_back_to_back_on_two_streams():
    """Workspaces of their own; calls that the device sends either way follow one another."""
    pair = []
    for seed, lens in ((48, None), (49, 30)):
        s = Groups([(4096, [4100 + i for i in range(24)])] + [(0, [30])] * 30, 8, 128, 128, BF, seed=seed)
        if lens:
            s.len.fill_(lens)
        pair.append((s, s.queries(16), bn.new_attn_shared_workspace(54, 16, 8, 128), torch.cuda.Stream()))
    want = [bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix) for s, q, _, _ in pair]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(15):
        for k, (s, q, ws, stream) in enumerate(pair):
            with torch.cuda.stream(stream):
                got[k].append(bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, workspace=ws))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[k]) for k in range(2) for g in got[k])
