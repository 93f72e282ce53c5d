"""Entries of the table below zero, whichever: where a token is read they are reported, and read as zeros."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from test_gpu_kv_attn import BF, HF, Paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 100, 128])
@pytest.mark.parametrize("new", [1, 20])
def test_negative_entries_are_all_alike(dim, new):
    p = Paged([300], 2, dim, 16, HF if dim == 100 else BF, seed=31)
    q = p.queries(new, 4, dim, p.cache.dtype)
    start = torch.tensor([0, new], dtype=torch.int32, device="cuda")

    def run(entry):
        table, status = p.table.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        if entry is not None:
            table[0, 3] = entry
        if new == 1:
            out = bn.bitnet_attn_decode(p.cache, p.layer, q, table, p.len, dev_status=status)
        else:
            out = bn.bitnet_attn_prompt(p.cache, p.layer, q, table, p.len, start, new, dev_status=status)
        torch.cuda.synchronize()
        return out, int(status)

    assert run(None)[1] == 0
    want, status = run(-1)
    assert status == 7 and torch.isfinite(want).all()
    for entry in (-2, -3, -2 ** 31):
        out, status = run(entry)
        assert status == 7 and torch.equal(out, want), entry


def test_negative_entries_of_shared_prefixes_and_own_tokens():
    ints = dict(dtype=torch.int32, device="cuda")
    p = Paged([300], 2, 64, 16, BF, seed=32)
    table, length = p.table.expand(2, -1).contiguous(), torch.tensor([300, 290], **ints)
    q = p.queries(2, 4, 64, BF)

    def run(row, entry, value):
        t, status = table.clone(), torch.zeros(1, **ints)
        t[row, entry] = value
        out = bn.bitnet_attn_shared(p.cache, p.layer, q, t, length, torch.tensor([0, 2], **ints), torch.tensor([160], **ints), dev_status=status)
        torch.cuda.synchronize()
        return out, int(status)

    for row, entry in ((0, 3), (1, 15)):
        want, status = run(row, entry, -1)
        assert status == 7
        for value in (-2, -3, -2 ** 31):
            out, status = run(row, entry, value)
            assert status == 7 and torch.equal(out, want)
