"""Page ids beyond 2^30, where twice the id passes 31 bits: a pool whose pages overlap, so that so many of them fit the device."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from test_gpu_kv_pages import i32

pytestmark = pytest.mark.gpu


def test_pages_beyond_2_to_30():
    pages = 2 ** 30 + 16                                    # a page every 8 elements, of 8 rows of 8
    flat = [torch.empty(pages * 8 + 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shape, stride = (1, pages, 1, 8, 8), (pages * 8, 8, 64, 8, 1)
    k, v = (t.as_strided(shape, stride) for t in flat)
    g = torch.Generator(device="cuda").manual_seed(1)
    for t in flat:
        t[:1024].normal_(generator=g)
        t[-1024:].normal_(generator=g)
    cache, last = bn.KvCache(k, v), pages - 1
    source = [t[last * 8:last * 8 + 64].clone() for t in flat]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bn.bitnet_kv_copy_pages(cache, i32([last]), i32([3]), dev_status=status)             # from there
    assert all(torch.equal(t[24:88], s) for t, s in zip(flat, source)) and int(status) == 0
    source = [t[512:576].clone() for t in flat]
    bn.bitnet_kv_copy_pages(cache, i32([64]), i32([last - 2]), dev_status=status)        # and to there
    at = (last - 2) * 8
    assert all(torch.equal(t[at:at + 64], s) for t, s in zip(flat, source)) and int(status) == 0
    x = torch.randn(1, 1, 8, generator=g, device="cuda")
    bn.bitnet_kv_append(cache, 0, x, -x, i32([[last]]), i32([8]), dev_status=status)     # row 7 of the last page
    at = last * 8 + 56
    assert torch.equal(flat[0][at:at + 8], x.view(8).bfloat16()) and torch.equal(flat[1][at:at + 8], -x.view(8).bfloat16())
    assert int(status) == 0


def test_reserve_of_more_than_2_to_31_entries():
    """Rows that together ask for more pages than 31 bits count: the first few get what the pool has, the rest none, and it is reported."""
    seqs, width, pages = 2049, 1 << 20, 10
    table = torch.full((seqs, width), 7, dtype=torch.int32, device="cuda")
    refs, zero = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.zeros(seqs, dtype=torch.int32, device="cuda")
    refs[4] = 1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bn.bitnet_kv_reserve(refs, table, zero, torch.full_like(zero, 8 * width), 8, dev_status=status)
    assert int(status) == 8 and bool((refs == 1).all())
    assert table[0, :9].tolist() == [0, 1, 2, 3, 5, 6, 7, 8, 9] and bool((table[0, 9:] == -1).all())
    for s in range(1, seqs, 64):
        assert bool((table[s:s + 64] == -1).all())
