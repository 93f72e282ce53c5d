"""Rotation where the other tests do not go: pairs side by side at odd strides and addresses, exact angles far out."""
import math
from decimal import Decimal as D

import pytest
import torch

import paper_2502_11880_b200 as bn
from test_gpu_kv_rope import BF, F32, HF, Case, close
from test_rope_steps_exact import turns

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stride,address", [(61, 0), (62, 0), (64, 1), (64, 2), (64, 4), (63, 3)])
@pytest.mark.parametrize("io,out", [(F32, F32), (F32, BF), (BF, BF), (BF, F32)])
def test_pairs_side_by_side_at_odd_strides_and_addresses(stride, address, io, out):
    """Vectors of one, two and four elements; the rotated part ends inside a vector, and the head."""
    for rot in (60, 38, 42, 2):
        for layout in ("interleaved", "half"):
            c = Case([(3, 70), (0, 5), (900, 1)], 8, 2, 60, 16, BF, io, seed=rot)
            n = c.q.shape[0]
            for name, heads in (("q", 8), ("k_new", 2), ("v_new", 2)):
                wide = torch.full((address + n * heads * stride,), 9.0, dtype=io, device="cuda")
                view = wide[address:].view(n, heads, stride)[..., :60]
                view.copy_(getattr(c, name))
                setattr(c, name, view)
            c.check(c.run(bn.Rope(rot, layout=layout), out), rot=rot, layout=layout)


@pytest.mark.parametrize("dim,rot", [(4, 2), (12, 10), (36, 34), (100, 98), (128, 126)])
def test_parts_of_odd_heads(dim, rot):
    for io in (F32, HF):
        for layout in ("interleaved", "half"):
            c = Case([(3, 40), (500, 1)], 5, 5, dim, 16, HF, io, seed=dim)
            c.check(c.run(bn.Rope(rot, layout=layout), F32), rot=rot, layout=layout)


@pytest.mark.parametrize("rope", [dict(rot=32, base=500000.0), dict(rot=128, base=1e6), dict(rot=64, base=10000.0, scaling="linear", factor=3.0)])
def test_angles_at_far_positions(rope):
    """Against turns of 60 digits: binary32's share of the error alone, at every position."""
    page, rot = 1 << 20, rope["rot"]
    lens = [2 ** 31 - 3 * page, 2 ** 31 - 3 * page - 12345, 2 ** 30 + 7, 2 ** 24 + 3, 131073]
    c = Case([(0, 1)] * len(lens), 2, 1, rot, 16, BF, F32, seed=rot)
    k = torch.zeros(1, len(lens), 1, page, rot, dtype=BF, device="cuda")
    cache = bn.KvCache(k, torch.zeros_like(k))
    table = torch.full((len(lens), 2048), -1, dtype=torch.int32, device="cuda")
    for i, n in enumerate(lens):
        table[i, (n - 1) // page] = i
    got = bn.bitnet_kv_append_rope(cache, 0, bn.Rope(**rope), c.q, c.k_new, c.v_new, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    part = [[float(2 * D(math.pi) * ((n - 1) * t % 1)) for t in turns(**rope)] for n in lens]          # (2 pi in 53 bits: 2^-50 off)
    angle = torch.tensor(part, dtype=torch.float64)[:, None]
    x = c.q.double().cpu()
    a, b = x[..., :rot // 2], x[..., rot // 2:]
    want = torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)
    # half turns to 2^-25 and what the step brings, 2^-23 radians together; the functions' 2 steps; two products and a sum
    err = (a.abs() + b.abs()) * (2.0 ** -22 + 3 * 2.0 ** -24)
    close(got, want, torch.cat([err, err], -1))
