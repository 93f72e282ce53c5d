"""Norm: the forms for many rows that come through shared memory, long rows and rows updated in place among them."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from test_gpu_add_rmsnorm import BF, F32, HF, check, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x", [F32, BF, HF])
@pytest.mark.parametrize("T,K", [(400, 8192), (400, 8196), (301, 12000), (400, 14336), (1000, 16380), (400, 16384), (400, 16388)])
def test_many_long_rows_without_a_residual(T, K, x):
    check(rows((T, K), x, K), None, rows((K,), F32, 1))


@pytest.mark.parametrize("x,residual", [(F32, F32), (F32, BF), (BF, BF), (HF, F32), (BF, HF)])
@pytest.mark.parametrize("T,K", [(400, 4), (700, 132), (400, 4096), (400, 8192), (400, 8196), (1000, 6148), (400, 14336)])
def test_many_rows_with_a_residual(T, K, x, residual):
    check(rows((T, K), x, K), rows((T, K), residual, K + 1, 3), rows((K,), BF, 1), y_type=BF)


@pytest.mark.parametrize("T,K", [(400, 1024), (1000, 4096), (900, 8192), (400, 14336), (400, 1001)])
@pytest.mark.parametrize("x,residual", [(F32, F32), (BF, BF), (F32, BF), (BF, F32)])
def test_many_rows_in_place(T, K, x, residual):
    """A row's sum is stored where other rows are on their way from: over the residual, and over x."""
    a, r, w = rows((T, K), x, K), rows((T, K), residual, K + 1, 3), rows((K,), F32, 2)
    apart = torch.empty_like(r)
    q, sc = bn.bitnet_add_rmsnorm_quant(a, w, residual=r, residual_out=apart)
    assert torch.equal(apart, (a.float() + r.float()).to(residual))
    r2 = r.clone()
    q2, sc2 = bn.bitnet_add_rmsnorm_quant(a, w, residual=r2)
    assert torch.equal(r2, apart) and torch.equal(q, q2) and torch.equal(sc, sc2)
    if x == residual:
        a2 = a.clone()
        q2, sc2 = bn.bitnet_add_rmsnorm_quant(a2, w, residual=r, residual_out=a2)
        assert torch.equal(a2, apart) and torch.equal(q, q2) and torch.equal(sc, sc2)
    # rows of a wider buffer, with a guard between them
    wide = torch.full((T, K + 8), 7.0, dtype=residual, device="cuda")
    wide[:, :K] = r
    q2, sc2 = bn.bitnet_add_rmsnorm_quant(a, w, residual=wide[:, :K])
    assert torch.equal(wide[:, :K], apart) and bool((wide[:, K:] == 7.0).all()) and torch.equal(q, q2) and torch.equal(sc, sc2)


def test_the_same_row_again_and_again():
    """x of stride 0."""
    x, r = rows((1, 4096), BF, 3), rows((500, 4096), F32, 4)
    out = torch.empty_like(r)
    q, sc = bn.bitnet_add_rmsnorm_quant(x.expand(500, -1), residual=r, residual_out=out)
    q2, sc2 = bn.bitnet_add_rmsnorm_quant(x.repeat(500, 1), residual=r)
    assert torch.equal(out, r) and torch.equal(q, q2) and torch.equal(sc, sc2)
