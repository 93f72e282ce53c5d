"""Residual addition, root-mean-square norm and int8 codes: against 64 bits, and code for code against the quantiser on the same y."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from helpers import Guarded

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = {F32: 2.0 ** -24, BF: 2.0 ** -8, HF: 2.0 ** -11}


def rows(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def check(x, residual=None, weight=None, eps=1e-5, y_type=F32, residual_out=None):
    T, K = x.shape
    x0, r0 = x.clone(), None if residual is None else residual.clone()
    y, q, sc, sm = Guarded((T, K), y_type), Guarded((T, K), torch.int8), Guarded((T,), F32), Guarded((T,), torch.int32)
    out = residual_out
    if residual is not None and out is None:
        out = torch.empty(T, K, dtype=residual.dtype, device="cuda")
    bn.bitnet_add_rmsnorm_quant(x, weight, eps, residual=residual, residual_out=out, y=y.t, q=q.t, act_scale=sc.t, act_sum=sm.t)
    torch.cuda.synchronize()
    assert y.intact() and q.intact() and sc.intact() and sm.intact()
    h = x0
    if residual is not None:
        h = (x0.float() + r0.float()).to(residual.dtype)
        assert torch.equal(out, h)
    h = h.double()
    want = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    if weight is not None:
        want = want * weight.double()
    # three binary32 roundings (r, h r, w), then one to y's type
    bound = want.abs() * (3.01 * 2.0 ** -24 + HALF_STEP[y_type] * 1.001) + (2.0 ** -25 if y_type == HF else 1e-37)
    assert bool(((y.t.double() - want).abs() <= bound).all())
    if y_type == F32:                               # the codes are the quantiser's for that y
        q2, sc2, sm2 = bn.bitnet_quant_act(y.t)
        assert torch.equal(q.t, q2) and torch.equal(sc.t, sc2) and torch.equal(sm.t, sm2)
    else:                                           # codes come from y before it was rounded
        full = torch.empty(T, K, device="cuda")
        q2, sc2 = bn.bitnet_add_rmsnorm_quant(x0, weight, eps, residual=r0, y=full)
        assert torch.equal(q.t, q2) and torch.equal(sc.t, sc2) and torch.equal(y.t, full.to(y_type))
    return q.t, sc.t


@pytest.mark.parametrize("T,K", [(1, 1), (2, 3), (1, 4), (5, 7), (3, 64), (2, 100), (1, 1536), (7, 4096), (2, 4098), (300, 3200), (400, 1028), (3, 8192),
                                 (1, 16384), (2, 16388), (1, 28672), (2, 32768), (1, 32772), (1, 40001), (2, 40000), (300, 20000), (40, 16384), (5, 70000), (1, 131072), (1, 131076)])
def test_sizes(T, K):
    check(rows((T, K), F32, K), rows((T, K), F32, K + 1, 3), rows((K,), F32, K + 2))


@pytest.mark.parametrize("x", [F32, BF, HF])
@pytest.mark.parametrize("residual", [None, F32, BF, HF])
@pytest.mark.parametrize("weight,y", [(None, F32), (F32, BF), (BF, HF), (HF, F32)])
def test_types(x, residual, weight, y):
    for T, K in ((5, 520), (320, 260), (2, 33), (3, 16400)):
        check(rows((T, K), x, 1, 2), None if residual is None else rows((T, K), residual, 2), None if weight is None else rows((K,), weight, 3), y_type=y)


def test_strides_and_odd_addresses():
    base = rows((9, 3000), F32, 4)
    for x in (base[:, 8:1032], base[:, 1:1025], base[::2, :777], base[3:4, 5:6]):
        check(x, rows(x.shape, BF, 5), rows((x.shape[1],), F32, 6))
    half = rows((4, 2050), BF, 7)
    check(half[:, 1:2049], half[:, 2:2050].clone(), rows((2049,), BF, 8)[1:])


def test_in_place():
    """residual_out is residual (the default), or x; a second call goes on from there."""
    for K in (4096, 1001):
        x, r = rows((6, K), BF, 9), rows((6, K), F32, 10)
        want = r + x.float()
        q, sc = bn.bitnet_add_rmsnorm_quant(x, residual=r)
        assert torch.equal(r, want)
        y = torch.empty(6, K, device="cuda")
        q2, sc2 = bn.bitnet_add_rmsnorm_quant(want, y=y)
        assert torch.equal(q, q2) and torch.equal(sc, sc2)
        x32, r2 = x.float(), rows((6, K), F32, 10)
        bn.bitnet_add_rmsnorm_quant(x32, residual=r2, residual_out=x32)
        assert torch.equal(x32, want)


def test_rows_of_zeros_infinities_and_no_numbers():
    """The codes stay the quantiser's for the y that binary32 gives; the other rows do not notice."""
    x = rows((6, 512), F32, 11)
    x[1] = 0
    x[2, 7] = float("inf")
    x[3, 100] = float("nan")
    x[4] = 1e-30
    x[5] *= 1e30
    y = torch.empty_like(x)
    for eps in (1e-5, 0.0):
        q, sc = bn.bitnet_add_rmsnorm_quant(x, eps=eps, y=y)
        q2, sc2, _ = bn.bitnet_quant_act(y)
        assert torch.equal(q, q2) and torch.equal(sc, sc2)
        assert torch.isnan(y[3]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[4:]).all()
    check(x[:1], eps=0.0)
    check(x[4:], eps=0.0)
    check(torch.zeros(3, 128, device="cuda"))


def test_rows_do_not_depend_on_the_batch():
    x, r, w = rows((500, 2048), F32, 12), rows((500, 2048), BF, 13), rows((2048,), BF, 14)
    out = torch.empty_like(r)
    q, sc = bn.bitnet_add_rmsnorm_quant(x, w, residual=r, residual_out=out)
    for i in (0, 77, 499):
        one = torch.empty_like(r[:1])
        q1, sc1 = bn.bitnet_add_rmsnorm_quant(x[i:i + 1], w, residual=r[i:i + 1], residual_out=one)
        assert torch.equal(q1[0], q[i]) and torch.equal(sc1[0], sc[i]) and torch.equal(one[0], out[i])


def test_stream_graph_and_no_rows():
    x, w = rows((3, 4096), F32, 15), rows((4096,), F32, 16)
    want = bn.bitnet_add_rmsnorm_quant(x, w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bn.bitnet_add_rmsnorm_quant(x, w, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0])
    q, sc = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bn.bitnet_add_rmsnorm_quant(x, w, q=q, act_scale=sc)
    x.mul_(-2)
    graph.replay()
    torch.cuda.synchronize()
    want = bn.bitnet_add_rmsnorm_quant(x, w)
    assert torch.equal(q, want[0]) and torch.equal(sc, want[1])
    q, sc = bn.bitnet_add_rmsnorm_quant(x[:0], w)
    assert q.shape == (0, 4096) and sc.shape == (0,)


def test_codes_feed_a_linear():
    """mpgemm on these codes is the linear of the normed row."""
    w = bn.synth.ternary(3, 0, 256, 1024, 1 / 3, 1 / 3, device="cuda")
    blob = bn.pack("i2s", w)
    x, g = rows((4, 1024), F32, 17), rows((1024,), F32, 18)
    y = torch.empty_like(x)
    q, sc = bn.bitnet_add_rmsnorm_quant(x, g, y=y)
    a, _ = bn.bitnet_mpgemm("i2s", blob, 0.5, 256, 1024, q, sc)
    b = bn.bitnet_linear("i2s", blob, 0.5, 256, 1024, y)[0]
    assert torch.equal(a, b)


def test_refusals():
    x = rows((2, 64), F32, 19)
    for bad in (dict(x=x.double()), dict(x=x.t()), dict(x=x.cpu()), dict(weight=x[0][:32].clone()), dict(residual=x[:1]), dict(eps=-1.0), dict(eps=float("nan")),
                dict(y=x[:, :32]), dict(q=torch.empty(2, 64, device="cuda")), dict(act_scale=torch.empty(3, device="cuda")),
                dict(residual=x.clone(), residual_out=x.to(BF)), dict(residual_out=x.clone()), dict(act_sum=torch.empty(2, device="cuda"))):
        args = dict(dict(x=x), **bad)
        with pytest.raises(bn.BitnetError):
            bn.bitnet_add_rmsnorm_quant(args.pop("x"), **args)
