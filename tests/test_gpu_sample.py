"""Drawing of tokens by temperature, top-k, top-p and min-p against a plain implementation in 64 bits."""
import math

import pytest
import torch

import paper_2502_11880_b200 as bn
from helpers import Guarded

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
# Weights are off by the exponential's 2^-22 and half a step of 2^-32 of the largest; a row's sums by no more.  A border may move by that.
EPS = 2.0 ** -21


def kept_weights(x, t, k, p, m):
    """Weights of what is kept, 0 elsewhere, of one row in 64 bits."""
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    w = [math.exp((v - x[order[0]]) / t) if v > -math.inf else 0.0 for v in x] if t > 0 else [0.0] * len(x)
    if not t > 0:
        w[order[0]] = 1.0
        return w
    if 0 < k < len(x):
        order = order[:k]
    if p < 1:
        total, run, n = sum(w[i] for i in order), 0.0, 0
        for i in order:
            if n and run >= p * total:
                break
            run += w[i]
            n += 1
        order = order[:n]
    keep = set(i for i in order if w[i] >= min(m, 1.0))
    return [v if i in keep else 0.0 for i, v in enumerate(w)]


def draws(x, u, t=1.0, k=0, p=1.0, m=0.0):
    """The tokens that the definition allows, with their probabilities: its own, and those next to borders by EPS."""
    allowed = {}
    for dp in (0, -EPS, EPS) if p < 1 else (0,):
        for dm in (0, -EPS, EPS) if m > 0 else (0,):
            w = kept_weights(x, t, k, p + dp * p, m + dm * m)
            total, run = sum(w), 0.0
            for i, v in enumerate(w):
                if v > 0 and run - EPS * total <= u * total < run + v + EPS * total:
                    allowed.setdefault(i, v / total)
                run += v
    return allowed


def check(logits, u, t=None, k=None, p=None, m=None, prob_bound=2.0 ** -18):
    rows = logits.shape[0]
    as_row = lambda v, d: None if v is None else torch.tensor(v, dtype=d, device="cuda")
    tokens, prob = Guarded((rows,), torch.int32), Guarded((rows,), F32)
    bn.bitnet_sample(logits, torch.tensor(u, device="cuda"), as_row(t, F32), as_row(k, torch.int32), as_row(p, F32), as_row(m, F32), tokens=tokens.t, prob=prob.t)
    torch.cuda.synchronize()
    assert tokens.intact() and prob.intact()
    for r in range(rows):
        x = logits[r].double().cpu().tolist()
        f = lambda v, d: d if v is None else torch.tensor(v[r], dtype=F32).double().item()
        want = draws([-math.inf if v != v else v for v in x], torch.tensor(u[r], dtype=F32).double().item(), f(t, 1.0), 0 if k is None else k[r], f(p, 1.0), f(m, 0.0))
        token = int(tokens.t[r])
        assert token in want, (r, token, want)
        assert abs(float(prob.t[r]) / want[token] - 1) <= prob_bound, (r, float(prob.t[r]), want)
    return tokens.t, prob.t


def logits(rows, vocab, dtype=F32, seed=0, spread=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g, device="cuda") * spread).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 64, 127, 1000, 4099, 32000])
def test_settings(vocab, dtype):
    x = logits(8, vocab, dtype, vocab)
    u = [0.0, 0.1, 0.3, 0.5, 0.7, 0.9, 0.99, 0.9999999]
    check(x, u)
    check(x, u, t=[0.7] * 8)
    check(x, u, k=[1, 2, 5, 40, 300, 0, -3, 10 ** 9])
    check(x, u, p=[0.0, 0.1, 0.5, 0.9, 0.99, 1.0, 0.95, 2.0])
    check(x, u, m=[0.0, 0.01, 0.1, 0.5, 1.0, 3.0, -1.0, 0.2])
    check(x, u, t=[0.0, 0.2, 1.0, 1.3, 5.0, 0.8, -1.0, 100.0], k=[50, 7, 0, 64, 200, 5, 3, 1000], p=[0.9, 0.8, 0.95, 1.0, 0.3, 0.99, 0.5, 0.9],
          m=[0.0, 0.1, 0.0, 0.05, 0.0, 0.3, 0.0, 0.9])


@pytest.mark.parametrize("rows,vocab,dtype", [(3, 128256, F32), (40, 128256, F32), (200, 5003, BF), (2, 300001, HF), (1, 700001, F32)])
def test_large(rows, vocab, dtype):
    """Slices in shared memory, one to eight CTAs per row, and rows that do not fit them (read again at every pass)."""
    x = logits(rows, vocab, dtype, rows)
    pick = [0, rows // 2, rows - 1]
    g = torch.Generator().manual_seed(rows)
    u, t = torch.rand(rows, generator=g), 0.5 + torch.rand(rows, generator=g)
    k, p, m = torch.randint(0, 2000, (rows,), generator=g).int(), 0.5 + 0.6 * torch.rand(rows, generator=g), 0.1 * torch.rand(rows, generator=g)
    all_tokens, all_prob = bn.bitnet_sample(x, u.cuda(), t.cuda(), k.cuda(), p.cuda(), m.cuda())
    one, _ = check(x[pick], u[pick].tolist(), t[pick].tolist(), k[pick].tolist(), p[pick].tolist(), m[pick].tolist())
    # a row's token does not depend on how many rows there are, nor on how the work is split
    assert torch.equal(all_tokens[pick], one)


def test_equal_logits():
    """Everything is a tie: the first of them count, by index."""
    for vocab, k in ((5000, 700), (128256, 100000), (128256, 3), (300, 255)):
        x = torch.zeros(3, vocab, device="cuda")
        tokens, prob = bn.bitnet_sample(x, torch.tensor([0.0, 0.5, 0.9999999], device="cuda"), top_k=torch.full((3,), k, dtype=torch.int32, device="cuda"))
        assert tokens.tolist() == [0, k // 2, k - 1] and torch.allclose(prob, torch.full_like(prob, 1 / k), rtol=1e-5)
        tokens, _ = bn.bitnet_sample(x, torch.tensor([0.0, 0.5, 0.9999999], device="cuda"), top_p=torch.full((3,), 0.25, device="cuda"))
        n = -(-vocab // 4)
        assert tokens.tolist() == [0, n // 2, n - 1]
        tokens, prob = bn.bitnet_sample(x, torch.full((3,), 0.7, device="cuda"), temperature=torch.zeros(3, device="cuda"))
        assert tokens.tolist() == [0] * 3 and prob.tolist() == [1.0] * 3


def test_many_ties_at_the_border():
    """Values of few bits: thousands of equal logits lie at every cut."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-6, 7, (6, 20000), generator=g, device="cuda").float()
    u = [0.05, 0.3, 0.5, 0.77, 0.9, 0.999]
    check(x, u, k=[1, 500, 1541, 3000, 9999, 19999])
    check(x, u, p=[0.1, 0.5, 0.6, 0.9, 0.99, 0.999])
    check(x, u, k=[2000] * 6, p=[0.1, 0.5, 0.6, 0.9, 0.99, 0.999], t=[0.3, 0.5, 1.0, 2.0, 4.0, 8.0])
    x[:, ::2] = -0.0                              # -0 equals 0
    x[:, 1::2] = 0.0
    tokens, _ = bn.bitnet_sample(x, torch.tensor(u, device="cuda"), top_k=torch.full((6,), 10, dtype=torch.int32, device="cuda"))
    assert tokens.tolist() == (torch.tensor(u).double() * 10).int().tolist()       # (binary32 has 0.9 just below 9 tenths)


@pytest.mark.parametrize("vocab,dtype", [(600, F32), (9000, BF), (30011, F32), (400001, F32)])
def test_short_and_long_lists(vocab, dtype):
    """Some 256 items that may be kept: on both sides of it, by either rule, by both, with ties across the cut, and with fewer items in reach."""
    ks = [1, 31, 32, 33, 127, 128, 129, 223, 224, 225, 255, 256, 257, 300]
    if vocab > 100000:
        ks = [128, 256, 257]
    u = [(i * 0.37 + 0.011) % 1 for i in range(len(ks))]
    x = logits(len(ks), vocab, dtype, 11, 3.0)
    check(x, u, k=ks)
    check(x, u, k=ks, p=[0.95, 0.5, 1.0, 0.999, 0.9, 0.3, 0.99, 0.9, 0.01, 0.97, 0.8, 0.9999, 0.6, 0.9][:len(ks)], m=([0.0, 0.05] * 7)[:len(ks)],
          t=([0.6, 1.0] * 7)[:len(ks)])
    check(x, u, p=[0.02 * (i + 1) for i in range(len(ks))], t=[0.8] * len(ks))
    check(x, u, k=[2000] * len(ks), p=[0.05 * (i + 1) for i in range(len(ks))])
    coarse = (x * 2).round() / 2                  # equal ones lie at the cut, more than there is room for in some rows
    check(coarse, u, k=ks)
    check(coarse, u, k=ks, p=[0.9] * len(ks))
    few = torch.full_like(x, -300.0)              # out of reach, but for a few
    few[:, ::vocab // 30] = x[:, ::vocab // 30].clamp(-3, 3)
    check(few, u, k=ks)
    check(few, u, k=ks, p=[0.7] * len(ks))


def test_close_values():
    """Neighbouring floats: the order goes by the last bit."""
    base = torch.arange(3000, dtype=torch.int32, device="cuda") + torch.tensor(5.0).view(torch.int32).item()
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.stack([base[torch.randperm(3000, generator=g, device="cuda")].view(F32) for _ in range(3)])
    for k in (1, 2, 700, 2999):
        tokens, _ = bn.bitnet_sample(x, torch.tensor([0.0, 0.5, 0.9999999], device="cuda"), top_k=torch.full((3,), k, dtype=torch.int32, device="cuda"))
        for r, at in enumerate((0, k // 2, k - 1)):
            kept = torch.topk(x[r], k).indices.sort().values
            assert abs((kept == int(tokens[r])).nonzero().item() - at) <= 1 and (k > 2 or int(tokens[r]) in kept.tolist())


def test_infinities_no_numbers_and_empty_rows():
    inf, nan = float("inf"), float("nan")
    x = logits(7, 400, seed=7)
    x[0, 100:] = -inf
    x[1, ::3] = nan
    x[2] = -inf
    x[3] = nan
    x[4, 50] = x[4, 60] = inf
    x[5, :] = -inf
    x[5, 399] = -3.0
    x[6] = 3e38 * torch.sign(x[6])
    u = torch.tensor([0.99, 0.5, 0.5, 0.5, 0.6, 0.3, 0.5], device="cuda")
    for kw in (dict(), dict(top_k=torch.full((7,), 150, dtype=torch.int32, device="cuda")), dict(top_p=torch.full((7,), 0.9, device="cuda")),
               dict(temperature=torch.full((7,), 1e-30, device="cuda")), dict(temperature=torch.full((7,), 1e30, device="cuda")), dict(temperature=torch.zeros(7, device="cuda"))):
        tokens, prob = bn.bitnet_sample(x, u, **kw)
        t = tokens.tolist()
        assert t[2] == t[3] == -1 and prob[2] == prob[3] == 0 and t[5] == 399 and prob[5] == 1
        assert 0 <= t[0] < 100 and t[1] % 3 != 0 and t[4] in (50, 60) and x[6, t[6]] > 0 or "temperature" in kw
        assert t[4] == (50 if "temperature" in kw and kw["temperature"][0] == 0 else t[4])
    check(x[:2], [0.99, 0.5], p=[0.9, 0.8])


def test_odd_settings():
    x, nan = logits(6, 500, seed=8), float("nan")
    dev = lambda v, d=F32: torch.tensor(v, dtype=d, device="cuda")
    plain, _ = bn.bitnet_sample(x, dev([0.0, 0.4, 0.99999994, 0.5, 0.5, 0.5]))
    odd, _ = bn.bitnet_sample(x, dev([-3.0, 0.4, 7.0, 0.5, 0.5, 0.5]), top_p=dev([nan] * 6), min_p=dev([nan] * 6))
    assert torch.equal(plain, odd)
    assert int(bn.bitnet_sample(x[:1], dev([nan]))[0]) == int(plain[0])
    tokens, prob = bn.bitnet_sample(x, dev([0.5] * 6), temperature=dev([nan, 0.0, -2.0, float("inf"), 1e-38, 1.0]))
    assert tokens[:3].tolist() == x[:3].argmax(-1).tolist() and int(tokens[3]) == 250 and abs(float(prob[3]) - 1 / 500) < 1e-8
    assert int(tokens[4]) == int(x[4].argmax())


def test_shares_follow_the_weights():
    """u over a fine grid: tokens come as often as their weights say."""
    x = logits(1, 50, seed=9, spread=1.0)
    n = 20000
    u = (torch.arange(n, device="cuda") + 0.5) / n
    tokens, prob = bn.bitnet_sample(x.expand(n, 50), u, top_k=torch.full((n,), 20, dtype=torch.int32, device="cuda"))
    w = torch.tensor(kept_weights(x[0].double().tolist(), 1.0, 20, 1.0, 0.0), dtype=torch.float64)
    share = torch.bincount(tokens.long().cpu(), minlength=50).double() / n
    assert float((share - w / w.sum()).abs().max()) <= 1.01 / n + EPS
    assert torch.allclose(prob.double().cpu(), (w / w.sum())[tokens.cpu().long()], rtol=2 ** -20)


def test_strides_stream_graph_and_no_rows():
    wide = logits(6, 2001, BF, 10)
    u = torch.linspace(0, 0.99, 6, device="cuda")
    p = torch.full((6,), 0.9, device="cuda")
    want, _ = bn.bitnet_sample(wide[:, 1:1998].contiguous(), u, top_p=p)
    assert torch.equal(bn.bitnet_sample(wide[:, 1:1998], u, top_p=p)[0], want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got, _ = bn.bitnet_sample(wide[:, 1:1998], u, top_p=p, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    tokens, prob = torch.empty_like(want), torch.empty(6, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bn.bitnet_sample(wide[:, 1:1998], u, top_p=p, tokens=tokens, prob=prob)
    u.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(tokens, bn.bitnet_sample(wide[:, 1:1998], u, top_p=p)[0])
    assert bn.bitnet_sample(wide[:0], u[:0])[0].shape == (0,)


def test_refusals():
    x, u = logits(2, 64), torch.zeros(2, device="cuda")
    for bad in (dict(logits=x.double()), dict(logits=x.t()), dict(logits=x[:, :0]), dict(u=u[:1]), dict(u=None), dict(u=u.double()), dict(top_k=u), dict(top_p=u[:1]),
                dict(temperature=u.cpu()), dict(tokens=torch.empty(2, dtype=torch.int64, device="cuda")), dict(prob=torch.empty(3, device="cuda"))):
        with pytest.raises(bn.BitnetError):
            bn.bitnet_sample(**dict(dict(logits=x, u=u), **bad))
