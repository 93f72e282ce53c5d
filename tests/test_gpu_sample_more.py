"""Drawing of tokens: what is never drawn under any setting, and how far probabilities may be off."""
import pytest
import torch

import paper_2502_11880_b200 as bn

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("vocab", [400, 40000])
def test_what_is_never_drawn(vocab, dtype):
    inf, nan = float("inf"), float("nan")
    g = torch.Generator(device="cuda").manual_seed(7)
    base = (torch.randn(7, vocab, generator=g, device="cuda") * 2.5).to(dtype)
    base[0, 100:] = -inf
    base[1, ::3] = nan
    base[2] = -inf
    base[3] = nan
    base[4, 50] = base[4, 60] = inf
    base[5, :] = -inf
    base[5, vocab - 1] = -3.0
    base[6] = torch.finfo(dtype).max * 0.9 * torch.sign(base[6].float()).to(dtype)
    full = lambda v, d=F32: torch.full((7,), v, dtype=d, device="cuda")
    for seed in range(6):
        u = torch.rand(7, generator=g, device="cuda")
        for kw in (dict(), dict(top_k=full(150, torch.int32)), dict(top_k=full(1000, torch.int32)), dict(top_p=full(0.9)), dict(min_p=full(0.1)), dict(temperature=full(1e-30)),
                   dict(temperature=full(0.0)), dict(temperature=full(3.0), top_k=full(60, torch.int32), top_p=full(0.8)), dict(temperature=full(1e30)), dict(temperature=full(1e30), top_p=full(0.7))):
            tokens, prob = bn.bitnet_sample(base, u, **kw)
            t, p = tokens.tolist(), prob.tolist()
            assert t[2] == t[3] == -1 and p[2] == p[3] == 0
            assert 0 <= t[0] < 100
            assert 0 <= t[1] < vocab and t[1] % 3 != 0
            assert t[4] in (50, 60) and p[4] in ((0.5, 1.0) if kw else (0.5,))
            assert t[5] == vocab - 1 and p[5] == 1
            # (fp16's range is small enough for all to be alike at the largest temperature)
            assert base[6, t[6]] > 0 or (dtype == HF and "temperature" in kw and float(kw["temperature"][0]) > 1e20)


def test_a_distance_beyond_the_range_counts_as_infinite():
    x = torch.tensor([[-3e38, 3e38, -3e38, 2e38]], device="cuda")
    for u in (0.0, 0.3, 0.999):
        token, _ = bn.bitnet_sample(x, torch.tensor([u], device="cuda"), temperature=torch.tensor([1e38], device="cuda"))
        assert int(token) in (1, 3)


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("temperature", [0.6, 1.0, 3.0, 40.0])
@pytest.mark.parametrize("top", [20.0, 3.0, 0.011])
def test_probabilities(top, temperature, dtype):
    """One large value and many small ones: max - x loses what the small ones differ in."""
    g = torch.Generator(device="cuda").manual_seed(3)
    vocab = 4000
    x = (torch.randn(1, vocab, generator=g, device="cuda") * 1e-3).to(dtype)
    x[0, ::7] = (torch.randn(1, vocab, generator=g, device="cuda")[0, ::7] * 1e-6).to(dtype)
    x[0, 17] = top
    u = torch.cat([torch.linspace(0, 0.9999, 200), 1 - torch.logspace(-1, -7, 200)]).cuda()
    n = u.numel()
    tokens, prob = bn.bitnet_sample(x.expand(n, -1), u, temperature=torch.full((n,), temperature, device="cuda"))
    z = x[0].double()
    t = float(torch.tensor(temperature))
    far = (z.max() - z) / torch.tensor(t, dtype=torch.float32).double().item()
    p = torch.softmax(-far, 0)
    far = far[tokens.long()]
    want = p[tokens.long()]
    # The weight's own 2^-22, the argument's rounding and prob's; of 16-bit logits the distance's too; and the same again for the sum (of terms no
    # farther), with half a unit of 2^-32 of the largest per term.
    of_weight = 2.0 ** -22 + 2.0 ** -25 + (0.0 if dtype == F32 else 2.0 ** -24 * far)
    bound = 2 * of_weight + 2.0 ** -24 + vocab * 2.0 ** -33 * p.max() + (0.0 if dtype == F32 else 2.0 ** -24 * float((z.max() - z).max()) / t)
    worst = ((prob.double() / want - 1).abs() / bound).max()
    assert worst <= 1, float(worst)
    # and the token is the one where the sum exceeds u, or lies a rounding beside it
    c = torch.cumsum(p, 0)
    at = u.double()
    slack = 2.0 ** -20
    assert bool((c[tokens.long()] + slack > at).all()) and bool((c[tokens.long()] - want - slack <= at).all())
