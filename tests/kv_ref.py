"""Plain 64-bit forms of the paged cache's attention, and the bounds that its kernels' outputs are held to."""
import torch


def attn_ref(k, v, q, table, pos, seq, scale, window=0, sinks=0):
    """k, v: pools of one layer [pages][heads][page][dim]; q [tokens][q_heads][dim]; token n belongs to sequence seq[n] and is at
    position pos[n].  Returns (out, weight, score_err): out in float64, weight = sum p |v| / sum p, and per row (token, head) a bound on the relative
    error of its probabilities from fp32 arithmetic."""
    k, v, q, table = k.double().cpu(), v.double().cpu(), q.double().cpu(), table.cpu()
    pages, hkv, page, dim = k.shape
    hq = q.shape[1]
    out, weight = torch.zeros_like(q), torch.zeros_like(q)
    rel = torch.zeros(q.shape[0], hq, 1, dtype=torch.float64)
    for n in range(q.shape[0]):
        p = int(pos[n])
        if p < 0:
            continue
        c = torch.arange(p + 1)
        if window:
            c = c[(c > p - window) | (c < sinks)]
        ids = table[int(seq[n])].long()[c // page]
        for h in range(hq):
            g = h // (hq // hkv)
            kk, vv = k[ids, g, c % page], v[ids, g, c % page]
            s = kk @ q[n, h] * scale
            e = torch.exp(s - s.max())
            out[n, h] = (e[:, None] * vv).sum(0) / e.sum()
            weight[n, h] = (e[:, None] * vv.abs()).sum(0) / e.sum()
            # fp32 products summed over dim, then scaled, subtracted and raised to a power of two; sums of len(c) terms by 8 chains
            dots = ((kk.abs() @ q[n, h].abs()) * abs(scale)).max()
            rel[n, h] = (dim + 4) * 2.0 ** -24 * dots + 2.0 ** -21 * (1 + s.abs().max()) + (len(c) / 8 + 16) * 2.0 ** -24
    return out, weight, rel


# unit roundoff of one conversion: 24, 8 and 11 significant bits
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def check_attn(out, ref, p_unit):
    """|out - ref| <= one rounding to out's type + 2 * weight * (relative error of the probabilities: fp32 arithmetic and their
    own rounding `p_unit`); the smallest normal of fp16 covers its subnormals."""
    want, weight, rel = ref
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    bound = UNIT[out.dtype] * want.abs() * 1.01 + 2 * weight * (rel + p_unit) + (2.0 ** -24 if out.dtype == torch.float16 else 1e-30)
    worst = ((got - want).abs() / bound.clamp(min=1e-300)).max()
    assert worst <= 1, float(worst)
