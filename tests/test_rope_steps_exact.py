"""The rotation's steps against arithmetic of 60 digits: what they are off by is multiplied by the position."""
from decimal import Decimal as D
from decimal import getcontext

import pytest

import paper_2502_11880_b200 as bn
from paper_2502_11880_b200 import build as bn_build

getcontext().prec = 60
TAU = 2 * D("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def turns(rot, base=10000.0, scaling="none", factor=1.0, low=1.0, high=4.0, context=8192, freqs=None):
    """Of each pair per position, in [0, 1)."""
    base, factor, low, high, context = (D(x) for x in (base, factor, low, high, context))        # (what the call gets: doubles, exactly)
    f = [(-2 * i * base.ln() / rot).exp() for i in range(rot // 2)] if freqs is None else [D(x) for x in freqs]
    if freqs is None and scaling == "linear":
        f = [x / factor for x in f]
    if freqs is None and scaling == "bands":
        s = [min(D(1), max(D(0), (x * context / TAU - low) / (high - low))) for x in f]
        f = [(1 - b) * x / factor + b * x for x, b in zip(f, s)]
    return [x / TAU - (x / TAU).to_integral_value(rounding="ROUND_FLOOR") for x in f]


@pytest.mark.parametrize("args", [dict(rot=128), dict(rot=128, base=1e6), dict(rot=64, base=500000.0), dict(rot=100, base=5e8), dict(rot=2), dict(rot=96, base=0.3),
                                  dict(rot=100, scaling="linear", factor=3.7), dict(rot=128, base=500000.0, scaling="bands", factor=8.0),
                                  dict(rot=128, base=10000.0, scaling="bands", factor=32.0, low=0.7, high=31.3, context=4097),
                                  dict(rot=12, freqs=[1.0, -0.25, 7.5, 0.1, 3.3e-9, -6.0])])
def test_steps_are_right_to_the_last_bits(args):
    bn_build.build()
    got = bn.Rope(**args).desc.step
    # half a unit of rounding; pow, two products, a sum and two quotients, each off by 2^-63 of itself at most, of up to 1.2 turns
    for i, want in enumerate(turns(**args)):
        off = abs(D(got[i]) / D(2) ** 64 - want)
        off = min(off, 1 - off) * D(2) ** 64
        assert off <= 0.5 + 6 * 1.2 * 2, (i, float(off))
