"""Entry points of a decode step around the linears without a GPU: refusals come before anything is launched; the rotation's description."""
import ctypes as C
import math

import pytest

import paper_2502_11880_b200 as bn
from paper_2502_11880_b200 import build as bn_build

NULL, FAKE, ODD = C.c_void_p(None), C.c_void_p(4096), C.c_void_p(4097)     # never dereferenced: validation fails first
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def L():
    bn_build.build()
    return bn.lib()


def norm(L, x=FAKE, xt=2, sx=64, r=FAKE, rt=2, sr=64, ro=FAKE, so=64, w=FAKE, wt=2, eps=1e-5, T=1, K=64, y=FAKE, yt=2, q=FAKE, sc=FAKE, sm=FAKE):
    return L.bitnet_add_rmsnorm_quant(x, xt, sx, r, rt, sr, ro, so, w, wt, eps, T, K, y, yt, q, sc, sm, NULL)


@pytest.mark.parametrize("bad", [dict(x=NULL), dict(x=ODD), dict(xt=3), dict(xt=-1), dict(rt=7), dict(wt=4), dict(yt=3), dict(ro=NULL), dict(r=NULL), dict(r=ODD), dict(ro=ODD), dict(T=2, so=0), dict(T=2, so=63), dict(T=2, so=-63), dict(xt=0),
                                 dict(w=ODD), dict(eps=-1.0), dict(eps=INF), dict(eps=NAN), dict(T=-1), dict(K=0), dict(T=1 << 31), dict(K=1 << 31), dict(q=NULL),
                                 dict(q=C.c_void_p(4104)), dict(y=C.c_void_p(4104)), dict(sc=NULL), dict(sc=C.c_void_p(4098)), dict(sm=C.c_void_p(4098))])
def test_norm_is_checked(L, bad):
    assert norm(L, **bad) == 1


@pytest.mark.parametrize("where", [dict(r=C.c_void_p(8192), sx=128), dict(x=C.c_void_p(8192), sr=128)])       # in place over x, over the residual
def test_norm_in_place_keeps_its_stride(L, where):
    assert norm(L, T=2, **where) == 1


def test_calls_with_nothing_to_do(L):
    assert norm(L, T=0, x=NULL, q=NULL, sc=NULL) == 0
    assert L.bitnet_sample(NULL, 2, 64, 0, 64, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL) == 0


def sample(L, x=FAKE, t=2, rows=1, vocab=64, u=FAKE, temp=FAKE, k=FAKE, p=FAKE, m=FAKE, tok=FAKE, prob=FAKE):
    return L.bitnet_sample(x, t, 64, rows, vocab, u, temp, k, p, m, tok, prob, NULL)


@pytest.mark.parametrize("bad", [dict(x=NULL), dict(x=ODD), dict(t=3), dict(rows=-1), dict(rows=1 << 29), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(u=NULL), dict(tok=NULL),
                                 dict(u=ODD), dict(temp=ODD), dict(k=ODD), dict(p=ODD), dict(m=ODD), dict(tok=ODD), dict(prob=ODD)])
def test_sample_is_checked(L, bad):
    assert sample(L, **bad) == 1


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=130), dict(rot_dim=-2), dict(scaling=3), dict(base=0.0), dict(base=-1.0), dict(base=INF), dict(base=NAN),
                                 dict(magnitude=NAN), dict(scaling=1, factor=0.0), dict(scaling=1, factor=NAN), dict(scaling=2, high=1.0), dict(scaling=2, context=0.0),
                                 dict(scaling=2, low=-INF), dict(freqs=(C.c_double * 32)(*[NAN] * 32))])
def test_ropes_are_checked(L, bad):
    d = bn.RopeDesc(rot_dim=64, base=10000.0, factor=2.0, low=1.0, high=4.0, context=8192.0, magnitude=1.0)
    assert L.bitnet_rope_init(C.byref(d)) == 0 and d.ready
    for k, v in bad.items():
        setattr(d, k, v)
    assert L.bitnet_rope_init(C.byref(d)) in (1, 2) and not d.ready
    assert L.bitnet_rope_init(None) == 1


def test_rope_steps_are_turns():
    def radians(r):
        return [s / 2.0 ** 64 * 2 * math.pi for s in r.desc.step]

    def same(got, want):               # one step of 2^-64 turns, and a few roundings of 64 bits
        return abs(got - want) <= 4e-19 + 2e-15 * want

    got = radians(bn.Rope(64, base=500000.0))
    assert all(same(got[i], 500000.0 ** (-i / 32)) for i in range(32)) and got[32:] == [0.0] * 32
    got = radians(bn.Rope(8, scaling="linear", factor=4.0))
    assert all(same(got[i], 10000.0 ** (-i / 4) / 4) for i in range(4))
    got = radians(bn.Rope(128, base=500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, context=8192))
    for i in range(64):
        f = 500000.0 ** (-i / 64)
        turns = f * 8192 / (2 * math.pi)
        s = min(1.0, max(0.0, (turns - 1) / 3))
        assert same(got[i], (1 - s) * f / 8 + s * f)
    # whole turns vanish, backwards is forwards by the rest
    got = radians(bn.Rope(8, freqs=[2 * math.pi, -0.25, 7.0, 0.0]))
    assert min(got[0], 2 * math.pi - got[0]) < 1e-15 and abs(got[1] - (2 * math.pi - 0.25)) < 1e-14 and abs(got[2] - (7 - 2 * math.pi)) < 1e-14 and got[3] == 0
    assert bn.Rope(8, magnitude=0.0).desc.magnitude == 1.0
    for bad in (dict(rot=7), dict(rot=8, layout="x"), dict(rot=8, scaling="x"), dict(rot=8, freqs=[1.0])):
        with pytest.raises(bn.BitnetError):
            bn.Rope(**bad)


def test_calls_refuse_what_was_not_initialised(L):
    cache, rope = bn.KvCacheDesc(kv_heads=2, page_size=16, head_dim=64, layers=1, num_pages=8), bn.RopeDesc(rot_dim=64)
    p, r = C.addressof(cache), C.addressof(rope)
    assert L.bitnet_kv_append_rope(p, 0, r, FAKE, 4, 256, 64, FAKE, FAKE, 2, 128, 64, 1, FAKE, 4, FAKE, NULL, 1, FAKE, 2, NULL, NULL) == 1
    assert L.bitnet_attn_shared(p, 0, FAKE, 0, 4, 256, 64, FAKE, 4, FAKE, 1, FAKE, FAKE, 1, 0.1, 0, 0, FAKE, FAKE, 1 << 30, NULL, NULL) == 1
    assert L.bitnet_kv_append_rope(None, 0, r, FAKE, 4, 256, 64, FAKE, FAKE, 2, 128, 64, 1, FAKE, 4, FAKE, NULL, 1, FAKE, 2, NULL, NULL) == 1


def test_shared_workspace_sizes(L):
    f = bn.bitnet_attn_shared_workspace_bytes
    assert f(0, 32, 8, 128) > bn.bitnet_attn_workspace_bytes(0, 32, 8, 128)
    assert f(64, 64, 8, 128) - f(0, 64, 8, 128) == 64 * 64 * 1056
    assert f(1, 30, 8, 128) == 0 and f(-1, 32, 8, 128) == 0 and f(1, 32, 8, 132) == 0 and f(1, 0, 1, 64) == 0
