"""The largest pages and pools that a handle takes: what the kernels count in 32 bits stays below 2^31."""
import ctypes as C

import pytest

import paper_2502_11880_b200 as bn
from paper_2502_11880_b200 import build as bn_build
from test_kv_abi import desc


@pytest.fixture(scope="module")
def L():
    bn_build.build()
    return bn.lib()


def code(L, **kw):
    d = desc(**kw)
    rc = L.bitnet_kv_cache_init(C.byref(d))
    assert d.ready == 0
    return rc


@pytest.mark.parametrize("heads,page", [(127, 1 << 20), ((1 << 24) - 8, 8), ((1 << 21) - 1, 64)])
def test_pages_up_to_the_limit_pass_the_check(L, heads, page):
    """These are refused later only, for addresses that are no device's."""
    assert heads * page * 16 + 1023 < 2 ** 31
    assert code(L, kv_heads=heads, page_size=page) not in (0, 2)


@pytest.mark.parametrize("heads,page", [(128, 1 << 20), ((1 << 24) - 1, 8), ((1 << 24) - 7, 8), (1 << 21, 64), (1 << 30, 8)])
def test_pages_beyond_are_refused(L, heads, page):
    """A block that copies a page in steps of 1024 pieces forms indices up to 1024 beyond the last one: they must not pass 2^31."""
    assert heads * page * 16 + 1023 >= 2 ** 31
    assert code(L, kv_heads=heads, page_size=page) == 2
