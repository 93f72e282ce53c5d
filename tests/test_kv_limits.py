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


MOST = 2 ** 31 - 8193


def test_counts_up_to_the_limit(L):
    """Kernels step up to 8191 beyond the last page, row or token before they compare: the index must stay below 2^31."""
    from test_kv_abi import FAKE, NULL
    assert code(L, num_pages=MOST) not in (0, 1) and code(L, num_pages=MOST + 1) == 1
    assert L.bitnet_kv_workspace_bytes(MOST, MOST) > 0
    assert L.bitnet_kv_workspace_bytes(MOST + 1, 0) == 0 and L.bitnet_kv_workspace_bytes(1, MOST + 1) == 0
    assert L.bitnet_attn_workspace_bytes(MOST + 1, 8, 8, 64) == 0
    # (nothing to do, but for the count)
    assert L.bitnet_kv_reserve(FAKE, MOST, NULL, 0, 4, NULL, NULL, 16, NULL, NULL) == 0
    assert L.bitnet_kv_reserve(FAKE, MOST + 1, NULL, 0, 4, NULL, NULL, 16, NULL, NULL) == 1
    assert L.bitnet_kv_free(FAKE, 8, FAKE, MOST, 4, FAKE, FAKE, 0, NULL, NULL) == 0
    assert L.bitnet_kv_free(FAKE, 8, FAKE, MOST + 1, 4, FAKE, FAKE, 0, NULL, NULL) == 1
    assert L.bitnet_kv_free(FAKE, 8, FAKE, 1, 4, FAKE, FAKE, MOST + 1, NULL, NULL) == 1
