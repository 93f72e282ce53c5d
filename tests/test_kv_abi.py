"""Cache and attention entry points without a GPU: argument checks return status codes before anything is launched, the compiled
binding and its mirror of the handle fit the library."""
import ctypes as C
import math
import os

import pytest
import torch

import paper_2502_11880_b200 as bn
from paper_2502_11880_b200 import build as bn_build

NULL, FAKE, ODD = C.c_void_p(None), C.c_void_p(4096), C.c_void_p(4098)     # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    bn_build.build()
    return bn.lib()


def desc(**kw):
    d = dict(dtype=0, kv_heads=2, page_size=16, head_dim=64, layers=1, num_pages=8, k=4096, v=8192, stride_layer=16384, stride_page=2048,
             stride_head=1024, stride_row=64)
    d.update(kw)
    return bn.KvCacheDesc(**d)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), 1), (dict(dtype=-1), 1), (dict(k=None), 1), (dict(v=4100), 1), (dict(kv_heads=0), 1), (dict(layers=0), 1),
    (dict(num_pages=0), 1), (dict(page_size=24), 2), (dict(page_size=4), 2), (dict(kv_heads=256, page_size=1 << 20), 2), (dict(page_size=1 << 21), 2), (dict(head_dim=0), 2),
    (dict(head_dim=130, stride_row=136), 2), (dict(head_dim=66, stride_row=72), 2), (dict(stride_row=56), 1), (dict(stride_row=68), 1),
    (dict(stride_page=2052), 1), (dict(stride_head=-1024), 1), (dict(stride_layer=1 << 40), 1)])
def test_handles_are_checked(L, change, code):
    d = desc(**change)
    assert L.bitnet_kv_cache_init(C.byref(d)) == code and d.ready == 0
    assert L.bitnet_kv_cache_init(None) == 1


def test_calls_refuse_handles_that_were_not_initialised(L):
    d = desc()
    p = C.addressof(d)
    assert L.bitnet_kv_append(p, 0, FAKE, FAKE, 2, 128, 64, 1, FAKE, 4, FAKE, NULL, 1, NULL, NULL) == 1
    assert L.bitnet_attn_decode(p, 0, FAKE, 2, 4, 256, 64, FAKE, 4, FAKE, 1, 0.1, 0, 0, FAKE, FAKE, 1 << 30, NULL, NULL) == 1
    assert L.bitnet_kv_fork(p, FAKE, FAKE, 4, 4, FAKE, FAKE, FAKE, 1, FAKE, 1 << 20, NULL, NULL) == 1
    assert L.bitnet_kv_compact(p, FAKE, FAKE, 4, 4, NULL, FAKE, 1 << 20, NULL) == 1
    assert L.bitnet_kv_copy_pages(p, FAKE, FAKE, 1, NULL, NULL) == 1
    assert L.bitnet_kv_append(None, 0, FAKE, FAKE, 2, 128, 64, 1, FAKE, 4, FAKE, NULL, 1, NULL, NULL) == 1


def test_books_are_checked(L):
    assert L.bitnet_kv_reserve(NULL, 8, FAKE, 1, 4, FAKE, FAKE, 16, NULL, NULL) == 1
    assert L.bitnet_kv_reserve(FAKE, 0, FAKE, 1, 4, FAKE, FAKE, 16, NULL, NULL) == 1
    assert L.bitnet_kv_reserve(FAKE, 8, FAKE, -1, 4, FAKE, FAKE, 16, NULL, NULL) == 1
    assert L.bitnet_kv_reserve(FAKE, 8, NULL, 0, 4, NULL, NULL, 16, NULL, NULL) == 0   # no rows
    assert L.bitnet_kv_reserve(FAKE, 8, FAKE, 1, 4, ODD, FAKE, 16, NULL, NULL) == 1
    assert L.bitnet_kv_reserve(FAKE, 8, FAKE, 1, 4, FAKE, FAKE, 10, NULL, NULL) == 2
    assert L.bitnet_kv_free(FAKE, 8, FAKE, 1, 4, FAKE, NULL, 1, NULL, NULL) == 1
    assert L.bitnet_kv_free(FAKE, 8, FAKE, 1, 4, FAKE, FAKE, -1, NULL, NULL) == 1
    assert L.bitnet_kv_free(FAKE, 8, FAKE, 1, 4, FAKE, FAKE, 0, NULL, NULL) == 0       # nothing to do: nothing is launched
    assert L.bitnet_kv_trim(FAKE, 8, FAKE, 1, 4, FAKE, 16, 0, 0, NULL) == 1
    assert L.bitnet_kv_trim(FAKE, 8, FAKE, 1, 4, FAKE, 16, 5, -1, NULL) == 1


def test_workspace_sizes(L):
    decode, prompt = bn.bitnet_attn_workspace_bytes(0, 32, 8, 128), bn.bitnet_attn_workspace_bytes(512, 32, 8, 128)
    assert 65536 < decode < 2 << 20 < prompt < 64 << 20
    assert bn.bitnet_attn_workspace_bytes(1, 30, 8, 128) == 0 and bn.bitnet_attn_workspace_bytes(-1, 32, 8, 128) == 0
    assert bn.bitnet_attn_workspace_bytes(1, 32, 8, 132) == 0
    assert bn.bitnet_kv_workspace_bytes(100, 0) >= 100 * 20 and bn.bitnet_kv_workspace_bytes(0, 1) == 0
    assert bn.bitnet_kv_workspace_bytes(1, 1000) >= 16000


def test_status_texts_of_the_books(L):
    assert len({bn.status_string(rc) for rc in range(9)}) == 9 and "unknown status" not in [bn.status_string(rc) for rc in range(9)]


def test_compiled_binding_refuses_what_is_no_cuda_tensor(L):
    cpu = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(bn.BitnetError, match="refs"):
        bn.bitnet_kv_reserve(cpu, cpu.view(2, 2), cpu, cpu, 16)
    with pytest.raises(bn.BitnetError, match="tensor"):
        bn.bitnet_kv_free(None, cpu.view(2, 2), cpu, cpu)
    d = desc()

    class Handle:
        ref, kv_heads, head_dim, scale, num_pages, device = C.addressof(d), 2, 64, 0.125, 8, "cpu"

    with pytest.raises(bn.BitnetError, match="q"):
        bn.bitnet_attn_decode(Handle, 0, torch.zeros(1, 4, 64), cpu.view(2, 2), cpu, workspace=torch.zeros(16))
    with pytest.raises(TypeError):
        bn._binding().kv_free(1, 2)
    with pytest.raises(bn.BitnetError):
        bn.KvCache(torch.zeros(1, 2, 2, 16, 64), torch.zeros(1, 2, 2, 16, 64))


def test_missing_binding_raises(monkeypatch, tmp_path):
    monkeypatch.setattr(bn, "_fast", None)
    monkeypatch.setattr(bn, "_PKG", str(tmp_path))
    with pytest.raises(bn.BitnetError, match="missing"):
        bn._binding()


def test_measured_cases_count_what_they_see():
    """The work of the measured cases against a count token by token."""
    import importlib.util
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("operators_cases", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    for window, sinks in ((0, 0), (1, 0), (5, 0), (5, 3), (7, 40), (100, 2)):
        for p in (0, 1, 4, 5, 6, 8, 30):
            seen = [c for c in range(p + 1) if not window or c > p - window or c < sinks]
            assert m._seen(p, window, sinks) == len(seen)
        for first, last in ((0, 3), (2, 20), (9, 9)):
            seen = {c for p in range(first, last + 1) for c in range(p + 1) if not window or c > p - window or c < sinks}
            assert m._span(first, last, window, sinks) == len(seen)
    assert all(math.isfinite(m.work(c)["bytes"]) and m.work(c)["bytes"] > 0 for c in m.listed())
