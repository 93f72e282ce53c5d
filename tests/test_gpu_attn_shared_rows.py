"""Which row of the table a shared prefix is read through, where rows of its group are empty or have given up pages; one long sequence among many short ones."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from kv_ref import attn_ref, check_attn
from test_gpu_attn_shared import BF, HF, PROMPT_P, Groups, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=["as it goes", "always shared"])
def path(request):
    bn.bitnet_debug_attn_shared(request.param == "always shared")
    yield request.param
    bn.bitnet_debug_attn_shared(False)


def check(s, q, window=0, sinks=0):
    """Against 64 bits, through every sequence's own row; nothing is reported, rows without tokens are 0."""
    status, scale = ints([0]), s.cache.head_dim ** -0.5
    out = bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, window=window, sinks=sinks, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and bn.bitnet_device_status() == 0
    lens = s.len.tolist()
    check_attn(out, attn_ref(s.k[1], s.v[1], q, s.table, [n - 1 for n in lens], range(len(lens)), scale, window, sinks), PROMPT_P[s.cache.dtype])
    assert all(bool((out[i] == 0).all()) for i, n in enumerate(lens) if n == 0)


def free(s, rows):
    """As bitnet_kv_free leaves them."""
    for i in rows:
        s.len[i] = 0
        s.table[i] = -1


@pytest.mark.parametrize("gone", [[0], [0, 1, 2], [0, 3, 6], [1, 5]])
def test_a_finished_sample_does_not_take_its_group_along(gone):
    """Samples end one after the other, the first ones too; the others go on."""
    for groups, hq, hkv, dim, page, dtype in (([(333, [340, 345, 401, 390]), (128, [129, 200, 150])], 8, 2, 128, 16, BF),
                                              ([(300, [320, 333, 310, 301]), (77, [80, 99, 90])], 4, 4, 96, 32, HF)):
        s = Groups(groups, hkv, dim, page, dtype, seed=31)
        free(s, gone)
        check(s, s.queries(hq))


def test_the_first_of_many_that_has_tokens():
    """More sequences than are looked at at a time, in several items; all of another group are gone."""
    s = Groups([(200, [210 + i % 50 for i in range(90)]), (64, [70, 80])], 1, 64, 16, BF, seed=32)
    free(s, [*range(70), 90, 91])
    check(s, s.queries(8))


def trimmed(s, window, sinks):
    """As bitnet_kv_trim leaves the table, each row by its own length; what is given up holds anything."""
    page = s.cache.page_size
    kept = set()
    for i, n in enumerate(s.len.tolist()):
        for e in range(-(-n // page)):
            if e * page >= sinks and (e + 1) * page <= n - window:
                s.table[i, e] = -1
        kept |= set(s.table[i].tolist())
    gone = [p for p in range(s.cache.num_pages) if p not in kept]
    for t in (s.k, s.v):
        t[1, gone] = float("nan")


@pytest.mark.parametrize("sinks", [0, 5])
def test_an_empty_row_does_not_undo_the_window(sinks):
    """What left the windows was given up: a row without tokens in the group (a padded batch) does not ask for it."""
    for idle in ([2], [0], [1, 3], [0, 1, 2, 3]):
        s = Groups([(900, [1000, 1000, 1000, 1000]), (640, [700] * 3)], 2, 64, 16, BF, seed=33)
        for i in idle:
            s.len[i], s.table[i] = 0, -1
        trimmed(s, 200, sinks)
        check(s, s.queries(8), window=200, sinks=sinks)


@pytest.mark.parametrize("window,sinks", [(200, 0), (200, 5), (64, 70), (333, 1)])
def test_rows_that_have_given_up_different_pages(window, sinks):
    """Sequences of very different lengths, each trimmed by its own: what one gave up another still sees."""
    for groups, hq, hkv, dim, page, dtype in (([(900, [1400, 950, 1000, 930])], 8, 2, 64, 16, BF),
                                              ([(900, [1400, 300, 1000, 600, 20]), (640, [700, 641])], 8, 8, 96, 32, HF),         # gaps between windows
                                              ([(910, [2000, 905, 0, 1050, 911])], 8, 2, 128, 16, BF),                             # part of a page
                                              ([(1200, [1900 - 12 * i for i in range(80)])], 4, 1, 64, 128, BF),                   # several items
                                              ([(1200, [1900, 1700, 1210])], 4, 1, 64, 256, HF)):
        s = Groups(groups, hkv, dim, page, dtype, seed=34)
        trimmed(s, window, sinks)
        check(s, s.queries(hq), window=window, sinks=sinks)


def test_one_long_sequence_among_many(path):
    """More rows than warps, one of them with nearly all tokens: it is taken by all warps, not by one after the other."""
    s = Groups([(64, [70 + i % 30 for i in range(600)]), (0, [9000])], 4, 64, 16, BF, seed=35)
    q = s.queries(8)
    check(s, q)
    if path == "always shared":
        ws, out = bn.new_attn_shared_workspace(601, 8, 4, 64), torch.empty_like(q)
        # some 48 us where its 563 tiles of a head are shared out, 390 where a warp has them all; the decode kernel takes 46
        times = []
        for run in (lambda: bn.bitnet_attn_shared(s.cache, 1, q, s.table, s.len, s.start, s.prefix, out=out, workspace=ws),
                    lambda: bn.bitnet_attn_decode(s.cache, 1, q, s.table, s.len, out=out, workspace=ws)):
            best = float("inf")
            for _ in range(20):
                a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
                a.record()
                run()
                b.record()
                torch.cuda.synchronize()
                best = min(best, a.elapsed_time(b))
            times.append(best)
        assert times[0] < 2 * times[1], times
