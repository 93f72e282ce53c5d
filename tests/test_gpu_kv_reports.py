"""What only the device sees -- positions beyond the table, pages beyond the pool -- and what the calls then do and report."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from kv_ref import check_attn
from test_gpu_kv_attn import BF, DECODE_P, F32, HF, PROMPT_P, Paged, prompt_args
from test_gpu_kv_pages import Books, i32

pytestmark = pytest.mark.gpu


def as_held(position, held, window, sinks):
    """(position, window, sinks) of a query inside a table of `held` tokens that sees what one at `position`, perhaps beyond, sees of them."""
    if position < held:
        return position, window, sinks
    left = window - (position - (held - 1))                        # of the window, the tokens that the table holds
    if left > 0:
        return held - 1, left, sinks
    return min(sinks, held) - 1, 0, 0                              # the sinks alone


def refs(p, q, positions, held, window, sinks):
    parts = []
    for i, pos in enumerate(positions):
        a, w, s = as_held(pos, held, window, sinks)
        parts.append(p.ref(q[i:i + 1], [a], [0], q.shape[2] ** -0.5, w, s))
    return tuple(torch.cat(x) for x in zip(*parts))


@pytest.mark.parametrize("io", [BF, F32])
@pytest.mark.parametrize("length,window,sinks", [(129, 100, 4), (200, 100, 4), (200, 100, 0), (227, 100, 0), (228, 100, 3), (5000, 1, 70),
                                                 (2 ** 31 - 1, 40, 5), (2 ** 31 - 1, 40, 0), (300, 10, 1000), (140, 2 ** 31 - 1, 0)])
def test_decode_window_of_a_position_beyond_the_table(length, window, sinks, io):
    """The window ends at the query, not at the table's end: what it has of the table's tokens is seen, and the call reports."""
    p = Paged([128], 2, 64, 16, BF, seed=41)
    p.table = p.table[:, :8].contiguous()
    p.len[0] = length
    q, status = p.queries(1, 4, 64, io), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = bn.bitnet_attn_decode(p.cache, p.layer, q, p.table, p.len, window=window, sinks=sinks, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 7 and bn.bitnet_device_status() == 0
    check_attn(out, refs(p, q, [length - 1], 128, window, sinks), DECODE_P[BF, io == F32])


@pytest.mark.parametrize("room", [True, False])
@pytest.mark.parametrize("held,length,new,window,sinks", [(128, 140, 60, 30, 0), (128, 300, 60, 100, 3), (1000 // 16 * 16, 1100, 150, 70, 2),
                                                          (128, 2 ** 31 - 1, 5, 40, 0), (128, 2 ** 31 - 1, 5, 40, 130), (144, 400, 300, 64, 20),
                                                          (1600, 1700, 4, 1500, 0), (128, 200, 2, 100, 3)])
def test_prompt_window_of_positions_beyond_the_table(held, length, new, window, sinks, room):
    p = Paged([held], 2, 64, 16, HF, seed=42)
    p.table = p.table[:, :held // 16].contiguous()
    p.len[0] = length
    start, status = i32([0, new]), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = p.queries(new, 4, 64, HF)
    ws = bn.new_attn_workspace(new if room else 0, 4, 2, 64)
    out = bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, start, new, window=window, sinks=sinks, workspace=ws, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 7 and bn.bitnet_device_status() == 0
    check_attn(out, refs(p, q, range(length - new, length), held, window, sinks), PROMPT_P[HF])


@pytest.mark.parametrize("new", [2, 40])
def test_prompt_without_window_beyond_the_table_sees_all_of_it(new):
    p = Paged([128], 2, 64, 16, BF, seed=43)
    p.table = p.table[:, :8].contiguous()
    p.len[0] = 128 + new
    q, status = p.queries(new, 4, 64, BF), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, i32([0, new]), new, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    check_attn(out, p.ref(q, [127] * new, [0] * new, 0.125, 0, 0), PROMPT_P[BF])


def test_positions_inside_the_table_are_not_reported():
    """The last place of the table, and places before the start."""
    p = Paged([128, 3], 2, 64, 16, BF, seed=44)
    p.table = p.table[:, :8].contiguous()
    q, status = p.queries(12, 4, 64, BF), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = bn.bitnet_attn_prompt(p.cache, p.layer, q, p.table, p.len, i32([0, 5, 12]), 7, window=9, sinks=1, dev_status=status)
    bn.bitnet_attn_decode(p.cache, p.layer, q[:2], p.table, p.len, window=9, sinks=1, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    pos = [123 + j for j in range(5)] + [3 - 7 + j for j in range(7)]
    check_attn(out, p.ref(q, pos, [0] * 5 + [1] * 7, 0.125, 9, 1), PROMPT_P[BF])


@pytest.mark.parametrize("row,length,child", [
    ([0, 40, 1, -1], 24, [0, -1, 1, -1]),        # a full page beyond the pool: not shared
    ([0, 1, 40, -1], 20, [0, 1, -1, -1]),        # the page filled in part beyond the pool: not copied
    ([0, 1, -1, -1], 20, [0, 1, -1, -1]),        # the page filled in part is none
    ([0, 1, 2, 3], 33, [0, 1, 2, 3]),            # a length beyond the table: its row is shared up to its end
])
def test_fork_reports_what_it_cannot_take_over(row, length, child):
    b = Books(3, 4, 6, 1, 8, 8, seed=11)
    b.table[0], b.len[0] = row, length
    b.refs = [int(i in row) for i in range(6)]
    b.load()
    bn.bitnet_kv_fork(b.cache, b.d_refs, b.d_table, b.d_len, i32([0]), i32([2]), dev_status=b.status)
    b.table[2], b.len[2] = child, min(length, 32)
    for e, page in enumerate(child):
        if page >= 0:
            b.refs[page] += 1
    b.check(7)


def test_fork_does_not_report_released_pages():
    b = Books(2, 4, 6, 1, 8, 8, seed=12)
    b.table[0], b.len[0], b.refs = [0, -1, 1, 3], 29, [1, 1, 0, 1, 0, 0]
    b.load()
    b.fork([0], [1])
    bn.bitnet_kv_fork(b.cache, b.d_refs, b.d_table, b.d_len, i32([0]), i32([1]), dev_status=b.status)
    b.check()


def test_free_reports_pages_beyond_the_pool():
    b = Books(2, 4, 6, 1, 8, 8, seed=13)
    b.table, b.len, b.refs = [[0, 6, -1, 2 ** 31 - 1], [1, -1, -1, -1]], [25, 3], [1, 1, 0, 0, 0, 0]
    b.load()
    bn.bitnet_kv_free(b.d_refs, b.d_table, b.d_len, i32([0]), dev_status=b.status)
    b.table[0], b.len[0], b.refs[0] = [-1] * 4, 0, 0
    b.check(7)
    b.status.zero_()
    bn.bitnet_kv_free(b.d_refs, b.d_table, b.d_len, i32([1, 0]), dev_status=b.status)
    b.table[1], b.len[1], b.refs[1] = [-1] * 4, 0, 0
    b.check()
