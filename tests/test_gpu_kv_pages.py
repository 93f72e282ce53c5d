"""The paged cache's books and moves against a plain implementation on the host: bits and counts have to be equal."""
import random

import pytest
import torch

import paper_2502_11880_b200 as bn

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Books:
    """The same state on the host and on the device."""

    def __init__(self, seqs, width, pages, heads, page, dim, dtype=BF, layers=2, nhd=False, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dp = -(-dim // 8) * 8
        shape = (layers, pages, page, heads, dp) if nhd else (layers, pages, heads, page, dp)
        self.full = [torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2)]
        pools = [t.permute(0, 1, 3, 2, 4) if nhd else t for t in self.full]
        self.k, self.v = (t[..., :dim] for t in pools)
        self.rows_k, self.rows_v = pools                   # rows with their padding, which pages carry along
        self.page, self.pages, self.dim = page, pages, dim
        self.hk, self.hv = self.rows_k.cpu().clone(), self.rows_v.cpu().clone()
        self.cache = bn.KvCache(self.k, self.v)
        self.refs, self.table, self.len = [0] * pages, [[-1] * width for _ in range(seqs)], [0] * seqs
        self.d_refs, self.d_table, self.d_len = i32(self.refs), i32(self.table), i32(self.len)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def load(self):
        self.d_refs.copy_(i32(self.refs))
        self.d_table.copy_(i32(self.table))
        self.d_len.copy_(i32(self.len))

    def free_page(self):
        for i, r in enumerate(self.refs):
            if r == 0:
                return i
        return None

    def reserve(self, to):
        for s, (a, b) in enumerate(zip(self.len, to)):
            for e in range(-(-a // self.page), min(len(self.table[s]), -(-b // self.page))):
                p = self.free_page()
                self.table[s][e] = -1 if p is None else p
                if p is not None:
                    self.refs[p] = 1

    def fork(self, parents, children):
        for p, c in zip(parents, children):
            n = self.len[p]
            self.table[c] = [-1] * len(self.table[c])
            for e in range(n // self.page):
                self.table[c][e] = self.table[p][e]
                if self.table[p][e] >= 0:
                    self.refs[self.table[p][e]] += 1
            self.len[c] = n
        for p, c in zip(parents, children):
            rows, e = self.len[p] % self.page, self.len[p] // self.page
            if rows and self.table[p][e] >= 0:
                to = self.free_page()
                if to is None:
                    continue
                self.refs[to] = 1
                self.table[c][e] = to
                for t in (self.hk, self.hv):
                    t[:, to, :, :rows] = t[:, self.table[p][e], :, :rows]

    def release(self, s, keep=lambda e: False):
        for e, p in enumerate(self.table[s]):
            if p >= 0 and not keep(e):
                self.refs[p] -= 1
                self.table[s][e] = -1

    def trim(self, window, sinks):
        for s in range(len(self.table)):
            self.release(s, lambda e: e * self.page < sinks or (e + 1) * self.page > self.len[s] - window)

    def put(self, layer, page, row, k, v):
        """One token's rows; their padding becomes 0."""
        for pool, x in ((self.hk, k), (self.hv, v)):
            pool[layer, page, :, row] = 0
            pool[layer, page, :, row, :self.dim] = x.to(pool.dtype).cpu()

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        src = [i for i in range(live, self.pages) if self.refs[i] > 0]
        dst = [i for i in range(live) if self.refs[i] == 0]
        for a, b in zip(src, dst):
            for t in (self.hk, self.hv):
                t[:, b] = t[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        place = dict(zip(src, dst))
        self.table = [[place.get(p, p) for p in row] for row in self.table]
        return live

    def check(self, status=0):
        torch.cuda.synchronize()
        assert self.d_refs.tolist() == self.refs
        assert self.d_table.tolist() == self.table
        assert self.d_len.tolist() == self.len
        for now, want in ((self.rows_k, self.hk), (self.rows_v, self.hv)):
            assert torch.equal(now.cpu().view(torch.int16), want.view(torch.int16))
        assert int(self.status) == status


SHAPES = [(2, 16, 64, BF, False), (1, 8, 100, HF, False), (3, 32, 128, HF, True), (4, 16, 36, BF, True), (1, 256, 4, BF, False)]


@pytest.mark.parametrize("heads,page,dim,dtype,nhd", SHAPES)
def test_life_of_a_pool(heads, page, dim, dtype, nhd):
    """Random growth, forks, releases, trims and compactions, compared after every step."""
    rng = random.Random(heads * page + dim)
    width, seqs = 6, 9
    b = Books(seqs, width, 40, heads, page, dim, dtype, nhd=nhd, seed=dim)
    for step in range(30):
        empty = [s for s in range(seqs) if b.len[s] == 0]
        busy = [s for s in range(seqs) if b.len[s] > 0]
        op = rng.choice(["grow", "grow", "fork", "free", "trim", "compact"])
        if op == "grow":
            to = [min(width * page, n + rng.choice([0, 1, page, rng.randrange(3 * page)])) if rng.random() < 0.5 else n for n in b.len]
            if sum(-(-t // page) - -(-n // page) for t, n in zip(to, b.len)) > b.refs.count(0):
                continue
            d_to, d_from = i32(to), b.d_len.clone()
            b.reserve(to)
            b.len = to
            bn.bitnet_kv_reserve(b.d_refs, b.d_table, d_from, d_to, page, dev_status=b.status)
            b.d_len.copy_(d_to)
        elif op == "fork" and busy and empty:
            children = rng.sample(empty, rng.randint(1, len(empty)))
            if len(children) > b.refs.count(0):
                continue
            parents = [rng.choice(busy) for _ in children]
            b.fork(parents, children)
            bn.bitnet_kv_fork(b.cache, b.d_refs, b.d_table, b.d_len, i32(parents), i32(children), dev_status=b.status)
        elif op == "free" and busy:
            rows = rng.sample(busy, rng.randint(1, len(busy) // 2 + 1))
            for s in rows:
                b.release(s)
                b.len[s] = 0
            bn.bitnet_kv_free(b.d_refs, b.d_table, b.d_len, i32(rows + rows[:1]), dev_status=b.status)   # listed twice: released once
        elif op == "trim":
            window, sinks = rng.randint(1, 3 * page), rng.choice([0, 1, page, page + 1])
            b.trim(window, sinks)
            bn.bitnet_kv_trim(b.d_refs, b.d_table, b.d_len, page, window, sinks)
        elif op == "compact":
            live = torch.zeros(1, dtype=torch.int32, device="cuda")
            want = b.compact()
            bn.bitnet_kv_compact(b.cache, b.d_refs, b.d_table, live=live)
            assert int(live) == want
        b.check()


@pytest.mark.parametrize("pages", [1, 1023, 4097, 20000])
def test_pools_of_many_pages(pages):
    """More pages than one step of the scans; holes everywhere; children by the hundred."""
    rng = random.Random(pages)
    seqs, width = 300, 4
    b = Books(seqs, width, pages, 1, 8, 8, layers=1, seed=1)
    for p in range(pages):
        if rng.random() < 0.7:
            b.refs[p] = 1
    held = [p for p in range(pages) if b.refs[p]]
    rng.shuffle(held)
    for s in range(100):
        n = rng.randint(0, min(2, len(held)))
        b.table[s][:n] = [held.pop() for _ in range(n)]
        b.len[s] = 8 * n - rng.randint(0, 7) if n else 0
    b.load()
    want = [b.len[s] for s in range(seqs)]
    for s in range(100):
        want[s] = min(32, b.len[s] + rng.randint(0, 9))
    short = sum(-(-w // 8) - -(-n // 8) for w, n in zip(want, b.len)) > b.refs.count(0)
    d_from = b.d_len.clone()
    b.reserve(want)
    bn.bitnet_kv_reserve(b.d_refs, b.d_table, d_from, i32(want), 8, dev_status=b.status)
    b.check(8 if short else 0)
    if short:
        return
    b.len = want
    b.load()
    children = list(range(100, 300))
    parents = [rng.randrange(100) for _ in children]
    short = sum(b.len[p] % 8 > 0 for p in parents) > b.refs.count(0)
    b.fork(parents, children)
    bn.bitnet_kv_fork(b.cache, b.d_refs, b.d_table, b.d_len, i32(parents), i32(children), dev_status=b.status)
    b.check(8 if short else 0)
    b.compact()
    bn.bitnet_kv_compact(b.cache, b.d_refs, b.d_table)
    b.check(8 if short else 0)


def test_reserve_for_more_rows_than_one_pass_plans():
    seqs, pages = 9000, 12000
    b = Books(seqs, 2, pages, 1, 8, 4, layers=1, seed=2)
    to = [(i * 5) % 17 for i in range(seqs)]
    free = iter(range(pages))
    for s, n in enumerate(to):
        for e in range(-(-n // 8)):
            if e < 2:
                p = next(free, None)
                b.table[s][e] = -1 if p is None else p
                if p is not None:
                    b.refs[p] = 1
    over = any(-(-n // 8) > 2 for n in to) or sum(min(2, -(-n // 8)) for n in to) > pages
    bn.bitnet_kv_reserve(b.d_refs, b.d_table, b.d_len, i32(to), 8, dev_status=b.status)
    b.check(8 if over else 0)


@pytest.mark.parametrize("heads,page,dim,dtype,nhd", SHAPES)
@pytest.mark.parametrize("io32", [True, False])
def test_append(heads, page, dim, dtype, nhd, io32):
    """Rows of several sequences, as slices of a fused matrix; rounding once, to nearest even."""
    spans = [(0, 3), (page - 1, 2), (5, 0), (2 * page, page), (7, 1)]
    b = Books(len(spans), 5, 24, heads, page, dim, dtype, nhd=nhd, seed=3)
    b.reserve([a + n for a, n in spans])
    b.len = [a + n for a, n in spans]
    b.load()
    tokens = sum(n for _, n in spans)
    start = [sum(n for _, n in spans[:i]) for i in range(len(spans) + 1)]
    g = torch.Generator(device="cuda").manual_seed(4)
    fused = torch.randn(tokens, 4 * heads * dim, generator=g, device="cuda").to(F32 if io32 else dtype)
    k = fused[:, 2 * heads * dim:3 * heads * dim].view(tokens, heads, dim)
    v = fused[:, 3 * heads * dim:].view(tokens, heads, dim)
    for s, (a, n) in enumerate(spans):
        for j in range(n):
            p, row = b.table[s][(a + j) // page], (a + j) % page
            b.put(1, p, row, k[start[s] + j], v[start[s] + j])
    bn.bitnet_kv_append(b.cache, 1, k, v, b.d_table, b.d_len, i32(start), dev_status=b.status)
    b.check()
    # one token each: no q_start
    one = fused[:len(spans)]
    k, v = one[:, :heads * dim].view(-1, heads, dim), one[:, heads * dim:2 * heads * dim].view(-1, heads, dim)
    for s, (a, n) in enumerate(spans):
        p = a + n - 1
        b.put(0, b.table[s][p // page], p % page, k[s], v[s])
    bn.bitnet_kv_append(b.cache, 0, k, v, b.d_table, b.d_len, dev_status=b.status)
    b.check()


def test_append_of_16_bit_rows_at_multiples_of_8_bytes():
    b = Books(2, 1, 4, 3, 8, 24, seed=9)
    b.table, b.len, b.refs = [[2], [0]], [3, 1], [1, 0, 1, 0]
    b.load()
    fused = torch.randn(2, 4 + 6 * 24 + 4, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(BF)
    k, v = fused[:, 4:4 + 72].view(2, 3, 24), fused[:, 76:148].view(2, 3, 24)
    assert k.data_ptr() % 16 == 8
    b.put(1, 2, 2, k[0], v[0])
    b.put(1, 0, 0, k[1], v[1])
    bn.bitnet_kv_append(b.cache, 1, k, v, b.d_table, b.d_len, dev_status=b.status)
    b.check()


def test_append_to_no_page_is_reported_and_writes_nothing():
    b = Books(3, 2, 6, 1, 8, 8, seed=5)
    b.table, b.len = [[0, -1], [6, 0], [1, 2]], [9, 3, 17]      # no page; beyond the pool; beyond the table
    b.load()
    k = torch.ones(3, 1, 8, device="cuda")
    bn.bitnet_kv_append(b.cache, 0, k, k, b.d_table, b.d_len, dev_status=b.status)
    b.check(7)
    b.len = [0, -5, 0]                                           # positions before the start: skipped
    b.load()
    b.status.zero_()
    bn.bitnet_kv_append(b.cache, 0, k, k, b.d_table, b.d_len, dev_status=b.status)
    b.check()


@pytest.mark.parametrize("heads,page,dim,dtype,nhd", SHAPES)
def test_copy_pages(heads, page, dim, dtype, nhd):
    b = Books(1, 1, 20, heads, page, dim, dtype, layers=3, nhd=nhd, seed=6)
    src, dst = [3, 3, 19, 0], [5, 7, 1, 18]
    for a, c in zip(src, dst):
        b.hk[:, c], b.hv[:, c] = b.hk[:, a], b.hv[:, a]
    bn.bitnet_kv_copy_pages(b.cache, i32(src), i32(dst), dev_status=b.status)
    b.check()
    bn.bitnet_kv_copy_pages(b.cache, i32([0, -1, 20]), i32([20, 2, 4]), dev_status=b.status)   # nothing is moved
    b.check(7)


def test_fork_without_free_pages_and_with_bad_rows():
    b = Books(4, 2, 3, 1, 8, 8, seed=7)
    b.table, b.len, b.refs = [[0, 1], [-1, -1], [-1, -1], [-1, -1]], [12, 0, 0, 0], [1, 1, 0]
    b.load()
    b.fork([0, 0], [1, 2])
    bn.bitnet_kv_fork(b.cache, b.d_refs, b.d_table, b.d_len, i32([0, 0]), i32([1, 2]), dev_status=b.status)
    b.check(8)
    assert b.table[1] == [0, 2] and b.table[2] == [0, -1]
    b.status.zero_()
    bn.bitnet_kv_fork(b.cache, b.d_refs, b.d_table, b.d_len, i32([9, -1, 0]), i32([3, 3, 4]), dev_status=b.status)
    b.check(7)
    b.status.zero_()
    bn.bitnet_kv_free(b.d_refs, b.d_table, b.d_len, i32([-1, 4]), dev_status=b.status)
    b.check(7)


def test_copy_offsets_beyond_32_bits():
    pages, page, dim = 70000, 64, 128
    k, v = (torch.empty(1, pages, 4, page, dim, dtype=BF, device="cuda") for _ in range(2))
    k[0, 5].normal_()
    v[0, 5].normal_()
    cache = bn.KvCache(k, v)
    bn.bitnet_kv_copy_pages(cache, i32([5]), i32([pages - 1]))
    assert torch.equal(k[0, 5], k[0, -1]) and torch.equal(v[0, 5], v[0, -1])
    x = torch.randn(1, 4, dim, device="cuda")
    bn.bitnet_kv_append(cache, 0, x, 2 * x, i32([[pages - 1]]), i32([page]))
    assert torch.equal(k[0, -1, :, -1], x[0].to(BF)) and torch.equal(v[0, -1, :, -1], (2 * x[0]).to(BF))


def test_refusals():
    b = Books(2, 2, 4, 1, 8, 8, seed=8)
    one = i32([0])
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_reserve(b.d_refs.long(), b.d_table, b.d_len, b.d_len, 8)
    with pytest.raises(bn.BitnetError, match="shape"):
        bn.bitnet_kv_reserve(b.d_refs, b.d_table, b.d_len, b.d_len, 12)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_trim(b.d_refs, b.d_table, b.d_len, 8, 0)
    with pytest.raises(bn.BitnetError, match="workspace"):
        bn.bitnet_kv_compact(b.cache, b.d_refs, b.d_table, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))
    with pytest.raises(bn.BitnetError, match="workspace"):
        bn.bitnet_kv_fork(b.cache, b.d_refs, b.d_table, b.d_len, one, i32([1]), workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_fork(b.cache, b.d_refs[:3], b.d_table, b.d_len, one, i32([1]))
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_copy_pages(b.cache, one, i32([1, 2]))
    none = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    nothing = torch.empty(0, dtype=torch.int32, device="cuda")
    bn.bitnet_kv_reserve(b.d_refs, none, nothing, nothing, 8)                        # nothing to do
    bn.bitnet_kv_trim(b.d_refs, none, nothing, 8, 5)
    bn.bitnet_kv_free(b.d_refs, b.d_table, b.d_len, nothing)
    bn.bitnet_kv_fork(b.cache, b.d_refs, b.d_table, b.d_len, nothing, nothing)
    bn.bitnet_kv_copy_pages(b.cache, nothing, nothing)
    bn.bitnet_kv_append(b.cache, 0, torch.empty(0, 1, 8, device="cuda"), torch.empty(0, 1, 8, device="cuda"), none, nothing)
    with pytest.raises(bn.BitnetError):
        bn.KvCache(torch.zeros(1, 2, 1, 8, 8, dtype=BF, device="cuda"), torch.zeros(1, 2, 1, 8, 8, dtype=BF))
    x = torch.zeros(2, 1, 8, device="cuda")
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_append(b.cache, 2, x, x, b.d_table, b.d_len)                    # no such layer
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_append(b.cache, 0, x.to(HF), x.to(HF), b.d_table, b.d_len)      # another 16-bit type
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_append(b.cache, 0, x, x.to(BF), b.d_table, b.d_len)
    with pytest.raises(bn.BitnetError):
        bn.bitnet_kv_append(b.cache, 0, x[:1], x[:1], b.d_table, b.d_len)            # tokens without q_start: one per sequence
