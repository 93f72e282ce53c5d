"""Measured cases of the paged key-value cache and the attention over it.

Five kinds of pass: "decode" (one new token per sequence over its pages), "prompt" (new tokens of prompts or chunks of
prompts, with an optional sliding window and sinks), "append" (pages for new tokens, their K and V rows written), "beam"
(sequences forked, the old ones freed) and "compact" (pages that left a window released, the rest moved together).

`own` selects the framework's entry points; otherwise the same results come from elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one user's token early in a chat, 8B-shaped layer (32 query heads, 8 kv heads of 128), q as the fp32 output of the Q/K/V linear
        dict(name="decode_1x517", kind="decode", seqs=1, ctx=517, ragged=0, heads=32, kv_heads=8, dim=128, dtype="bf16", io="f32", page=16,
             window=0, sinks=0),
        # a full serving batch of ragged contexts, 100B-shaped layer (64 query heads, 8 kv heads of 128)
        dict(name="decode_64x8192_ragged", kind="decode", seqs=64, ctx=8192, ragged=1, heads=64, kv_heads=8, dim=128, dtype="bf16", io="bf16",
             page=16, window=0, sinks=0),
        # one long document: few rows, all of the machine has to share one cache
        dict(name="decode_1x131072", kind="decode", seqs=1, ctx=131072, ragged=0, heads=64, kv_heads=8, dim=128, dtype="bf16", io="bf16",
             page=64, window=0, sinks=0),
        # 3B-shaped layer (32 heads of 100, no grouping) with a sliding window and sinks, odd ragged lengths
        dict(name="decode_window_9x16001", kind="decode", seqs=9, ctx=16001, ragged=2, heads=32, kv_heads=32, dim=100, dtype="f16", io="f32",
             page=32, window=4096, sinks=4),
        # a short question, 1536-wide layer (16 heads of 96)
        dict(name="prompt_77", kind="prompt", seqs=1, new=77, ctx=77, ragged=0, heads=16, kv_heads=16, dim=96, dtype="f16", page=16,
             window=0, sinks=0),
        # chunks of four prompts on top of what is cached, 8B-shaped layer, window and sinks
        dict(name="prompt_chunk_4x512", kind="prompt", seqs=4, new=512, ctx=5003, ragged=3, heads=32, kv_heads=8, dim=128, dtype="bf16",
             page=32, window=2048, sinks=16),
        # a long prompt of the 100B-shaped layer, window and sinks
        dict(name="prompt_8192", kind="prompt", seqs=1, new=8192, ctx=8192, ragged=0, heads=64, kv_heads=8, dim=128, dtype="bf16", page=64,
             window=4096, sinks=4),
        # one decode step's new rows, 3B-shaped layer
        dict(name="append_32x1", kind="append", seqs=32, new=1, ctx=2048, ragged=4, heads=32, kv_heads=32, dim=100, dtype="f16", io="f32", page=16),
        # prompts of a batch, 8B-shaped layer
        dict(name="append_4x2048", kind="append", seqs=4, new=2048, ctx=4099, ragged=5, heads=32, kv_heads=8, dim=128, dtype="bf16", io="f32", page=32),
        # parallel samples of one answer
        dict(name="beam_1to4", kind="beam", seqs=1, children=4, ctx=701, ragged=0, kv_heads=8, dim=128, dtype="bf16", page=16, layers=4),
        # a step of beam search of a batch over many layers
        dict(name="beam_16to128", kind="beam", seqs=16, children=128, ctx=4000, ragged=6, kv_heads=8, dim=128, dtype="bf16", page=64, layers=16),
        # a pool that a windowed service has fragmented is packed, so that its end can be given back
        dict(name="compact_48x4096", kind="compact", seqs=48, ctx=4096, ragged=7, kv_heads=8, dim=128, dtype="bf16", page=32, layers=8,
             window=1024, sinks=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# head layouts: the 8B-, 100B-, 3B- and 1536-wide shapes, and a generic one
LAYOUTS = [(32, 8, 128), (64, 8, 128), (32, 32, 100), (16, 16, 96), (12, 4, 64)]


def draw(rng):
    kind = rng.choice(["decode", "decode", "prompt", "prompt", "append", "beam", "compact"])
    heads, kv_heads, dim = rng.choice(LAYOUTS)
    case = dict(kind=kind, ragged=rng.randrange(1, 1 << 20), dtype=rng.choice(["bf16", "f16"]), page=rng.choice([8, 16, 32, 64, 128]),
                heads=heads, kv_heads=kv_heads, dim=dim)
    windows = [(0, 0), (_log(rng, 16, 4096), rng.choice([0, 1, 4, 16, 33]))]
    if kind == "decode":
        seqs = _log(rng, 1, 96)
        # at most the bytes of the largest listed case
        case.update(seqs=seqs, ctx=_log(rng, 1, min(131072, 40 * 8192 * 1024 // (seqs * kv_heads * 128))), io=rng.choice(["f32", case["dtype"]]))
        case["window"], case["sinks"] = rng.choice(windows)
    elif kind == "prompt":
        seqs, new = _log(rng, 1, 8), _log(rng, 1, 4096)
        ctx = min(8192, new + rng.choice([0, _log(rng, 1, 8192)]))
        # the plain form holds seqs * heads * new * ctx scores: at most those of the largest listed case
        new = max(1, min(new, 64 * 8192 * 8192 // (3 * seqs * heads * ctx)))
        case.update(seqs=seqs, new=new, ctx=ctx)
        case["window"], case["sinks"] = rng.choice(windows)
    elif kind == "append":
        seqs = _log(rng, 1, 128)
        new = rng.choice([1, _log(rng, 1, max(1, 8192 // seqs))])
        case.update(seqs=seqs, new=new, ctx=new + rng.choice([0, _log(rng, 1, 4096)]), io=rng.choice(["f32", case["dtype"]]))
    elif kind == "beam":
        seqs, children, ctx = _log(rng, 1, 16), _log(rng, 1, 96), _log(rng, 1, 2048)
        # pools up to half the listed case's
        case.update(seqs=seqs, children=children, ctx=ctx, layers=min(_log(rng, 1, 16), max(1, 16 * 4000 * 16 * 512 // (kv_heads * dim * (seqs * ctx + children * case["page"])))))
        del case["heads"]
    else:
        seqs, ctx = _log(rng, 2, 48), _log(rng, 64, 3000)
        case.update(seqs=seqs, ctx=ctx, layers=min(_log(rng, 1, 8), max(1, 48 * 4096 * 8 * 512 // (kv_heads * dim * seqs * ctx))),
                    window=_log(rng, 16, 1024), sinks=rng.choice([0, 4, 16]))
        del case["heads"]
    return case


def lengths(case):
    """Tokens cached per sequence after the pass, and new tokens per sequence: given by the case alone."""
    n, ctx, new = case["seqs"], case["ctx"], case.get("new", 1)
    r = random.Random(case["ragged"])
    if not case["ragged"]:
        return [ctx] * n, [new] * n
    lens = [ctx] + [max(1, int(ctx * r.uniform(0.3, 1.0))) for _ in range(n - 1)]
    news = [new] + [max(1, int(new * r.uniform(0.5, 1.0))) for _ in range(n - 1)]
    if "new" in case:
        lens = [max(a, b) for a, b in zip(lens, news)]
    return lens, news


def pages_of(tokens, page):
    return -(-tokens // page)


# ---------------------------------------------------------------------------------------------- inputs
def _pool(case, layers, pages, g):
    shape = (layers, pages, case["kv_heads"], case["page"], -(-case["dim"] // 8) * 8)   # rows start at multiples of 16 bytes
    k = torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[case["dtype"]])
    v = torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[case["dtype"]])
    return k[..., :case["dim"]], v[..., :case["dim"]]


def prepare(case, seed):
    kind, page, hkv, dim = case["kind"], case["page"], case["kv_heads"], case["dim"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    lens, news = lengths(case)
    layers = case.get("layers", 1)
    rows = case["seqs"] + case.get("children", 0)
    width = pages_of(max(lens), page)
    before = [a - b for a, b in zip(lens, news)] if kind == "append" else lens
    need = sum(pages_of(n, page) for n in lens)
    extra = need // 8 + 8 + case.get("children", 0) if kind != "compact" else need // 4 + 8
    pages = need + extra
    s = dict(case=case, layers=layers, width=width, pages=pages)
    s["k"], s["v"] = _pool(case, layers, pages, g)
    # every sequence's pages, in the order in which a used pool gives them out: any
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    book = torch.zeros(pages + rows + rows * width, dtype=torch.int32, device="cuda")
    s["book"], s["refs"], s["len"], s["table"] = book, book[:pages], book[pages:pages + rows], book[pages + rows:].view(rows, width)
    s["table"].fill_(-1)
    at = 0
    table = torch.full((rows, width), -1, dtype=torch.int32)
    order_host = order.cpu()
    for i, n in enumerate(before):
        c = pages_of(n, page)
        table[i, :c] = order_host[at:at + c]
        at += c
    s["table"].copy_(table)
    s["refs"][order[:at].long()] = 1
    s["len"][:len(before)] = torch.tensor(before, dtype=torch.int32, device="cuda")
    if kind in ("append", "beam", "compact"):
        s["book0"] = book.clone()      # a pass begins with this state of the books
    if kind in ("decode", "prompt"):
        hq = case["heads"]
        tokens = sum(news)
        q = torch.randn(tokens, hq, dim, generator=g, device="cuda")
        # the first tokens draw attention, as they do in trained models
        pull = torch.randn(hkv, dim, generator=g, device="cuda")
        s["k"][0][s["table"][:, 0].long(), :, :4] += (0.7 * pull).to(s["k"].dtype)[None, :, None]
        q += 0.7 * pull.repeat_interleave(hq // hkv, 0)[None]
        s["q"] = q.to(DTYPES[case.get("io", case["dtype"])])
        s["scale"] = 1.0 / math.sqrt(dim)
        s["window"], s["sinks"] = case["window"], case["sinks"]
    if kind == "append":
        # the fused output of the Q/K/V linear: K and V are slices of its rows
        qkv = torch.randn(sum(news), (case["heads"] + 2 * hkv) * dim, generator=g, device="cuda").to(DTYPES[case["io"]])
        q_cols = case["heads"] * dim
        s["k_new"] = qkv[:, q_cols:q_cols + hkv * dim].view(-1, hkv, dim)
        s["v_new"] = qkv[:, q_cols + hkv * dim:].view(-1, hkv, dim)
        s["to_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["from_len"] = torch.tensor(before, dtype=torch.int32, device="cuda")
    if kind in ("prompt", "append"):
        s["q_start"] = torch.tensor([0] + [sum(news[:i + 1]) for i in range(len(news))], dtype=torch.int32, device="cuda")
        s["max_new"] = max(news)
    if kind == "beam":
        n = case["children"]
        s["parents"] = torch.randint(0, case["seqs"], (n,), generator=g, device="cuda", dtype=torch.int32)
        s["children"] = torch.arange(case["seqs"], rows, dtype=torch.int32, device="cuda")
        s["old"] = torch.arange(case["seqs"], dtype=torch.int32, device="cuda")
    if kind == "compact":
        # every third sequence has ended: its pages are holes
        gone = list(range(0, case["seqs"], 3))
        ids = s["table"][gone].flatten().long()
        s["refs"][ids[ids >= 0]] = 0
        s["table"][gone] = -1
        s["len"][gone] = 0
        s["book0"] = book.clone()
    if own:
        import paper_2502_11880_b200 as bn
        s["bn"] = bn
        s["cache"] = bn.KvCache(s["k"], s["v"])
        s["ws"] = None
        if kind in ("decode", "prompt"):
            s["ws"] = bn.new_attn_workspace(s["q"].shape[0], case["heads"], hkv, dim)
        elif kind in ("beam", "compact"):
            s["ws"] = bn.new_kv_workspace(pages, max(rows, 1))
    return s


# ---------------------------------------------------------------------------------------------- passes
def run(s):
    return (OWN if own else PLAIN)[s["case"]["kind"]](s)


def _own_decode(s):
    return s["bn"].bitnet_attn_decode(s["cache"], 0, s["q"], s["table"], s["len"], scale=s["scale"], window=s["window"], sinks=s["sinks"],
                                      workspace=s["ws"])


def _own_prompt(s):
    return s["bn"].bitnet_attn_prompt(s["cache"], 0, s["q"], s["table"], s["len"], s["q_start"], s["max_new"], scale=s["scale"],
                                      window=s["window"], sinks=s["sinks"], workspace=s["ws"])


def _own_append(s):
    s["book"].copy_(s["book0"])
    bn = s["bn"]
    bn.bitnet_kv_reserve(s["refs"], s["table"], s["from_len"], s["to_len"], s["case"]["page"])
    bn.bitnet_kv_append(s["cache"], 0, s["k_new"], s["v_new"], s["table"], s["to_len"], s["q_start"])
    return dict(k=s["k"], v=s["v"], refs=s["refs"], table=s["table"])


def _own_beam(s):
    s["book"].copy_(s["book0"])
    bn = s["bn"]
    bn.bitnet_kv_fork(s["cache"], s["refs"], s["table"], s["len"], s["parents"], s["children"], workspace=s["ws"])
    bn.bitnet_kv_free(s["refs"], s["table"], s["len"], s["old"])
    return dict(k=s["k"], v=s["v"], refs=s["refs"], table=s["table"], len=s["len"])


def _own_compact(s):
    s["book"].copy_(s["book0"])
    bn = s["bn"]
    bn.bitnet_kv_trim(s["refs"], s["table"], s["len"], s["case"]["page"], s["case"]["window"], s["case"]["sinks"])
    bn.bitnet_kv_compact(s["cache"], s["refs"], s["table"], workspace=s["ws"])
    return dict(k=s["k"], v=s["v"], refs=s["refs"], table=s["table"])


OWN = dict(decode=_own_decode, prompt=_own_prompt, append=_own_append, beam=_own_beam, compact=_own_compact)


def _gather(s, pool):
    """[sequences][kv heads][tokens][dim] in 32 bits, from the pages of layer 0."""
    got = pool[0][s["table"].clamp(min=0).long()].float()                       # S, P, H, page, D
    return got.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _softmax_sum(scores, visible, v):
    """Rows of softmax(scores where visible) @ v; a row that sees nothing is 0."""
    scores = scores.masked_fill(~visible, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return (p @ v) / torch.where(total == 0, torch.ones_like(total), total)


def _visible(position, columns, window, sinks):
    see = (columns <= position) & (position >= 0)
    if window:
        see = see & ((columns > position - window) | (columns < sinks))
    return see


def _plain_decode(s):
    k, v = _gather(s, s["k"]), _gather(s, s["v"])
    n, hkv, tokens, dim = k.shape
    q = s["q"].float().view(n, hkv, -1, dim) * s["scale"]
    columns = torch.arange(tokens, device="cuda")
    position = (s["len"] - 1).view(n, 1, 1, 1)
    v = v * (columns[:, None] <= position)
    out = _softmax_sum(q @ k.transpose(-1, -2), _visible(position, columns, s["window"], s["sinks"]), v)
    return out.reshape(s["q"].shape).to(s["q"].dtype)


def _plain_prompt(s):
    k, v = _gather(s, s["k"]), _gather(s, s["v"])
    n, hkv, tokens, dim = k.shape
    hq = s["q"].shape[1]
    start = s["q_start"].long()
    j = torch.arange(s["max_new"], device="cuda")
    row = torch.minimum(start[:-1, None] + j, start[-1] - 1)                      # S, T: rows past a sequence's end repeat others
    q = s["q"].float()[row] * s["scale"]                                          # S, T, Hq, D
    q = q.view(n, s["max_new"], hkv, hq // hkv, dim).permute(0, 2, 3, 1, 4).flatten(2, 3)
    new = (start[1:] - start[:-1])[:, None]
    position = s["len"][:, None] - new + j                                        # S, T
    position = position.view(n, 1, 1, -1).expand(n, 1, hq // hkv, -1).flatten(2, 3)[..., None]
    columns = torch.arange(tokens, device="cuda")
    v = v * (columns[:, None] < s["len"].view(n, 1, 1, 1))
    see = _visible(position, columns, s["window"], s["sinks"]) & (columns < s["len"].view(n, 1, 1, 1))
    out = _softmax_sum(q @ k.transpose(-1, -2), see, v)
    out = out.view(n, hkv, hq // hkv, -1, dim).permute(0, 3, 1, 2, 4).reshape(n, -1, hq, dim)
    return out[j < new].to(s["q"].dtype)


def _plain_append(s):
    s["book"].copy_(s["book0"])
    page = s["case"]["page"]
    table, refs = s["table"], s["refs"]
    i = torch.arange(s["width"], device="cuda")
    first, last = ((t[:, None] + page - 1) // page for t in (s["from_len"], s["to_len"]))
    wanted = (i >= first) & (i < last) & (table < 0)
    free = torch.nonzero(refs == 0).flatten()[:int(wanted.sum())]
    table[wanted] = free.to(torch.int32)
    refs[free] = 1
    token = torch.arange(s["k_new"].shape[0], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].contiguous(), token.to(torch.int32), right=True)
    position = s["to_len"][seq] - s["q_start"][seq + 1] + token
    at = table[seq, position // page].long()
    s["k"][0][at, :, position % page] = s["k_new"].to(s["k"].dtype)
    s["v"][0][at, :, position % page] = s["v_new"].to(s["v"].dtype)
    return dict(k=s["k"], v=s["v"], refs=refs, table=table)


def _plain_beam(s):
    s["book"].copy_(s["book0"])
    page, table, refs, length = s["case"]["page"], s["table"], s["refs"], s["len"]
    parents, children, old = s["parents"].long(), s["children"].long(), s["old"].long()
    used = length[parents]
    full = used // page
    i = torch.arange(s["width"], device="cuda")
    rows = torch.where(i < full[:, None], table[parents], torch.full_like(table[parents], -1))
    refs.index_add_(0, rows[rows >= 0].long(), torch.ones_like(rows[rows >= 0]))
    partial = torch.nonzero(used % page).flatten()
    fresh = torch.nonzero(refs == 0).flatten()[:partial.numel()]
    source = table[parents[partial], full[partial].long()].long()
    rows[partial, full[partial].long()] = fresh.to(torch.int32)
    refs[fresh] = 1
    in_use = (torch.arange(page, device="cuda") < (used % page)[partial][:, None])[None, :, None, :, None]
    for pool in (s["k"], s["v"]):
        pool[:, fresh] = torch.where(in_use, pool[:, source], pool[:, fresh])
    table[children] = rows
    length[children] = used
    ids = table[old]
    refs.index_add_(0, ids[ids >= 0].long(), -torch.ones_like(ids[ids >= 0]))
    table[old] = -1
    length[old] = 0
    return dict(k=s["k"], v=s["v"], refs=refs, table=table, len=length)


def _plain_compact(s):
    s["book"].copy_(s["book0"])
    page, table, refs, length = s["case"]["page"], s["table"], s["refs"], s["len"]
    i = torch.arange(s["width"], device="cuda")
    left = (i * page >= s["case"]["sinks"]) & ((i + 1) * page <= length[:, None] - s["case"]["window"]) & (table >= 0)
    ids = table[left].long()
    refs.index_add_(0, ids, torch.full_like(table[left], -1))
    table[left] = -1
    live = refs > 0
    index = torch.arange(s["pages"], device="cuda")
    count = live.sum()
    source, target = torch.nonzero(live & (index >= count)).flatten(), torch.nonzero(~live & (index < count)).flatten()
    for pool in (s["k"], s["v"]):
        pool[:, target] = pool[:, source]
    index[source] = target
    table.copy_(torch.where(table >= 0, index[table.clamp(min=0).long()].to(torch.int32), table))
    refs[target] = refs[source]
    refs[source] = 0
    return dict(k=s["k"], v=s["v"], refs=refs, table=table)


PLAIN = dict(decode=_plain_decode, prompt=_plain_prompt, append=_plain_append, beam=_plain_beam, compact=_plain_compact)


# ---------------------------------------------------------------------------------------------- work and exact values
def _seen(position, window, sinks):
    """Tokens that the query at `position` sees."""
    if position < 0:
        return 0
    if not window or position < window:
        return position + 1
    return window + min(sinks, position + 1 - window)


def _span(first, last, window, sinks):
    """Tokens that the queries at first..last see together."""
    low = max(0, first - window + 1) if window else 0
    return last + 1 - low + min(sinks, low)


def work(case):
    kind, page, hkv, dim = case["kind"], case["page"], case["kv_heads"], case["dim"]
    lens, news = lengths(case)
    row = hkv * dim * 2                                                           # bytes of one token's K (or V) in one layer
    if kind in ("decode", "prompt"):
        if kind == "decode":
            news = [1] * len(lens)
        io = {"f32": 4}.get(case.get("io"), 2)
        pairs = sum(_seen(p, case["window"], case["sinks"]) for a, b in zip(lens, news) for p in range(a - b, a))
        tokens = sum(_span(a - b, a - 1, case["window"], case["sinks"]) for a, b in zip(lens, news))
        return dict(bytes=2 * tokens * row + 2 * sum(news) * case["heads"] * dim * io + 4 * (tokens // page + 2 * len(lens)),
                    flops=4 * pairs * case["heads"] * dim)
    width, rows = pages_of(max(lens), page), case["seqs"] + case.get("children", 0)
    pages = sum(pages_of(n, page) for n in lens)
    if kind == "append":
        io = 4 if case["io"] == "f32" else 2
        fresh = sum(pages_of(a, page) - pages_of(a - b, page) for a, b in zip(lens, news))
        return dict(bytes=2 * sum(news) * hkv * dim * (io + 2) + 8 * fresh, flops=0)
    layers = case["layers"]
    if kind == "beam":
        # the average parent's part of a page, read and written, and the tables' rows
        part = sum(n % page for n in lens) / len(lens)
        return dict(bytes=case["children"] * part * 2 * row * layers * 2 + 8 * (rows * width + pages), flops=0)
    kept = 0
    for i, n in enumerate(lens):
        if i % 3:
            gone = sum(1 for p in range(pages_of(n, page)) if p * page >= case["sinks"] and (p + 1) * page <= n - case["window"])
            kept += pages_of(n, page) - gone
    # pages lie anywhere in the pool: of those in use, the share beyond the first `kept` places moves
    total = pages + pages // 4 + 8
    moved = kept * (1 - kept / total)
    return dict(bytes=moved * page * 2 * row * layers * 2 + 8 * (rows * width + total), flops=0)


def exact(case, seed):
    """In 64 bits from the definition, one sequence and one kv head at a time.  Moves of pages have no computed values."""
    kind = case["kind"]
    if kind in ("beam", "compact"):
        return None
    s = prepare(case, seed)
    page = case["page"]
    if kind == "append":
        new = _plain_append(s)
        k, v = s["k"].double(), s["v"].double()
        lens, news = lengths(case)
        at = 0
        for i, (n, c) in enumerate(zip(lens, news)):
            position = torch.arange(n - c, n, device="cuda")
            ids = new["table"][i].long()[position // page]
            k[0, ids, :, position % page] = s["k_new"][at:at + c].double()
            v[0, ids, :, position % page] = s["v_new"][at:at + c].double()
            at += c
        return dict(k=k, v=v, refs=None, table=None)
    lens, news = lengths(case)
    if kind == "decode":
        news = [1] * len(lens)
    hkv, hq, dim = case["kv_heads"], case["heads"], case["dim"]
    group = hq // hkv
    out = torch.zeros(sum(news), hq, dim, dtype=torch.float64, device="cuda")
    at = 0
    for i, (n, c) in enumerate(zip(lens, news)):
        ids = s["table"][i, :pages_of(n, page)].long()
        p = torch.arange(n - c, n, device="cuda")[:, None]
        columns = torch.arange(n, device="cuda")[None]
        hidden = columns > p
        if case["window"]:
            hidden = hidden | ((p - columns >= case["window"]) & (columns >= case["sinks"]))
        for h in range(hkv):
            k = s["k"][0, ids, h].reshape(-1, dim)[:n].double()
            v = s["v"][0, ids, h].reshape(-1, dim)[:n].double()
            for x in range(h * group, (h + 1) * group):
                t = (s["q"][at:at + c, x].double() @ k.T) * s["scale"]
                t.masked_fill_(hidden, float("-inf"))
                out[at:at + c, x] = torch.softmax(t, -1) @ v
        at += c
    return out
