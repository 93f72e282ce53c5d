"""Measured cases of a decode step's operators around the ternary linears and the paged cache.

Four kinds of pass: "norm" (residual addition, root-mean-square norm, int8 codes for the next linear), "rope" (queries and keys rotated
by their positions, keys and values written into their pages), "shared" (attention of one token per sequence, groups of sequences sharing
a prefix) and "sample" (a token per row of logits by temperature, top-k, top-p and min-p from a given random number).

`own` selects the framework's entry points; otherwise the same results come from elementary torch operations.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one user's token before the Q/K/V linear of the 8B-shaped layer: all latency
        dict(name="norm_1x4096", kind="norm", tokens=1, width=4096, x="f32", residual="f32", weight="f32", y=""),
        # a batch before the down linear of the 100B-shaped layer: a norm inside the feed-forward part, no residual
        dict(name="norm_16x28672", kind="norm", tokens=16, width=28672, x="f32", residual="", weight="bf16", y=""),
        # a long prompt, 100B-shaped layer, 16-bit residual stream
        dict(name="norm_4099x8192", kind="norm", tokens=4099, width=8192, x="f32", residual="bf16", weight="bf16", y=""),
        # one decode step of 32 sequences far into their contexts, 100B-shaped layer, frequencies scaled by wavelength
        dict(name="rope_32x1", kind="rope", seqs=32, new=1, ctx=100003, ragged=1, heads=64, kv_heads=8, dim=128, rot=128, layout="half",
             scaling="bands", dtype="bf16", io="f32", out="f32", page=16),
        # three short prompts on top of what is cached, 3B-shaped layer (32 heads of 100), positions interpolated
        dict(name="rope_3x517", kind="rope", seqs=3, new=517, ctx=1201, ragged=2, heads=32, kv_heads=32, dim=100, rot=100, layout="interleaved",
             scaling="linear", dtype="f16", io="f16", out="f16", page=32),
        # prompts of a batch, 8B-shaped layer, half of the head rotated
        dict(name="rope_4x2048", kind="rope", seqs=4, new=2048, ctx=4099, ragged=3, heads=32, kv_heads=8, dim=128, rot=64, layout="half",
             scaling="none", dtype="bf16", io="f32", out="bf16", page=32),
        # eight samples of one answer, 8B-shaped layer
        dict(name="shared_8x2048", kind="shared", groups="8", prefix="2048", tail=60, ragged=4, heads=32, kv_heads=8, dim=128, dtype="bf16",
             page=16, window=0, sinks=0),
        # requests of three services with system prompts of their own, 1536-wide layer, window and sinks
        dict(name="shared_24_15_1", kind="shared", groups="24,15,1", prefix="4000,704,0", tail=300, ragged=5, heads=16, kv_heads=16, dim=96,
             dtype="f16", page=32, window=2048, sinks=4),
        # a full serving batch over one long document, 100B-shaped layer
        dict(name="shared_64x16384", kind="shared", groups="64", prefix="16384", tail=400, ragged=6, heads=64, kv_heads=8, dim=128, dtype="bf16",
             page=64, window=0, sinks=0),
        # one user's token, a vocabulary of 32000
        dict(name="sample_1x32000", kind="sample", rows=1, vocab=32000, dtype="f32", mix=0, top_k=50, top_p=0.9, min_p=0.0),
        # a serving batch, a vocabulary of 128256, every row with settings of its own
        dict(name="sample_64x128256", kind="sample", rows=64, vocab=128256, dtype="f32", mix=1, top_k=400, top_p=0.95, min_p=0.02),
        # a large batch of 16-bit logits, an odd vocabulary, top-p alone
        dict(name="sample_256x50021", kind="sample", rows=256, vocab=50021, dtype="bf16", mix=0, top_k=0, top_p=0.92, min_p=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# head layouts: the 8B-, 100B-, 3B- and 1536-wide shapes, and a generic one
LAYOUTS = [(32, 8, 128), (64, 8, 128), (32, 32, 100), (16, 16, 96), (12, 4, 64)]


def draw(rng):
    kind = rng.choice(["norm", "rope", "shared", "sample"])
    case = dict(kind=kind)
    if kind == "norm":
        width = rng.choice([1536, 3200, 4096, 8192, 8640, 14336, 28672, _log(rng, 64, 28672)])
        case.update(tokens=_log(rng, 1, min(8192, 4099 * 8192 // width)), width=width, x=rng.choice(["f32", "f32", "bf16", "f16"]),
                    residual=rng.choice(["", "f32", "bf16", "f16"]), weight=rng.choice(["", "f32", "bf16"]), y=rng.choice(["", "", "f32", "bf16"]))
    elif kind == "rope":
        heads, kv_heads, dim = rng.choice(LAYOUTS)
        seqs = _log(rng, 1, 64)
        new = rng.choice([1, _log(rng, 1, max(1, 8192 // seqs))])
        # tokens of all heads: at most the largest listed case's
        new = max(1, min(new, 4 * 2048 * 48 * 128 // (seqs * (heads + 2 * kv_heads) * dim)))
        dtype = rng.choice(["bf16", "f16"])
        case.update(seqs=seqs, new=new, ctx=new + rng.choice([0, _log(rng, 1, 131072)]), ragged=rng.randrange(1, 1 << 20), heads=heads,
                    kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim // 2, _log(rng, 4, dim) // 2 * 2]), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "bands"]), dtype=dtype, io=rng.choice(["f32", dtype]), out=rng.choice(["f32", dtype]),
                    page=rng.choice([8, 16, 32, 64, 128]))
    elif kind == "shared":
        heads, kv_heads, dim = rng.choice(LAYOUTS)
        counts = [_log(rng, 1, 64) for _ in range(rng.choice([1, 1, 2, 5]))]
        page = rng.choice([8, 16, 32, 64, 128])
        # what the plain form gathers: at most the largest listed case's
        most = max(256, 64 * 16784 * 8 * 128 // (sum(counts) * kv_heads * dim))
        prefix = [min(_log(rng, 1, 16384), most - 200) if not i or rng.random() < 0.75 else 0 for i in range(len(counts))]
        # a fork shares full pages; a length inside a page is one whose rest was copied
        prefix = [p // page * page if rng.random() < 0.8 else p for p in prefix]
        case.update(groups=",".join(map(str, counts)), prefix=",".join(map(str, prefix)), tail=_log(rng, 1, 600 if most > 2000 else 100),
                    ragged=rng.randrange(1, 1 << 20), heads=heads, kv_heads=kv_heads, dim=dim, dtype=rng.choice(["bf16", "f16"]), page=page)
        case["window"], case["sinks"] = rng.choice([(0, 0), (0, 0), (_log(rng, 16, 4096), rng.choice([0, 1, 4, 33]))])
    else:
        vocab = rng.choice([32000, 50021, 128256, _log(rng, 1000, 260000)])
        case.update(rows=_log(rng, 1, min(512, 64 * 128256 // vocab)), vocab=vocab, dtype=rng.choice(["f32", "f32", "bf16", "f16"]), mix=rng.choice([0, 1]),
                    top_k=rng.choice([0, _log(rng, 1, 1000)]), top_p=rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                    min_p=rng.choice([0.0, round(rng.uniform(0.001, 0.3), 4)]))
    return case


def _ints(text):
    return [int(x) for x in text.split(",")]


def lengths(case):
    """Given by the case alone.  rope: tokens per sequence after the pass, and new ones; shared: tokens per sequence."""
    r = random.Random(case["ragged"])
    if case["kind"] == "rope":
        n = case["seqs"]
        lens = [case["ctx"]] + [max(1, int(case["ctx"] * r.uniform(0.3, 1.0))) for _ in range(n - 1)]
        news = [case["new"]] + [max(1, int(case["new"] * r.uniform(0.5, 1.0))) for _ in range(n - 1)]
        return [max(a, b) for a, b in zip(lens, news)], news
    return [p + r.randint(1, case["tail"]) for c, p in zip(_ints(case["groups"]), _ints(case["prefix"])) for _ in range(c)]


def pages_of(tokens, page):
    return -(-tokens // page)


def rope_args(case):
    """Arguments of the rotation as a model's configuration has them."""
    a = dict(rot=case["rot"], base=500000.0 if case["scaling"] == "bands" else 10000.0, layout=case["layout"], scaling=case["scaling"])
    if case["scaling"] == "linear":
        a.update(factor=4.0)
    if case["scaling"] == "bands":
        a.update(factor=8.0, low=1.0, high=4.0, context=8192)
    return a


# ---------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    s.update({"norm": _prepare_norm, "rope": _prepare_rope, "shared": _prepare_shared, "sample": _prepare_sample}[case["kind"]](case, g))
    if own:
        import paper_2502_11880_b200 as bn
        s["bn"] = bn
        if case["kind"] in ("rope", "shared"):
            s["cache"] = bn.KvCache(s["k"], s["v"])
        if case["kind"] == "rope":
            s["rope"] = bn.Rope(**rope_args(case))
        if case["kind"] == "shared":
            s["ws"] = bn.new_attn_shared_workspace(s["q"].shape[0], case["heads"], case["kv_heads"], case["dim"])
    return s


def _prepare_norm(case, g):
    shape = case["tokens"], case["width"]
    # activations as a layer leaves them: most of unit size, a few channels far larger
    scale = 1 + 20 * (torch.rand(shape[1], generator=g, device="cuda") < 0.002)
    s = dict(x=(torch.randn(shape, generator=g, device="cuda") * scale).to(DTYPES[case["x"]]), residual=None, weight=None, eps=1e-5)
    if case["residual"]:
        s["residual"] = (3 * torch.randn(shape, generator=g, device="cuda") * scale).to(DTYPES[case["residual"]])
        s["residual_out"] = torch.empty_like(s["residual"])
    if case["weight"]:
        s["weight"] = (1 + 0.2 * torch.randn(shape[1], generator=g, device="cuda")).to(DTYPES[case["weight"]])
    s["y"] = torch.empty(shape, dtype=DTYPES[case["y"]], device="cuda") if case["y"] else None
    s["q"] = torch.empty(shape, dtype=torch.int8, device="cuda")
    s["act_scale"] = torch.empty(shape[0], dtype=torch.float32, device="cuda")
    s["values"] = torch.empty(shape, dtype=torch.bfloat16, device="cuda")            # what the codes stand for
    return s


def _prepare_rope(case, g):
    lens, news = lengths(case)
    page, hkv, dim = case["page"], case["kv_heads"], case["dim"]
    # only the pages that new tokens go to are looked at: the pool holds those (earlier ones are in use elsewhere, or were released)
    first = [(a - b) // page for a, b in zip(lens, news)]
    count = [pages_of(a, page) - f for a, f in zip(lens, first)]
    pages = sum(count) + 8
    shape = (1, pages, hkv, page, -(-dim // 8) * 8)
    s = {n: torch.zeros(shape, device="cuda", dtype=DTYPES[case["dtype"]])[..., :dim] for n in "kv"}
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((len(lens), pages_of(max(lens), page)), -1, dtype=torch.int32)
    at = 0
    for i, (f, c) in enumerate(zip(first, count)):
        table[i, f:f + c] = order[at:at + c]
        at += c
    # the fused output of the Q/K/V linear: q, k and v are slices of its rows
    tokens, cut = sum(news), (case["heads"] * dim, (case["heads"] + hkv) * dim)
    qkv = torch.randn(tokens, cut[1] + hkv * dim, generator=g, device="cuda").to(DTYPES[case["io"]])
    s.update(table=table.cuda(), len=torch.tensor(lens, dtype=torch.int32, device="cuda"), q=qkv[:, :cut[0]].view(tokens, -1, dim),
             k_new=qkv[:, cut[0]:cut[1]].view(tokens, -1, dim), v_new=qkv[:, cut[1]:].view(tokens, -1, dim),
             q_out=torch.empty(tokens, case["heads"], dim, dtype=DTYPES[case["out"]], device="cuda"),
             q_start=torch.tensor([0] + [sum(news[:i + 1]) for i in range(len(news))], dtype=torch.int32, device="cuda"))
    return s


def _prepare_shared(case, g):
    counts, prefix, lens = _ints(case["groups"]), _ints(case["prefix"]), lengths(case)
    page, hkv, dim, hq = case["page"], case["kv_heads"], case["dim"], case["heads"]
    # as a fork leaves them: full pages of the prefix shared, the page filled in part copied, then tokens of their own
    rows, at = [], 0
    for i, (c, p) in enumerate(zip(counts, prefix)):
        full = p // page
        shared = list(range(at, at + full))
        at += full
        for n in lens[len(rows):len(rows) + c]:
            more = pages_of(n, page) - full
            rows.append(shared + list(range(at, at + more)))
            at += more
    pages = at + 8
    shape = (1, pages, hkv, page, -(-dim // 8) * 8)
    s = {n: torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[case["dtype"]])[..., :dim] for n in "kv"}
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((len(rows), max(map(len, rows))), -1, dtype=torch.int32)
    for i, r in enumerate(rows):
        table[i, :len(r)] = order[r]
    start = [sum(counts[:i]) for i in range(len(counts) + 1)]
    for i, p in enumerate(prefix):
        if p % page:                                  # copies of the page filled in part
            part = table[start[i]:start[i + 1], p // page].long().cuda()
            for n in "kv":
                s[n][0, part, :, :p % page] = s[n][0, part[0], :, :p % page].clone()
    # the first tokens draw attention, as they do in trained models
    pull = 0.7 * torch.randn(hkv, dim, generator=g, device="cuda")
    s["k"][0, table[:, 0].unique().long().cuda(), :, :4] += pull.to(s["k"].dtype)[None, :, None]
    q = torch.randn(len(rows), hq, dim, generator=g, device="cuda") + pull.repeat_interleave(hq // hkv, 0)[None]
    s.update(q=q.to(DTYPES[case["dtype"]]), table=table.cuda(), len=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             group_start=torch.tensor(start, dtype=torch.int32, device="cuda"),
             prefix_len=torch.tensor(prefix, dtype=torch.int32, device="cuda"), scale=1.0 / math.sqrt(dim))
    return s


def _prepare_sample(case, g):
    rows, vocab = case["rows"], case["vocab"]
    # a few tokens stand out of a broad rest, more or less so from row to row
    x = torch.randn(rows, vocab, generator=g, device="cuda") * (1.5 + 1.5 * torch.rand(rows, 1, generator=g, device="cuda"))
    x[:, torch.randint(0, vocab, (20,), generator=g, device="cuda")] += 6 * torch.rand(rows, 20, generator=g, device="cuda")
    s = dict(logits=x.to(DTYPES[case["dtype"]]), u=torch.rand(rows, generator=g, device="cuda"),
             temperature=0.5 + torch.rand(rows, generator=g, device="cuda"))

    def setting(value, off, spread):
        t = torch.full((rows,), value, device="cuda") if not case["mix"] else value * spread(torch.rand(rows, generator=g, device="cuda"))
        return torch.where(torch.rand(rows, generator=g, device="cuda") < 0.2, torch.full_like(t, off), t) if case["mix"] else t

    s["top_k"] = setting(float(case["top_k"]), 0.0, lambda r: 0.01 + r).ceil().to(torch.int32) if case["top_k"] else None
    s["top_p"] = setting(case["top_p"], 1.0, lambda r: 0.5 + 0.5 * r) if case["top_p"] < 1 else None
    s["min_p"] = setting(case["min_p"], 0.0, lambda r: 0.5 + r) if case["min_p"] > 0 else None
    if case["mix"]:
        s["temperature"][::7] = 0.0               # rows that take the largest logit
    s["tokens"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    s["prob"] = torch.empty(rows, dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- passes
def run(s):
    return (OWN if own else PLAIN)[s["case"]["kind"]](s)


def _own_norm(s):
    s["bn"].bitnet_add_rmsnorm_quant(s["x"], s["weight"], s["eps"], residual=s["residual"], residual_out=s.get("residual_out"), y=s["y"], q=s["q"],
                                     act_scale=s["act_scale"])
    return dict(values=torch.mul(s["q"], s["act_scale"][:, None], out=s["values"]), scale=s["act_scale"], h=s.get("residual_out"), y=s["y"])


def _own_rope(s):
    s["bn"].bitnet_kv_append_rope(s["cache"], 0, s["rope"], s["q"], s["k_new"], s["v_new"], s["table"], s["len"], s["q_start"], q_out=s["q_out"])
    return dict(q=s["q_out"], k=s["k"], v=s["v"])


def _own_shared(s):
    return s["bn"].bitnet_attn_shared(s["cache"], 0, s["q"], s["table"], s["len"], s["group_start"], s["prefix_len"], scale=s["scale"],
                                      window=s["case"]["window"], sinks=s["case"]["sinks"], workspace=s["ws"])


def _own_sample(s):
    s["bn"].bitnet_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                          tokens=s["tokens"], prob=s["prob"])
    return dict(tokens=s["tokens"], prob=s["prob"])


OWN = dict(norm=_own_norm, rope=_own_rope, shared=_own_shared, sample=_own_sample)


def _plain_norm(s):
    """The sum of the squares in 64 bits, one rounding of 1 / root; from there binary32 steps, as the int8 quantiser's: next to a border
    of two codes other roundings would give other codes."""
    h = s["x"].float()
    if s["residual"] is not None:
        s["residual_out"].copy_(s["residual"].float() + h)
        h = s["residual_out"].float()
    r = (1 / torch.sqrt(h.double().square().mean(-1, keepdim=True) + s["eps"])).float()
    y = h * r
    if s["weight"] is not None:
        y = y * s["weight"].float()
    top = y.abs().amax(-1, keepdim=True).clamp(min=1e-5)
    codes = torch.round(y * (torch.full_like(top, 127.0) / top)).clamp(-128, 127)
    scale = top / torch.full_like(top, 127.0)
    return dict(values=(codes * scale).bfloat16(), scale=scale[:, 0], h=s.get("residual_out"), y=y.to(s["y"].dtype) if s["y"] is not None else None)


def _frequencies(case):
    """Radians per position of each rotated pair, in 64 bits."""
    a = rope_args(case)
    f = a["base"] ** (-torch.arange(0, a["rot"], 2, device="cuda", dtype=torch.float64) / a["rot"])
    if a["scaling"] == "linear":
        f = f / a["factor"]
    if a["scaling"] == "bands":
        # turns within the original context: many, kept; few, divided; in between, blended
        blend = ((f * a["context"] / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])).clamp(0, 1)
        f = (1 - blend) * f / a["factor"] + blend * f
    return f


def _where(s):
    """Sequence and position of every new token."""
    token = torch.arange(s["k_new"].shape[0], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].contiguous(), token.to(torch.int32), right=True)
    return seq, s["len"][seq] - s["q_start"][seq + 1] + token


def _rotate(x, position, case, exact=False):
    angle = position.double()[:, None] * _frequencies(case)                         # far positions: 64 bits
    cos, sin = ((t if exact else t.float())[:, None] for t in (torch.cos(angle), torch.sin(angle)))
    rot = case["rot"]
    x = (x.double() if exact else x.float()).clone()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    p, q = x[..., a].clone(), x[..., b].clone()
    x[..., a] = p * cos - q * sin
    x[..., b] = q * cos + p * sin
    return x


def _plain_rope(s):
    case, page = s["case"], s["case"]["page"]
    seq, position = _where(s)
    at = s["table"][seq, position // page].long()
    s["k"][0][at, :, position % page] = _rotate(s["k_new"], position, case).to(s["k"].dtype)
    s["v"][0][at, :, position % page] = s["v_new"].to(s["v"].dtype)
    s["q_out"].copy_(_rotate(s["q"], position, case))
    return dict(q=s["q_out"], k=s["k"], v=s["v"])


def _plain_shared(s):
    case = s["case"]
    ids = s["table"].clamp(min=0).long()
    k, v = (s[n][0][ids].float().permute(0, 2, 1, 3, 4).flatten(2, 3) for n in "kv")  # sequences, kv heads, tokens, dim
    n, hkv, tokens, dim = k.shape
    column, length = torch.arange(tokens, device="cuda"), s["len"].view(n, 1, 1, 1)
    see = column < length
    if case["window"]:
        see = see & ((column >= length - case["window"]) | (column < case["sinks"]))
    v = v * (column[:, None] < length)
    scores = (s["q"].float().view(n, hkv, -1, dim) * s["scale"]) @ k.transpose(-1, -2)
    scores = scores.masked_fill(~see, float("-inf"))
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    return ((p @ v) / p.sum(-1, keepdim=True)).reshape(s["q"].shape).to(s["q"].dtype)


def _plain_sample(s):
    """In 64 bits: long sums, and what is kept is decided next to borders."""
    x = s["logits"].double()
    rows, vocab = x.shape
    z, index = torch.sort(x, dim=-1, descending=True, stable=True)                   # ties: lowest index first
    greedy = s["temperature"] <= 0
    t = torch.where(greedy, torch.ones_like(s["temperature"]), s["temperature"]).double()[:, None]
    w = torch.exp((z - z[:, :1]) / t)
    rank = torch.arange(vocab, device="cuda")
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"], vocab)[:, None]
        w = w * (rank < k)
    if s["top_p"] is not None:
        p = torch.where(s["top_p"] < 1, s["top_p"].double(), 2.0)[:, None]
        c = torch.cumsum(w, -1)
        w = w * ((c - w < p * c[:, -1:]) | (rank == 0))
    if s["min_p"] is not None:
        w = w * (w >= s["min_p"].double()[:, None])
    w = w * ((rank == 0) | ~greedy[:, None])
    w = torch.zeros_like(w).scatter_(1, index, w)                                    # in the order of the vocabulary
    c = torch.cumsum(w, -1)
    total = c[:, -1:]
    token = torch.searchsorted(c, s["u"].double()[:, None] * total, right=True).clamp(max=vocab - 1)
    return dict(tokens=token[:, 0].to(torch.int32), prob=(w.gather(1, token) / total)[:, 0].float())


PLAIN = dict(norm=_plain_norm, rope=_plain_rope, shared=_plain_shared, sample=_plain_sample)


# ---------------------------------------------------------------------------------------------- work and exact values
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "": 0}


def _seen(length, window, sinks):
    """How many of a sequence's tokens its last one sees, and which: [0, first) and [second, length)."""
    second = max(0, length - window) if window else 0
    return min(sinks, second), second


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n = case["tokens"] * case["width"]
        return dict(bytes=n * (SIZE[case["x"]] + 2 * SIZE[case["residual"]] + SIZE[case["y"]] + 1) + case["width"] * SIZE[case["weight"]] + 4 * case["tokens"],
                    flops=6 * n)
    if kind == "rope":
        tokens, io, out = sum(lengths(case)[1]), SIZE[case["io"]], SIZE[case["out"]]
        return dict(bytes=tokens * case["dim"] * (case["heads"] * (io + out) + 2 * case["kv_heads"] * (io + 2)),
                    flops=3 * tokens * case["rot"] * (case["heads"] + case["kv_heads"]))
    if kind == "sample":
        return dict(bytes=case["rows"] * (case["vocab"] * SIZE[case["dtype"]] + 28), flops=3 * case["rows"] * case["vocab"])
    lens, at, tokens, pairs = lengths(case), 0, 0, 0
    for c, p in zip(_ints(case["groups"]), _ints(case["prefix"])):
        spans = [_seen(n, case["window"], case["sinks"]) for n in lens[at:at + c]]
        pairs += sum(a + n - b for (a, b), n in zip(spans, lens[at:at + c]))
        # the prefix once, as far as any of the group sees it, and each one's own tokens
        a, b = max(x[0] for x in spans), min(x[1] for x in spans)
        tokens += p if a >= b else min(a, p) + max(0, p - b)
        tokens += sum(max(0, x - p) + n - max(y, p) for (x, y), n in zip(spans, lens[at:at + c]))
        at += c
    return dict(bytes=4 * tokens * case["kv_heads"] * case["dim"] + 4 * len(lens) * case["heads"] * case["dim"], flops=4 * pairs * case["heads"] * case["dim"])


def exact(case, seed):
    """In 64 bits from the definitions, attention one sequence and one kv head at a time."""
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rope": _exact_rope, "shared": _exact_shared, "sample": _exact_sample}[case["kind"]](s)


def _exact_norm(s):
    h = s["x"].double()
    stream = None
    if s["residual"] is not None:
        stream = h + s["residual"].double()
        h = stream.float().to(s["residual"].dtype).double()                          # the norm is of the stream as it is kept
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + s["eps"])
    if s["weight"] is not None:
        y = y * s["weight"].double()
    scale = y.abs().amax(-1, keepdim=True).clamp(min=1e-5) / 127
    return dict(values=torch.round(y / scale) * scale, scale=scale[:, 0], h=stream, y=y if s["y"] is not None else None)


def _exact_rope(s):
    case, page = s["case"], s["case"]["page"]
    k, v, lens = s["k"].double(), s["v"].double(), s["len"].tolist()
    start, q = s["q_start"].tolist(), []
    for i, n in enumerate(lens):
        part = slice(start[i], start[i + 1])
        position = torch.arange(n - (start[i + 1] - start[i]), n, device="cuda")
        ids = s["table"][i].long()[position // page]
        k[0, ids, :, position % page] = _rotate(s["k_new"][part], position, case, exact=True)
        v[0, ids, :, position % page] = s["v_new"][part].double()
        q.append(_rotate(s["q"][part], position, case, exact=True))
    return dict(q=torch.cat(q), k=k, v=v)


def _exact_shared(s):
    case, lens = s["case"], s["len"].tolist()
    hkv, hq, dim, page = case["kv_heads"], case["heads"], case["dim"], case["page"]
    out = torch.zeros(len(lens), hkv, hq // hkv, dim, dtype=torch.float64, device="cuda")
    q = s["q"].double().view(out.shape)
    for i, n in enumerate(lens):
        first, second = _seen(n, case["window"], case["sinks"])
        c = torch.cat([torch.arange(first, device="cuda"), torch.arange(second, n, device="cuda")])
        ids = s["table"][i].long()[c // page]
        for h in range(hkv):
            k, v = (s[x][0, ids, h, c % page].double() for x in "kv")
            out[i, h] = torch.softmax(q[i, h] @ k.T * s["scale"], -1) @ v
    return out.view(s["q"].shape)


def _exact_sample(s):
    """The probability of the drawn token; a row at a time."""
    prob = torch.empty(s["u"].shape[0], dtype=torch.float64, device="cuda")
    for i, x in enumerate(s["logits"].double()):
        t = float(s["temperature"][i])
        if t <= 0:
            prob[i] = 1.0
            continue
        p = torch.softmax(x / t, 0)
        order = torch.sort(x, descending=True, stable=True).indices
        k = int(s["top_k"][i]) if s["top_k"] is not None else 0
        order = order[:k] if k > 0 else order
        q = p[order] / p[order].sum()
        if s["top_p"] is not None and float(s["top_p"][i]) < 1:
            before = torch.cumsum(q, 0) - q
            order = order[:max(1, int((before < float(s["top_p"][i])).sum()))]
        kept = torch.zeros_like(p)
        kept[order] = p[order]
        if s["min_p"] is not None:
            kept[p < float(s["min_p"][i]) * p.max()] = 0
        c = torch.cumsum(kept, 0)
        prob[i] = kept[min(int((c <= float(s["u"][i]) * c[-1]).sum()), kept.numel() - 1)] / c[-1]
    return dict(tokens=None, prob=prob)
