"""One decoder layer's attention half as it is used: ternary Q/K/V and O linears with the paged cache and the attention between them
(an example of the Python binding; prints what it did and how far its attention is from a plain one in 64 bits).

    python -m paper_2502_11880_b200.run_decode [--hidden 4096] [--heads 32] [--kv-heads 8] [--prompt 300] [--steps 40]
                                               [--samples 3] [--window 128] [--sinks 4]

A prompt goes through the Q/K/V linear, its K and V rows into pages, its attention and the O linear.  The sequence is forked into
samples that share its full pages.  Every step then takes one token of each sample through the layer: reserve, append, attention
with a sliding window and sinks.  At the end pages that left the window are given up, the rest packed, and the next token's attention is
the same as before.

    python -m paper_2502_11880_b200.run_decode --full [--vocab 32000] [--temperature 0.8] [--top-k 50] [--top-p 0.95] [--min-p 0.02] ...

runs the samples as whole steps: embedding, norm and int8 codes, Q/K/V linear, rotation on the way into the pages, attention that reads the prompt once
for all samples, O linear, residual addition and norm, head linear, and a token drawn for each sample.
"""
import argparse

import torch

import paper_2502_11880_b200 as bn
from paper_2502_11880_b200 import synth


class Layer:
    """I2_S Q/K/V and O linears with seeded ternary weights."""

    def __init__(self, hidden, heads, kv_heads, seed=0):
        self.hidden, self.heads, self.kv_heads, self.dim = hidden, heads, kv_heads, hidden // heads
        self.rows = [(heads + 2 * kv_heads) * self.dim, hidden]
        cols = [hidden, heads * self.dim]
        w = [synth.ternary(seed, i, m, k, 1 / 3, 1 / 3, device="cuda") for i, (m, k) in enumerate(zip(self.rows, cols))]
        self.blobs = [bn.pack("i2s", x) for x in w]
        # scales that keep activations of unit size
        self.scales = [(k * 2 / 3) ** -0.5 for k in cols]

    def linear(self, i, x):
        return bn.bitnet_linear("i2s", self.blobs[i], self.scales[i], self.rows[i], x.shape[1], x)[0]

    def qkv(self, x):
        """Views of the fused fp32 output: q [T][heads][dim], k and v [T][kv_heads][dim]."""
        y, d = self.linear(0, x), self.dim
        cut = self.heads * d, (self.heads + self.kv_heads) * d
        return y[:, :cut[0]].view(-1, self.heads, d), y[:, cut[0]:cut[1]].view(-1, self.kv_heads, d), y[:, cut[1]:].view(-1, self.kv_heads, d)


class Step(Layer):
    """A layer with what surrounds its linears: embedding, norms, rotation, head."""

    def __init__(self, hidden, heads, kv_heads, vocab, seed=0):
        super().__init__(hidden, heads, kv_heads, seed)
        self.vocab, self.head_rows = vocab, -(-vocab // 16) * 16                     # (a linear has a multiple of 16 rows)
        self.embedding = synth.normal(seed, 100, self.vocab, hidden).cuda()
        self.norms = [1 + 0.1 * synth.normal(seed, 101 + i, 1, hidden)[0].cuda() for i in range(2)]
        self.rope = bn.Rope(self.dim, base=500000.0, scaling="bands", factor=8.0, context=8192)
        self.head = bn.pack("i2s", synth.ternary(seed, 2, self.head_rows, hidden, 1 / 3, 1 / 3, device="cuda"))
        self.head_scale = 2.0 * (hidden * 2 / 3) ** -0.5

    def _linear(self, blob, scale, rows, codes, act_scale):
        return bn.bitnet_mpgemm("i2s", blob, scale, rows, codes.shape[1], codes, act_scale)[0]

    def begin(self, tokens):
        """The residual stream, and views of q, k and v."""
        stream = self.embedding[tokens.long()]
        y, d = self._linear(self.blobs[0], self.scales[0], self.rows[0], *bn.bitnet_add_rmsnorm_quant(stream, self.norms[0])), self.dim
        cut = self.heads * d, (self.heads + self.kv_heads) * d
        return stream, y[:, :cut[0]].view(-1, self.heads, d), y[:, cut[0]:cut[1]].view(-1, self.kv_heads, d), y[:, cut[1]:].view(-1, self.kv_heads, d)

    def end(self, stream, attn):
        """Logits; the stream is updated in place."""
        o = self.linear(1, attn.float().reshape(attn.shape[0], -1))
        return self._linear(self.head, self.head_scale, self.head_rows, *bn.bitnet_add_rmsnorm_quant(o, self.norms[1], residual=stream))[:, :self.vocab]


def full(a):
    """Samples of one prompt as whole steps; returns how far attention is off, the tokens [steps][samples], the status word."""
    step = Step(a.hidden, a.heads, a.kv_heads, a.vocab)
    n, page = a.samples, a.page
    width = -(-(a.prompt + a.steps) // page)
    pages = (n + 1) * width
    cache = bn.new_kv_cache(1, pages, a.kv_heads, page, step.dim)
    ints = dict(dtype=torch.int32, device="cuda")
    refs, table, length = torch.zeros(pages, **ints), torch.full((1 + n, width), -1, **ints), torch.zeros(1 + n, **ints)
    status = torch.zeros(1, **ints)
    ws = bn.new_attn_workspace(a.prompt, a.heads, a.kv_heads, step.dim)
    u = torch.rand(a.steps, n, generator=torch.Generator().manual_seed(7)).cuda()
    settings = dict(temperature=torch.full((n,), a.temperature, device="cuda"), top_k=torch.full((n,), a.top_k, **ints),
                    top_p=torch.full((n,), a.top_p, device="cuda"), min_p=torch.full((n,), a.min_p, device="cuda"))

    # ---- the prompt: sequence 0
    start, to = torch.tensor([0, a.prompt], **ints), length.clone()
    to[0] = a.prompt
    stream, q, k, v = step.begin(torch.randint(0, step.vocab, (a.prompt,), generator=torch.Generator().manual_seed(8)).cuda())
    bn.bitnet_kv_reserve(refs, table, length, to, page, dev_status=status)
    length.copy_(to)
    q = bn.bitnet_kv_append_rope(cache, 0, step.rope, q, k, v, table[:1], length[:1], start, q_dtype=cache.dtype, dev_status=status)
    attn = bn.bitnet_attn_prompt(cache, 0, q, table[:1], length[:1], start, a.prompt, window=a.window, sinks=a.sinks, workspace=ws, dev_status=status)
    logits = step.end(stream, attn)[-1:]
    tokens = [bn.bitnet_sample(logits.expand(n, -1), u[0], **settings)[0]]

    # ---- samples 1..n share the prompt's full pages; its own row stays
    rows = torch.arange(1, 1 + n, **ints)
    bn.bitnet_kv_fork(cache, refs, table, length, torch.zeros(n, **ints), rows, dev_status=status)
    table, length = table[1:].contiguous(), length[1:].contiguous()
    group_start, prefix = torch.tensor([0, n], **ints), torch.tensor([a.prompt], **ints)
    ws = bn.new_attn_shared_workspace(n, a.heads, a.kv_heads, step.dim)
    worst = 0.0
    for i in range(1, a.steps):
        stream, q, k, v = step.begin(tokens[-1])
        to = length + 1
        bn.bitnet_kv_reserve(refs, table, length, to, page, dev_status=status)
        length.copy_(to)
        q = bn.bitnet_kv_append_rope(cache, 0, step.rope, q, k, v, table, length, q_dtype=cache.dtype, dev_status=status)
        attn = bn.bitnet_attn_shared(cache, 0, q, table, length, group_start, prefix, window=a.window, sinks=a.sinks, workspace=ws, dev_status=status)
        if i in (1, a.steps - 1):
            ref = plain(cache, q, table, length, a.window, a.sinks)
            worst = max(worst, float((attn.double() - ref).norm() / ref.norm()))
        tokens.append(bn.bitnet_sample(step.end(stream, attn), u[i], **settings)[0])
    tokens = torch.stack(tokens)
    torch.cuda.synchronize()
    print(f"{a.prompt} prompt tokens, {n} samples x {a.steps} tokens of {step.vocab}: {tokens[:, 0].tolist()[:8]} ...; attention off by {worst:.1e}; "
          f"status {int(status)}, {bn.bitnet_device_status()}")
    return worst, tokens, int(status)


def plain(cache, q, table, length, window, sinks):
    """Attention of one token per row of the table in 64 bits."""
    out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    for s in range(q.shape[0]):
        n = int(length[s])
        c = torch.arange(n, device=q.device)
        c = c[(c >= n - window) | (c < sinks)] if window else c
        ids = table[s].long()[c // cache.page_size]
        k, v = (p[0][ids, :, c % cache.page_size].double() for p in (cache.k, cache.v))            # tokens, heads, dim
        g = q.shape[1] // cache.kv_heads
        score = torch.einsum("hgd,chd->hgc", q[s].double().view(cache.kv_heads, g, -1), k) * cache.scale
        out[s] = torch.einsum("hgc,chd->hgd", torch.softmax(score, -1), v).reshape(q.shape[1], -1)
    return out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in dict(hidden=4096, heads=32, kv_heads=8, prompt=300, steps=40, samples=3, window=128, sinks=4, page=16).items():
        ap.add_argument("--" + name.replace("_", "-"), type=int, default=value)
    ap.add_argument("--full", action="store_true")
    for name, value in {"vocab": 32000, "temperature": 0.8, "top_k": 50, "top_p": 0.95, "min_p": 0.02}.items():
        ap.add_argument("--" + name.replace("_", "-"), type=type(value), default=value)
    a = ap.parse_args(argv)
    if a.full:
        return full(a)
    layer = Layer(a.hidden, a.heads, a.kv_heads)
    dim, page = layer.dim, a.page
    width = -(-(a.prompt + a.steps + 1) // page)
    pages = (a.samples + 1) * width
    cache = bn.new_kv_cache(1, pages, a.kv_heads, page, dim)
    ints = dict(dtype=torch.int32, device="cuda")
    refs, table, length = torch.zeros(pages, **ints), torch.full((1 + a.samples, width), -1, **ints), torch.zeros(1 + a.samples, **ints)
    status = torch.zeros(1, **ints)
    ws, books = bn.new_attn_workspace(a.prompt, a.heads, a.kv_heads, dim), bn.new_kv_workspace(pages, a.samples)

    # ---- the prompt: sequence 0
    q, k, v = layer.qkv(synth.normal(1, 0, a.prompt, a.hidden).cuda())
    start, to = torch.tensor([0, a.prompt], **ints), length.clone()
    to[0] = a.prompt
    bn.bitnet_kv_reserve(refs, table, length, to, page, dev_status=status)
    length.copy_(to)
    bn.bitnet_kv_append(cache, 0, k, v, table[:1], length[:1], start, dev_status=status)
    attn = bn.bitnet_attn_prompt(cache, 0, q.to(cache.dtype), table[:1], length[:1], start, a.prompt, window=a.window, sinks=a.sinks,
                                 workspace=ws, dev_status=status)
    x = layer.linear(1, attn.float().view(a.prompt, -1))[-1:]

    # ---- samples 1..: they share the prompt's full pages; the prompt's own row is given up
    rows = torch.arange(1, 1 + a.samples, **ints)
    bn.bitnet_kv_fork(cache, refs, table, length, torch.zeros(a.samples, **ints), rows, workspace=books, dev_status=status)
    bn.bitnet_kv_free(refs, table, length, torch.zeros(1, **ints), dev_status=status)
    used = int((refs > 0).sum())
    table, length = table[1:].contiguous(), length[1:].contiguous()
    x = x + 0.1 * synth.normal(1, 1, a.samples, a.hidden).cuda()

    # ---- one token of each sample at a time
    worst = 0.0
    for step in range(a.steps):
        q, k, v = layer.qkv(x)
        to = length + 1
        bn.bitnet_kv_reserve(refs, table, length, to, page, dev_status=status)
        length.copy_(to)
        bn.bitnet_kv_append(cache, 0, k, v, table, length, dev_status=status)
        attn = bn.bitnet_attn_decode(cache, 0, q, table, length, window=a.window, sinks=a.sinks, workspace=ws, dev_status=status)
        if step in (0, a.steps - 1):
            ref = plain(cache, q, table, length, a.window, a.sinks)
            worst = max(worst, float((attn.double() - ref).norm() / ref.norm()))
        x = layer.linear(1, attn.view(a.samples, -1)) + 0.1 * synth.normal(1, 2 + step, a.samples, a.hidden).cuda()

    # ---- pages outside the window go, the rest moves together; attention does not change
    before = bn.bitnet_attn_decode(cache, 0, q, table, length, window=a.window, sinks=a.sinks, workspace=ws)
    bn.bitnet_kv_trim(refs, table, length, page, a.window, a.sinks)
    live = torch.zeros(1, **ints)
    bn.bitnet_kv_compact(cache, refs, table, live=live, workspace=books)
    after = bn.bitnet_attn_decode(cache, 0, q, table, length, window=a.window, sinks=a.sinks, workspace=ws, dev_status=status)
    same = torch.equal(before, after)
    torch.cuda.synchronize()
    print(f"{a.prompt} prompt tokens, {a.samples} samples x {a.steps} tokens; pages in use after the fork {used}, at the end {int(live)} of {pages}; "
          f"attention off by {worst:.1e}; the same after trimming and packing: {same}; status {int(status)}, {bn.bitnet_device_status()}")
    return worst, same, int(status)


if __name__ == "__main__":
    main()
