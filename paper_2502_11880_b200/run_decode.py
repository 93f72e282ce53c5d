"""One decoder layer's attention half as it is used: ternary Q/K/V and O linears with the paged cache and the attention between them
(an example of the Python binding; prints what it did and how far its attention is from a plain one in 64 bits).

    python -m paper_2502_11880_b200.run_decode [--hidden 4096] [--heads 32] [--kv-heads 8] [--prompt 300] [--steps 40]
                                               [--samples 3] [--window 128] [--sinks 4]

A prompt goes through the Q/K/V linear, its K and V rows into pages, its attention and the O linear.  The sequence is forked into
samples that share its full pages.  Every step then takes one token of each sample through the layer: reserve, append, attention
with a sliding window and sinks.  At the end pages that left the window are given up, the rest packed, and the next token's attention is
the same as before.
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


def plain(cache, q, table, length, window, sinks):
    """Attention of one token per row of the table in 64 bits."""
    out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    for s in range(q.shape[0]):
        n = int(length[s])
        c = torch.arange(n, device=q.device)
        c = c[(c >= n - window) | (c < sinks)]
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
    a = ap.parse_args(argv)
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
