"""Whole decode steps of samples that share a prompt: norm, codes, linears, rotation into the pages, shared attention, drawn tokens."""
import pytest
import torch

import paper_2502_11880_b200 as bn
from paper_2502_11880_b200 import run_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("args", [
    ["--steps", "20", "--window", "0"],                                                                    # 8B-shaped layer
    ["--steps", "12", "--samples", "9", "--window", "100", "--prompt", "333"],
    ["--hidden", "3200", "--heads", "32", "--kv-heads", "32", "--prompt", "77", "--steps", "9", "--samples", "2", "--window", "40", "--page", "8", "--vocab", "1000"],
    ["--hidden", "1536", "--heads", "16", "--kv-heads", "16", "--prompt", "1", "--steps", "3", "--samples", "1", "--window", "2", "--sinks", "0"],
])
def test_samples_of_a_prompt(args):
    worst, tokens, status = run_decode.main(["--full", *args])
    # outputs and probabilities of 16 bits: 2^-8 of the result, and 2^-8 of sum p |v|, which is some eight times the result at a few hundred random values
    assert worst < 2 ** -4 and status == 0
    assert tokens.dtype == torch.int32 and int(tokens.min()) >= 0
    again = run_decode.main(["--full", *args])[1]
    assert torch.equal(tokens, again)


class Service:
    """Steps of n samples of one prompt over two layers' worth of pools, every buffer allocated once."""

    def __init__(self, n, prompt, steps, vocab=500, page=16):
        self.n, self.page = n, page
        self.step = run_decode.Step(512, 8, 2, vocab)
        ints = dict(dtype=torch.int32, device="cuda")
        width = -(-(prompt + steps) // page)
        full = prompt // page
        pages = full + n * (width - full) + 2
        self.cache = bn.new_kv_cache(1, pages, 2, page, 64)
        g = torch.Generator(device="cuda").manual_seed(1)
        for t in (self.cache.k, self.cache.v):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        self.table = torch.full((n, width), -1, **ints)
        own = width - full
        for i in range(n):
            self.table[i, :full] = torch.arange(full, **ints)
            self.table[i, full:] = full + i * own + torch.arange(own, **ints)
            if prompt % page:                    # the page filled in part: copies
                for t in (self.cache.k, self.cache.v):
                    t[0, full + i * own] = t[0, full]
        self.first = torch.full((n,), prompt, **ints)
        self.length, self.tokens = self.first.clone(), torch.zeros(n, **ints)
        self.start, self.prefix = torch.tensor([0, n], **ints), torch.tensor([prompt], **ints)
        self.ws, self.status = bn.new_attn_shared_workspace(n, 8, 2, 64), torch.zeros(1, **ints)
        self.u, self.top_p = torch.zeros(n, device="cuda"), torch.full((n,), 0.9, device="cuda")
        self.logits = torch.zeros(n, self.step.vocab, device="cuda")
        torch.cuda.synchronize()

    def run(self, wait=False):
        wait = torch.cuda.synchronize if wait else lambda: None
        self.length.add_(1)
        stream, q, k, v = self.step.begin(self.tokens)
        wait()
        q = bn.bitnet_kv_append_rope(self.cache, 0, self.step.rope, q, k, v, self.table, self.length, q_dtype=self.cache.dtype, dev_status=self.status)
        wait()
        attn = bn.bitnet_attn_shared(self.cache, 0, q, self.table, self.length, self.start, self.prefix, workspace=self.ws, dev_status=self.status)
        wait()
        self.logits.copy_(self.step.end(stream, attn))
        wait()
        bn.bitnet_sample(self.logits, self.u, top_p=self.top_p, tokens=self.tokens)
        wait()

    def reset(self):
        self.length.copy_(self.first)
        self.tokens.copy_(torch.arange(self.n, dtype=torch.int32, device="cuda"))

    def draw(self, i):
        self.u.copy_(torch.rand(self.n, generator=torch.Generator().manual_seed(i)))


@pytest.mark.parametrize("n,prompt", [(4, 333), (40, 64), (1, 5)])
def test_steps_back_to_back_and_in_a_graph(n, prompt):
    """Without a synchronisation between the kernels, and captured once and replayed: the tokens and logits of steps that wait after every call."""
    s = Service(n, prompt, 30)

    def steps(run):
        s.reset()
        out = []
        for i in range(25):
            s.draw(i)
            run()
            out += [s.tokens.clone(), s.logits.clone()]
        torch.cuda.synchronize()
        return out

    want = steps(lambda: s.run(wait=True))
    assert all(torch.equal(a, b) for a, b in zip(want, steps(s.run)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(want, steps(graph.replay)))
    assert int(s.status) == 0 and bn.bitnet_device_status() == 0


def test_two_services_on_two_streams():
    """Calls of two streams at once, each with a workspace of its own."""
    pair = [Service(6, 200, 30), Service(3, 100, 30)]
    want = []
    for s in pair:
        s.reset()
        for i in range(20):
            s.draw(i)
            s.run()
        torch.cuda.synchronize()
        want.append((s.tokens.clone(), s.logits.clone()))
    streams = [torch.cuda.Stream() for _ in pair]
    for s in pair:
        s.reset()
    torch.cuda.synchronize()
    for i in range(20):
        for s, stream in zip(pair, streams):
            with torch.cuda.stream(stream):
                s.draw(i)
                s.run()
    torch.cuda.synchronize()
    assert all(torch.equal(s.tokens, t) and torch.equal(s.logits, x) for s, (t, x) in zip(pair, want))


def test_steps_through_prefix_own_tokens_and_join():
    """The same with the shared attention in its own three kernels, small as the calls are."""
    bn.bitnet_debug_attn_shared(1)
    try:
        for n, prompt in ((4, 333), (40, 64), (150, 600)):
            test_steps_back_to_back_and_in_a_graph(n, prompt)
        test_two_services_on_two_streams()
    finally:
        bn.bitnet_debug_attn_shared(0)
