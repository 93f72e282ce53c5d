"""Steps whose vocabulary is not a multiple of what a linear's rows are."""
import pytest
import torch

from paper_2502_11880_b200 import run_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [17, 1001, 1016])
def test_no_token_beyond_the_vocabulary(vocab):
    step = run_decode.Step(512, 8, 2, vocab)
    stream, q, _, _ = step.begin(torch.arange(3, device="cuda"))
    assert step.vocab == vocab and step.end(stream, q.contiguous()).shape == (3, vocab)
    _, tokens, status = run_decode.main(["--full", "--hidden", "512", "--heads", "8", "--kv-heads", "2", "--prompt", "20", "--steps", "40", "--samples", "16",
                                         "--vocab", str(vocab), "--temperature", "5", "--top-k", "0", "--top-p", "1", "--min-p", "0"])
    assert status == 0 and 0 <= int(tokens.min()) and int(tokens.max()) < vocab
