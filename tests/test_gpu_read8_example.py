"""The example that retrieves and reads, with keys and values in 8 bits."""
import gc
import importlib.util
import os

import pytest
import torch

from paper_1712_02912_amd import binding

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location(
    "read_passages", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "read_passages.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


@pytest.fixture(autouse=True)
def collected():
    """Tensors that errors' frames hold do not outlive a test: later ones watch the memory that is allocated."""
    yield
    gc.collect()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_answers(dtype):
    """Every step's draw and the score of its token are one number, and answers repeat themselves."""
    ctx = binding.Context(0)
    decoder = example.Decoder(vocab=512, width=256, dtype=example.DTYPES[dtype])
    gen = torch.Generator(device="cuda").manual_seed(3)
    prompts = [torch.randint(512, (n,), device="cuda", generator=gen) for n in (37, 1, 90)]
    noise = torch.rand((6, 3, 512), device="cuda", generator=gen).clamp(1e-7, 1 - 1e-7)
    tokens, logprobs, logits = example.answer(ctx, decoder, prompts, 6, noise, cache8=True)
    assert tokens.shape == (3, 6) and all(bool(torch.isfinite(l).all()) for l in logits)
    for i, l in enumerate(logits):
        scored = ctx.pq_token_logprobs(l, tokens[:, i].contiguous())[0]
        assert bool(((scored - logprobs[:, i]).abs() <= 4e-6 * (1 + logprobs[:, i].abs())).all())
    again = example.answer(ctx, decoder, prompts, 6, noise, cache8=True)
    assert torch.equal(again[0], tokens) and all(torch.equal(a, b) for a, b in zip(again[2], logits))
    ctx.close()


def test_the_program_runs(capsys):
    tokens = example.main(["--questions", "3", "--passages", "2000", "--tokens", "4", "--cache8"])
    assert tokens.shape == (3, 4) and "likeliest" in capsys.readouterr().out
