"""The example that retrieves and reads, against a decoder that computes every token anew from the whole sequence."""
import gc
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import read_oracle as orc
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


def norm(x):
    return x / (x.square().mean(dim=-1, keepdim=True) + 1e-6).sqrt()


def logits_of(d, tokens):
    """Logits of the last of the tokens, in 64 bits on the CPU, without a cache."""
    t, group = len(tokens), d.q_heads // d.heads
    x = d.embedding.cpu().double()[tokens]
    cos, sin = (a.cpu().double()[:t, None] for a in (d.cos, d.sin))

    def turn(y, weight):
        y = norm(y) * weight.cpu().double()
        a, b = y.chunk(2, dim=2)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=2)

    for w in d.layers:
        q, k, v = (norm(x) @ w["qkv"].cpu().double()).view(t, -1, d.dim).split((d.q_heads, d.heads, d.heads), dim=1)
        q, k = turn(q, w["q_norm"]), turn(k, w["k_norm"])
        k, v = (y.repeat_interleave(group, dim=1) for y in (k, v))
        scores = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) * d.dim ** -0.5
        scores = scores.masked_fill(torch.ones(t, t).triu(1).bool(), -np.inf)
        out = torch.matmul(scores.softmax(dim=2), v.transpose(0, 1)).transpose(0, 1).reshape(t, -1)
        x = x + out @ w["out"].cpu().double()
        y = norm(x) @ w["up"].cpu().double()
        x = x + (y * y.sigmoid()) @ w["down"].cpu().double()
    return norm(x[-1:]) @ d.head.cpu().double()


# Logits are of size 1 (normalised rows by weights of size width^-1/2).  Behind each are two layers of about ten roundings to the
# type and fp32 sums of up to 1024 products; relative errors of u each add up to 20 u at most in the mean square, and the largest of
# 4 x 6 x 512 logits lies within 5 times that.
@pytest.mark.parametrize("dtype,bound", [("f32", 100 * 2.0 ** -22), ("f16", 100 * 2.0 ** -11), ("bf16", 100 * 2.0 ** -8)])
def test_answers(dtype, bound):
    ctx = binding.Context(0)
    d = example.Decoder(vocab=512, width=256, layers=2, q_heads=8, heads=2, dim=64, positions=512, dtype=example.DTYPES[dtype])
    gen = torch.Generator(device="cuda").manual_seed(3)
    prompts = [torch.randint(d.vocab, (n,), device="cuda", generator=gen) for n in (1, 16, 31, 200)]
    steps = 6
    noise = torch.rand((steps, 4, d.vocab), device="cuda", generator=gen)
    temperature, top_k = torch.full((4,), 0.7, device="cuda"), torch.tensor([0, 40, 3, 200], dtype=torch.int32, device="cuda")
    tokens, logprobs, logits = example.answer(ctx, d, prompts, steps, noise, temperature=temperature, top_k=top_k)
    for r, prompt in enumerate(prompts):
        for i in range(steps):
            want = logits_of(d, torch.cat([prompt.cpu(), tokens[r, :i].cpu()]))[0].numpy()
            got = logits[i][r].double().cpu().numpy()
            assert np.abs(got - want).max() <= bound
            # the draw, from the logits that were there
            token, logprob, _, _ = orc.sample(got, noise[i, r].cpu().numpy(), 0.7, int(top_k[r]), 1.0, 0.0)
            assert token == int(tokens[r, i]) and abs(logprob - float(logprobs[r, i])) < 1e-5
    ctx.close()


def test_the_command_runs():
    tokens = example.main(["--questions", "3", "--passages", "5000", "--tokens", "4"])
    assert tokens.shape == (3, 4) and int(tokens.min()) >= 0
    with pytest.raises(RuntimeError):
        ctx = binding.Context(0)
        d = example.Decoder(vocab=64, width=64, layers=1, q_heads=1, heads=1, positions=64)
        example.answer(ctx, d, [torch.zeros(4, dtype=torch.int64, device="cuda")], 2, torch.rand((2, 1, 64), device="cuda"))
        reader = example.Reader(ctx, d, 1, 1, 1)
        reader.step(torch.zeros(17, dtype=torch.int64, device="cuda"), [17], torch.rand((1, 64), device="cuda"))


def test_a_full_cache_is_refused_on_the_host():
    """Too few blocks, or a row of the table too short: nothing is changed, and what fits is served afterwards."""
    ctx = binding.Context(0)
    d = example.Decoder(vocab=64, width=64, layers=1, q_heads=1, heads=1, positions=64)
    tokens, noise = torch.zeros(40, dtype=torch.int64, device="cuda"), torch.rand((1, 64), device="cuda")
    for blocks, width in ((1, 3), (3, 1)):
        reader = example.Reader(ctx, d, 1, blocks, width)
        with pytest.raises(RuntimeError, match="the cache is full"):
            reader.step(tokens[:17], [17], noise)
        drawn, _, _ = reader.step(tokens[:16], [16], noise)
        assert drawn.shape == (1,) and reader.lens.tolist() == [16] and reader.used == 1
        with pytest.raises(RuntimeError, match="the cache is full"):
            reader.step(tokens[:1], [1], noise)
        assert reader.lens.tolist() == [16] and reader.counts == [16]
    ctx.close()
