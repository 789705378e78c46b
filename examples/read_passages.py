"""Retrieve and read: the search finds passages for each question, a small decoder reads them and answers.

    python examples/read_passages.py [--questions 16] [--passages 100000] [--tokens 32] [--dtype bf16] [--cache8]

Passages are embeddings in a PQ 8x8 index; a question's nearest ones come from the tables and scan calls.  Their tokens and the
question's are one chunk of new tokens of a request, then every step adds one drawn token to each.  A step is the plan of
the paged cache, for every layer the append and the attention (between torch's products with the layer's weights), and the
draw.  With --cache8 the cache holds 8 bits an element.  Data and weights are random: what is shown is how the calls go together, and what a step takes.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1712_02912_amd import binding, datagen  # noqa: E402

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def find_passages(ctx, index, codebooks, questions, count):
    """Ids [questions][count] of the passages nearest to each question."""
    luts = ctx.pq_build_luts(questions, codebooks)
    return ctx.pq_adc_scan_topk(index, binding.CODES_U8, luts, count)[1]


class Decoder:
    """Weights of a small decoder with grouped heads, norms of queries and keys, and rotated positions."""

    def __init__(self, vocab=4096, width=512, layers=2, q_heads=8, heads=2, dim=64, positions=4096, dtype=torch.bfloat16, seed=0):
        self.vocab, self.width, self.q_heads, self.heads, self.dim, self.dtype = vocab, width, q_heads, heads, dim, dtype
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(rows, columns):
            return (torch.randn((rows, columns), device="cuda", generator=gen) * rows ** -0.5).to(dtype)

        self.embedding = torch.randn((vocab, width), device="cuda", generator=gen).to(dtype)
        self.head = weight(width, vocab)
        self.layers = [dict(qkv=weight(width, (q_heads + 2 * heads) * dim), out=weight(q_heads * dim, width),
                            up=weight(width, 4 * width), down=weight(4 * width, width),
                            q_norm=torch.rand(dim, device="cuda", generator=gen) + 0.5,
                            k_norm=torch.rand(dim, device="cuda", generator=gen) + 0.5) for _ in range(layers)]
        angles = torch.arange(positions, device="cuda")[:, None] * 10000.0 ** (-torch.arange(dim // 2, device="cuda") / (dim // 2))
        self.cos, self.sin = angles.cos(), angles.sin()

    @staticmethod
    def norm(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(dim=-1, keepdim=True) + 1e-6)).to(x.dtype)


class Reader:
    """Requests in a paged cache: the state of a batch that is being served."""

    def __init__(self, ctx, decoder, requests, blocks, width, block_size=16, cache8=False):
        self.ctx, self.decoder, self.block_size = ctx, decoder, block_size
        shape = (blocks, block_size, decoder.heads, decoder.dim)
        # of each layer keys and values, of 8 bits also their scales
        if cache8:
            self.append, self.attention = ctx.pq_kv_append8, ctx.pq_kv_attention8
            self.caches = [tuple(torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)) +
                           tuple(torch.ones((blocks, decoder.heads), device="cuda") for _ in range(2)) for _ in decoder.layers]
        else:
            self.append, self.attention = ctx.pq_kv_append, ctx.pq_kv_attention
            self.caches = [tuple(torch.zeros(shape, dtype=decoder.dtype, device="cuda") for _ in range(2)) for _ in decoder.layers]
        self.tables = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.counts = [0] * requests                      # the same on the host, which hands out the blocks
        self.free = torch.arange(blocks, dtype=torch.int32, device="cuda")
        self.used = 0

    def step(self, tokens, new, noise, **filters):
        """Takes new[r] further tokens of every request (`tokens`: one request after another) and draws the next one of each
        with noise [requests][vocab].  Returns (tokens, logprobs, logits)."""
        ctx, d = self.ctx, self.decoder
        blocks = sum(-(-(c + n) // self.block_size) - -(-c // self.block_size) for c, n in zip(self.counts, new))
        if self.used + blocks > self.free.numel() or max(c + n for c, n in zip(self.counts, new)) > self.tables.shape[1] * self.block_size:
            raise RuntimeError("the cache is full")
        lens = torch.tensor(new, dtype=torch.int32, device="cuda")
        cu, kv, positions, slots, _ = ctx.pq_kv_plan(lens, self.lens, self.tables, self.free[self.used:self.used + blocks],
                                                     self.block_size, len(tokens))
        self.used += blocks
        self.counts = [c + n for c, n in zip(self.counts, new)]
        self.lens = kv                                    # (a refused request, of which there is none here, would stay refused)
        x = d.embedding[tokens]
        for w, cache in zip(d.layers, self.caches):
            qkv = (d.norm(x) @ w["qkv"]).view(len(tokens), d.q_heads + 2 * d.heads, d.dim)
            q, k, v = qkv.split((d.q_heads, d.heads, d.heads), dim=1)       # (views: the append reads them with their strides)
            q = self.append(q, k, v, positions, slots, *cache, d.cos, d.sin, w["q_norm"], w["k_norm"])
            out, _ = self.attention(q, *cache, self.tables, cu, kv, max(new))
            x = x + out.view(len(tokens), -1) @ w["out"]
            x = x + torch.nn.functional.silu(d.norm(x) @ w["up"]) @ w["down"]
        logits = d.norm(x[(cu[1:] - 1).long()]) @ d.head
        drawn, logprobs = ctx.pq_sample_tokens(logits, noise, **filters)
        return drawn, logprobs, logits


def answer(ctx, decoder, prompts, tokens, noise, cache8=False, **filters):
    """Draws `tokens` tokens for each prompt (lists of token tensors) with noise [tokens][prompts][vocab].  Returns the tokens
    [prompts][tokens], their logprobs and every step's logits."""
    block_size, longest = 16, max(len(p) for p in prompts) + tokens
    width = -(-longest // block_size)
    reader = Reader(ctx, decoder, len(prompts), len(prompts) * width, width, block_size, cache8)
    drawn, logprobs, logits = [], [], []
    for i in range(tokens):
        inputs, new = (torch.cat(prompts), [len(p) for p in prompts]) if i == 0 else (drawn[-1], [1] * len(prompts))
        t, lp, l = reader.step(inputs, new, noise[i], **filters)
        drawn.append(t)
        logprobs.append(lp)
        logits.append(l)
    return torch.stack(drawn, dim=1), torch.stack(logprobs, dim=1), logits


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--questions", type=int, default=16)
    parser.add_argument("--passages", type=int, default=100000)
    parser.add_argument("--tokens", type=int, default=32, help="tokens of each answer")
    parser.add_argument("--dtype", choices=sorted(DTYPES), default="bf16")
    parser.add_argument("--cache8", action="store_true", help="keys and values in 8 bits")
    args = parser.parse_args(argv)

    ctx = binding.Context(0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    decoder = Decoder(dtype=DTYPES[args.dtype])
    # passages of 64 tokens and their embeddings; a question lies near one of them
    mix = datagen.sift_like()
    embeddings = mix.sample_device(args.passages, datagen.SEED_DATA)
    passages = torch.randint(decoder.vocab, (args.passages, 64), device="cuda", generator=gen)
    codebooks = torch.from_numpy(datagen.sampled_codebooks(mix, 8, 256)).cuda()
    index = ctx.pq_encode(embeddings, codebooks)
    meant = torch.randint(args.passages, (args.questions,), device="cuda", generator=gen)
    questions = embeddings[meant] + torch.randn((args.questions, embeddings.shape[1]), device="cuda", generator=gen)

    ids = find_passages(ctx, index, codebooks, questions, 4)
    found = int((ids == meant[:, None]).any(dim=1).sum())
    prompts = [torch.cat([passages[i].flatten(), torch.randint(decoder.vocab, (5 + q % 20,), device="cuda", generator=gen)])
               for q, i in enumerate(ids)]
    noise = torch.rand((args.tokens, args.questions, decoder.vocab), device="cuda", generator=gen)
    filters = dict(temperature=torch.full((args.questions,), 0.8, device="cuda"), top_p=torch.full((args.questions,), 0.95, device="cuda"))
    for run in ("first", "second"):
        torch.cuda.synchronize()
        start = time.perf_counter()
        tokens, logprobs, logits = answer(ctx, decoder, prompts, args.tokens, noise, args.cache8, **filters)
        torch.cuda.synchronize()
        print(f"{run} run: {args.questions} answers of {args.tokens} tokens over {sum(len(p) for p in prompts)} tokens of passages and "
              f"questions: {1e3 * (time.perf_counter() - start):.2f} ms")
    print(f"the passage that was meant is among the four found for {found} of {args.questions} questions")
    print("first answer:", tokens[0].tolist(), f"log-likelihood {logprobs[0].sum().item():.2f}")
    # what the model itself says of the drawn tokens, without temperature and filters, and which it had found likeliest
    _, ranks, entropy, likeliest, _ = ctx.pq_token_logprobs(logits[0], tokens[:, 0].contiguous(), 3)
    print(f"its first token is number {ranks[0].item()} of {decoder.vocab} (likeliest: {likeliest[0].tolist()}), entropy {entropy[0].item():.2f}")
    ctx.close()
    return tokens


if __name__ == "__main__":
    main()
