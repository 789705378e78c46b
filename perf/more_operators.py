"""Measured cases of the reading step over a cache of 8 bits, and of the log-probabilities of tokens.

Three operators: the append of keys and values to a paged cache of e4m3 numbers with a scale for each block and head (norm and
position rotation on the way, as without the 8 bits), the attention over such a cache, and the log-probabilities of given tokens with
rank, entropy and the likeliest tokens of each row of logits.

``listed`` holds the measured cases, ``draw`` gives further ones of the same ranges, ``prepare`` makes a case's inputs
from a seed, ``run`` is one pass: with ``own`` the library's entry points, else the same result from elementary torch
operations in 32 bits (keys, whose rounding to 8 bits has borders, in 64).  ``exact`` computes it from the definition in 64 bits,
``work`` says what a pass has to move and compute.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
MAX_POSITIONS = 32768   # rows of the rotation tables
EPS = 1e-6
LARGEST = 448.0         # of e4m3
LEAST_SCALE = 2.0 ** -126

_context = None


def listed():
    return [
        # the projections of a decoding step: each request adds one token to a block that it has begun before
        dict(name="append8, 64 single tokens", op="append8", tokens=64, requests=64, q_heads=32, kv_heads=8, dim=128, rot=128, pairs=False,
             block=16, dtype="bf16", norm=True),
        # prompt chunks of several requests
        dict(name="append8, 16384 tokens", op="append8", tokens=16384, requests=9, q_heads=32, kv_heads=8, dim=128, rot=128, pairs=False,
             block=16, dtype="bf16", norm=True),
        # a model that rotates a part of each head, in neighbouring pairs; odd numbers of tokens, larger blocks
        dict(name="append8, 4099 part", op="append8", tokens=4099, requests=131, q_heads=12, kv_heads=12, dim=80, rot=32, pairs=True, block=24,
             dtype="f16", norm=True),
        # decoding for a ragged batch of long contexts
        dict(name="attention8, 64 single tokens", op="attention8", requests=64, new_low=1, new_high=1, cached=8191, q_heads=32, kv_heads=8,
             dim=128, block=16, window=0, dtype="bf16"),
        # decoding for one request whose context is a whole collection of passages
        dict(name="attention8, one long", op="attention8", requests=1, new_low=1, new_high=1, cached=131037, q_heads=32, kv_heads=8,
             dim=128, block=64, window=0, dtype="bf16"),
        # drafts of a few tokens each, checked in one call
        dict(name="attention8, 33 drafts", op="attention8", requests=33, new_low=2, new_high=6, cached=5003, q_heads=28, kv_heads=4,
             dim=128, block=32, window=0, dtype="f16"),
        # single tokens and prompt chunks in one call, a window, odd pages, one request that got no memory
        dict(name="attention8, mixed chunks", op="attention8", requests=23, new_low=1, new_high=517, cached=3001, q_heads=16, kv_heads=16,
             dim=64, block=24, window=1024, dtype="f16"),
        # prompt chunks behind long cached contexts
        dict(name="attention8, two chunks of 2048", op="attention8", requests=2, new_low=2048, new_high=2048, cached=14336, q_heads=32,
             kv_heads=8, dim=128, block=16, window=0, dtype="bf16"),
        # a decoding step of a small batch that shows the likeliest tokens
        dict(name="logprobs, 8 of 32000", op="logprobs", rows=8, vocab=32000, top=20, dtype="bf16"),
        # a prompt's tokens scored, an odd vocabulary
        dict(name="logprobs, 517 of 50021", op="logprobs", rows=517, vocab=50021, top=5, dtype="f16"),
        # a large batch of answers over a large vocabulary
        dict(name="logprobs, 4096 of 131072", op="logprobs", rows=4096, vocab=131072, top=20, dtype="bf16"),
        # the same kept in 32 bits, scores alone
        dict(name="logprobs, 1024 of 131072", op="logprobs", rows=1024, vocab=131072, top=0, dtype="f32"),
    ]


def _between(rng, low, high):
    """A whole number of low ... high, spread over the logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["append8", "attention8", "attention8", "logprobs"])
    if op == "append8":
        dim = rng.choice([64, 80, 96, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8])
        tokens = _between(rng, 1, 8191)
        return dict(op=op, tokens=tokens, requests=_between(rng, 1, min(tokens, 300)), q_heads=kv_heads * rng.choice([1, 4, 7]), kv_heads=kv_heads,
                    dim=dim, rot=rng.choice([dim, dim // 2]), pairs=rng.random() < 0.5, block=rng.choice([8, 16, 24, 64]),
                    dtype=rng.choice(["bf16", "f16", "f32"]), norm=rng.random() < 0.8)
    if op == "attention8":
        kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 4, 7, 8])
        q_heads = kv_heads * group
        dim = rng.choice([64, 96, 128, 256])
        new = 1 if rng.random() < 0.4 else _between(rng, 2, 1500)
        cached = _between(rng, 16, 30000)
        most = 3.0e8 if new > 1 else 5.0e7   # (query head, new token, key) triples of the padded batch
        most = min(most / (q_heads * new), 5.0e8 / (kv_heads * dim))   # (and no more keys than the listed cases have)
        requests = max(1, min(_between(rng, 1, 96), int(most / (new + cached))))
        return dict(op=op, requests=requests, new_low=1, new_high=new, cached=cached, q_heads=q_heads, kv_heads=kv_heads, dim=dim,
                    block=rng.choice([8, 16, 24, 64, 128]), window=rng.choice([0, 0, 0, _between(rng, 1, 4096)]),
                    dtype=rng.choice(["bf16", "f16"]))
    vocab = _between(rng, 1000, 131072)
    return dict(op=op, rows=max(1, min(_between(rng, 1, 4096), 2 ** 28 // vocab)), vocab=vocab, top=rng.choice([0, 1, 5, 20, 64]),
                dtype=rng.choice(["bf16", "f16", "f32"]))


def _lengths(case):
    """New and cached lengths of the requests: the same for every seed up to their order, the longest among them."""
    rng = random.Random(case["requests"] * 1000003 + case["cached"])
    new = [_between(rng, case["new_low"], case["new_high"]) for _ in range(case["requests"])]
    cached = [_between(rng, max(1, case["cached"] // 8), case["cached"]) for _ in range(case["requests"])]
    new[0], cached[0] = case["new_high"], case["cached"]
    return new, cached


def _refused(case):
    """Batches of eight and more hold one request that got no memory (by its place in ``_lengths``): its rows see nothing."""
    return 5 if case["requests"] >= 8 else -1


def _handle():
    """The library's context: one for the process, as a serving program keeps it."""
    global _context
    if own and _context is None:
        from paper_1712_02912_amd import binding
        _context = binding.Context(0)
    return _context


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case, ctx=_handle())
    globals()["_prepare_" + case["op"]](case, seed, gen, state)
    return state


def _normal(gen, *shape):
    return torch.randn(shape, device="cuda", generator=gen)


def _whole(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _needed_scale(amax):
    """The smallest power of two s with amax <= 448 s, from 2^-126 on."""
    part, power = torch.frexp(amax)
    power = torch.where(part <= LARGEST / 512, power - 9, power - 8).clamp(min=-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), power), LEAST_SCALE)


def _cached(gen, blocks, block, heads, dim, loud=None):
    """What a cache of so many blocks holds: codes, and a scale for each block and head."""
    x = _normal(gen, blocks, block, heads, dim)
    if loud is not None:
        x *= loud
    scale = _needed_scale(x.abs().amax(dim=(1, 3)))
    return (x / scale[:, None, :, None]).to(torch.float8_e4m3fn), scale


def _prepare_append8(case, seed, gen, state):
    t, requests, hq, hkv, dim, block, dtype = (case[k] for k in ("tokens", "requests", "q_heads", "kv_heads", "dim", "block", "dtype"))
    # one projection's output holds queries, keys and values side by side; a few of the dimensions are much larger
    loud = 1 + 7 * (torch.rand((hq + 2 * hkv) * dim, device="cuda", generator=gen) > 0.98)
    qkv = (_normal(gen, t, (hq + 2 * hkv) * dim) * loud).to(DTYPES[dtype])
    state["q"], state["k"], state["v"] = (x.unflatten(1, (-1, dim)) for x in qkv.split([hq * dim, hkv * dim, hkv * dim], dim=1))
    # the requests' new tokens, and the place in its block that each of them begins at (the same for every seed up to their order)
    rng = random.Random(t * 1000003 + requests)
    cuts = [0] + sorted(rng.sample(range(1, t), requests - 1)) + [t]
    starts = [(b - a, rng.randrange(block)) for a, b in zip(cuts, cuts[1:])]
    random.Random(seed).shuffle(starts)
    lens, firsts = _whole([n for n, _ in starts], torch.int64), _whole([f for _, f in starts], torch.int64)
    held = (firsts + lens + block - 1) // block
    blocks = sum(-(-(f + n) // block) for n, f in starts) + 2
    request = torch.repeat_interleave(torch.arange(requests, device="cuda"), lens, output_size=t)
    place = firsts[request] + torch.arange(t, device="cuda") - (lens.cumsum(0) - lens)[request]
    pool = torch.randperm(blocks, device="cuda", generator=gen)
    state["slots"] = pool[(held.cumsum(0) - held)[request] + place // block] * block + place % block
    before = torch.randint(0, (MAX_POSITIONS - t) // block, (requests,), device="cuda", generator=gen) * block
    state["positions"] = (before[request] + place).to(torch.int32)
    half = case["rot"] // 2
    angle = torch.arange(MAX_POSITIONS, device="cuda", dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    state["cos"], state["sin"] = angle.cos().float(), angle.sin().float()
    state["q_weight"] = 1 + 0.2 * _normal(gen, dim) if case["norm"] else None
    state["k_weight"] = 1 + 0.2 * _normal(gen, dim) if case["norm"] else None
    # what the blocks hold already: of the new tokens' size, or smaller, so that some of their scales have to grow
    for what in ("key", "value"):
        codes, scale = _cached(gen, blocks, block, hkv, dim, 2.0 ** -torch.randint(0, 4, (blocks, 1, hkv, 1), device="cuda", generator=gen))
        state[what + "_cache"], state[what + "_scales"] = codes, scale
    state["out"] = torch.empty((t, hq, dim), dtype=DTYPES[dtype], device="cuda")


def _prepare_attention8(case, seed, gen, state):
    new, cached = _lengths(case)
    order = list(range(len(new)))
    random.Random(seed).shuffle(order)
    new, cached = [new[i] for i in order], [cached[i] for i in order]
    hq, hkv, dim, block, dtype = (case[k] for k in ("q_heads", "kv_heads", "dim", "block", "dtype"))
    kv = [n + c for n, c in zip(new, cached)]
    # block tables at places of a pool in no order
    counts, width = [-(-x // block) for x in kv], -(-max(kv) // block)
    total, held = sum(counts), _whole(counts, torch.int64)
    pool = torch.randperm(total + 8, device="cuda", generator=gen).to(torch.int32)
    column = torch.arange(width, device="cuda")
    at = (held.cumsum(0) - held)[:, None] + column[None, :]
    table = torch.where(column[None, :] < held[:, None], pool[at.clamp(max=total + 7)], -1).contiguous()
    # queries of all sharpness: some spread over all keys, for others a few keys matter; some dimensions of the keys are larger
    loud = 1 + 3 * (torch.rand(dim, device="cuda", generator=gen) > 0.97)
    state["key_cache"], state["key_scales"] = _cached(gen, total + 8, block, hkv, dim, loud)
    state["value_cache"], state["value_scales"] = _cached(gen, total + 8, block, hkv, dim)
    t = sum(new)
    gain = 0.5 + 2 * torch.rand((t, hq, 1), device="cuda", generator=gen)
    state["q"] = (_normal(gen, t, hq, dim) * gain / loud).to(DTYPES[dtype])
    if _refused(case) >= 0:
        kv[order.index(_refused(case))] = -1
    state.update(block_tables=table, max_new=max(new), max_kv=max(kv), kv_lens=_whole(kv), scale=dim ** -0.5,
                 cu_new=_whole([0] + torch.tensor(new).cumsum(0).tolist()))
    state["out"] = torch.empty((t, hq, dim), dtype=DTYPES[dtype], device="cuda")
    state["lse"] = torch.empty((t, hq), dtype=torch.float32, device="cuda")


def _prepare_logprobs(case, seed, gen, state):
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    # a bulk of unlikely tokens, a head of likely ones, some that a grammar rules out
    logits = _normal(gen, rows, vocab).mul_(2)
    likely = torch.rand((rows, vocab), device="cuda", generator=gen)
    logits += (likely < 40 / vocab) * (4 + 3 * torch.rand((rows, 1), device="cuda", generator=gen)) * (1 + likely * (vocab / 40))
    logits.masked_fill_(likely > 0.99, -math.inf)
    # tokens as the model would draw them, a few as a text has them against all odds
    drawn = (logits - likely.uniform_(generator=gen).log_().neg_().log_()).argmax(dim=1)
    odd = torch.rand(rows, device="cuda", generator=gen) < 0.1
    state["tokens"] = torch.where(odd, torch.randint(0, vocab, (rows,), device="cuda", generator=gen), drawn)
    state["logits"] = logits.to(DTYPES[case["dtype"]])
    state["results"] = (torch.empty(rows, dtype=torch.float32, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"),
                        torch.empty(rows, dtype=torch.float32, device="cuda"), torch.empty((rows, top), dtype=torch.int64, device="cuda"),
                        torch.empty((rows, top), dtype=torch.float32, device="cuda"))


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["op"]](state)


# -- the library's entry points ---------------------------------------------------------------------------------------
def _own_append8(s):
    q = s["ctx"].pq_kv_append8(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["key_cache"], s["value_cache"], s["key_scales"],
                               s["value_scales"], s["cos"], s["sin"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, norm=s["norm"],
                               pairs=s["pairs"], out=s["out"])
    return q, s["key_cache"], s["value_cache"], s["key_scales"], s["value_scales"]


def _own_attention8(s):
    return s["ctx"].pq_kv_attention8(s["q"], s["key_cache"], s["value_cache"], s["key_scales"], s["value_scales"], s["block_tables"],
                                     s["cu_new"], s["kv_lens"], s["max_new"], scale=s["scale"], window=s["window"], out=s["out"], lse=s["lse"])


def _own_logprobs(s):
    return s["ctx"].pq_token_logprobs(s["logits"], s["tokens"], top=s["top"], out=s["results"])


# -- the plain forms --------------------------------------------------------------------------------------------------
def _plain_turn(x, weight, s):
    """Norm and rotation of heads [t][h][dim], in x's type."""
    if s["norm"]:
        x = x * torch.rsqrt((x * x).mean(dim=2, keepdim=True) + EPS) * weight
    position, half = s["positions"].long(), s["rot"] // 2
    cos, sin = s["cos"][position][:, None, :], s["sin"][position][:, None, :]
    if s["pairs"]:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=3).flatten(2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=2)
    return torch.cat([turned, x[..., 2 * half:]], dim=2)


def _plain_store(codes, scales, x, s):
    """Rows x [t][h][dim] into a cache [blocks][block][h][dim] with scales [blocks][h]."""
    block = codes.shape[1]
    at, place = s["slots"] // block, s["slots"] % block
    amax = torch.where(x.abs() < math.inf, x.abs(), 0).amax(dim=2)
    most = torch.full_like(scales, -1).scatter_reduce(0, at[:, None].expand_as(amax), amax, "amax")
    first = torch.full((codes.shape[0],), block, device="cuda").scatter_reduce(0, at, place, "amin")   # rows before it stay
    held = (first > 0)[:, None]
    fresh = torch.maximum(torch.where(held, scales, LEAST_SCALE), _needed_scale(most))
    fresh = torch.where(most < 0, scales, fresh)
    shrink = torch.where(held, scales / fresh, 1)
    kept = torch.arange(block, device="cuda")[None, :] < torch.where(most[:, 0] < 0, 0, first)[:, None]
    factor = torch.where(kept[:, :, None], shrink[:, None, :], 1)[..., None]
    codes.copy_(torch.where(factor == 1, codes.float(), codes.float() * factor).to(codes.dtype))
    scales.copy_(fresh)
    codes.view(torch.uint8).flatten(0, 1)[s["slots"]] = \
        (x / fresh[at][..., None]).clamp(-LARGEST, LARGEST).to(codes.dtype).view(torch.uint8)


def _plain_append8(s):
    q = _plain_turn(s["q"].float(), s["q_weight"], s).to(s["q"].dtype)
    _plain_store(s["key_cache"], s["key_scales"], _plain_turn(s["k"].double(), s["k_weight"], s).float(), s)
    _plain_store(s["value_cache"], s["value_scales"], s["v"].float(), s)
    return q, s["key_cache"], s["value_cache"], s["key_scales"], s["value_scales"]


def _plain_attention8(s):
    t, hq, dim = s["q"].shape
    hkv, block = s["kv_heads"], s["block"]
    group, requests, max_new, max_kv = hq // hkv, s["requests"], s["max_new"], s["max_kv"]
    new, kv = s["cu_new"][1:] - s["cu_new"][:-1], s["kv_lens"]
    # queries padded to [request][kv head][head of the group, token][dim], keys and values to [request][kv head][key][dim]
    step = torch.arange(max_new, device="cuda")
    row = (s["cu_new"][:-1, None] + step).clamp(max=t - 1)
    q = s["q"][row].float().unflatten(2, (hkv, group)).permute(0, 2, 3, 1, 4).reshape(requests, hkv, group * max_new, dim)
    place = torch.arange(max_kv, device="cuda")
    at = s["block_tables"][:, place // block].long().clamp(min=0)
    slot = at * block + place % block
    keys = s["key_cache"].view(torch.uint8).flatten(0, 1)[slot].view(torch.float8_e4m3fn).float() * s["key_scales"][at][..., None]
    values = s["value_cache"].view(torch.uint8).flatten(0, 1)[slot].view(torch.float8_e4m3fn).float() * s["value_scales"][at][..., None]
    keys, values = keys.permute(0, 2, 3, 1), values.permute(0, 2, 1, 3)
    score = (torch.matmul(q, keys) * s["scale"]).view(requests, hkv, group, max_new, max_kv)
    at = kv[:, None] - new[:, None] + step                       # the position of each new token
    seen = (place <= at[:, :, None]) & (kv[:, None, None] > 0)
    if s["window"] > 0:
        seen = seen & (place > at[:, :, None] - s["window"])
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(dim=4, keepdim=True)
    weight = torch.exp(score - top.clamp(min=-1e30))
    total = weight.sum(dim=4, keepdim=True)
    out = torch.matmul(weight.view(requests, hkv, group * max_new, max_kv), values).view(requests, hkv, group, max_new, dim)
    out = out / torch.where(total > 0, total, 1)
    lse = (top + torch.log(total))[..., 0]
    request = torch.repeat_interleave(torch.arange(requests, device="cuda"), new, output_size=t)
    index = torch.arange(t, device="cuda") - s["cu_new"][request]
    return out[request, :, :, index].reshape(t, hq, dim).to(s["q"].dtype), lse[request, :, :, index].reshape(t, hq)


def _plain_logprobs(s):
    x, tokens = s["logits"].float(), s["tokens"][:, None]
    vocab = x.shape[1]
    top = x.amax(dim=1, keepdim=True)
    below = x - top
    weight = torch.exp(below)
    total = weight.sum(dim=1, keepdim=True)
    chosen = x.gather(1, tokens)
    logprob = chosen - top - torch.log(total)
    entropy = torch.log(total) - torch.where(weight > 0, weight * below, 0).sum(dim=1, keepdim=True) / total
    place = torch.arange(vocab, device="cuda")
    rank = ((x > chosen) | ((x == chosen) & (place < tokens))).sum(dim=1)
    # one whole number for each token: by the logit, equal ones by the smaller index
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * 2 ** 20 + (vocab - 1 - place)
    first = torch.topk(key, s["top"], dim=1, sorted=True)[1]
    return logprob[:, 0], rank.int(), entropy[:, 0], first, x.gather(1, first) - top - torch.log(total)


# -- from the definitions, in 64 bits ---------------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    return globals()["_exact_" + case["op"]](state)


def _exact_rounded(x):
    """The e4m3 numbers nearest to x, ties to the even one: eight steps in each octave, from 2^-6 downwards steps of 2^-9."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(-LARGEST, LARGEST)


def _exact_append8(s):
    half = s["rot"] // 2
    place = s["positions"].long()
    cos, sin = s["cos"].double()[place].unsqueeze(1), s["sin"].double()[place].unsqueeze(1)
    # where the two members of rotated pair i are
    first = torch.arange(half, device="cuda") * (2 if s["pairs"] else 1)
    second = first + (1 if s["pairs"] else half)
    found = []
    for x, weight in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.double()
        if s["norm"]:
            y = y / (y.square().sum(-1, keepdim=True) / y.shape[-1] + EPS).sqrt() * weight.double()
        z = y.clone()
        z[..., first] = y[..., first] * cos - y[..., second] * sin
        z[..., second] = y[..., second] * cos + y[..., first] * sin
        found.append(z)
    # the new rows of each block side by side: [touched block][place][head][dim], zeros where there is none
    size = s["block"]
    touched, index = torch.unique(s["slots"] // size, return_inverse=True)
    there = torch.zeros((len(touched), size), dtype=torch.bool, device="cuda")
    there[index, s["slots"] % size] = True
    started = there.long().argmax(dim=1)
    before = torch.arange(size, device="cuda")[None, :] < started[:, None]
    caches, all_scales = [], []
    for what, rows in (("key", found[1]), ("value", s["v"].double())):
        cache, scales = s[what + "_cache"].double(), s[what + "_scales"].double()
        fresh = torch.zeros((len(touched), size, *rows.shape[1:]), dtype=torch.float64, device="cuda")
        fresh[index, s["slots"] % size] = rows
        need = torch.exp2(torch.ceil(torch.log2(fresh.abs().amax(dim=(1, 3)).clamp(min=LEAST_SCALE) / LARGEST)).clamp(min=-126))
        old = scales[touched]
        scale = torch.where((started > 0)[:, None], torch.maximum(old, need), need)
        kept = cache[touched]
        kept = torch.where(before[..., None, None], _exact_rounded(kept * (old / scale)[:, None, :, None]), kept)
        cache[touched] = torch.where(there[..., None, None], _exact_rounded(fresh / scale[:, None, :, None]), kept)
        scales[touched] = scale
        caches.append(cache)
        all_scales.append(scales)
    return found[0], *caches, *all_scales


def _exact_attention8(s):
    t, hq, dim = s["q"].shape
    group = hq // s["kv_heads"]
    out = torch.zeros((t, hq, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((t, hq), -math.inf, dtype=torch.float64, device="cuda")
    cu, kv = s["cu_new"].tolist(), s["kv_lens"].tolist()
    for r in range(s["requests"]):
        n = kv[r]
        if n <= 0:
            continue
        blocks = s["block_tables"][r, :-(-n // s["block"])].long()
        keys, values = ((s[w + "_cache"].view(torch.uint8)[blocks].view(torch.float8_e4m3fn).double() * s[w + "_scales"].double()[blocks][:, None, :, None])
                        .flatten(0, 1)[:n] for w in ("key", "value"))
        for a in range(cu[r], cu[r + 1], 512):
            b = min(cu[r + 1], a + 512)
            at = n - cu[r + 1] + torch.arange(a, b, device="cuda")[:, None]
            key = torch.arange(n, device="cuda")[None, :]
            hidden = (key > at) | ((key <= at - s["window"]) if s["window"] > 0 else (key < 0))
            for h in range(hq):
                score = (s["q"][a:b, h].double() @ keys[:, h // group].T) * s["scale"]
                score[hidden] = -math.inf
                lse[a:b, h] = torch.logsumexp(score, dim=1)
                share = torch.where(hidden, 0.0, torch.exp(score - lse[a:b, h, None]))
                out[a:b, h] = share @ values[:, h // group]
    return out, lse


def _exact_logprobs(s):
    found = []
    for a in range(0, s["rows"], 256):
        x, token = s["logits"][a:a + 256].double(), s["tokens"][a:a + 256]
        total = torch.logsumexp(x, dim=1)
        value, order = torch.sort(x, dim=1, descending=True, stable=True)
        share = value - total[:, None]
        found.append((x[torch.arange(len(token), device="cuda"), token] - total, (order == token[:, None]).long().argmax(dim=1).int(),
                      -torch.where(share > -math.inf, share * share.exp(), 0).sum(dim=1), order[:, :s["top"]].clone(), share[:, :s["top"]].clone()))
    return tuple(torch.cat(x) for x in zip(*found))


# -- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "append8":
        t, hq, hkv, dim = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"]
        blocks = t // case["block"] + case["requests"]
        return {"bytes": t * ((2 * hq + 2 * hkv) * dim * BYTES[case["dtype"]] + 2 * hkv * dim + 4 * case["rot"] + 12) + 16 * blocks * hkv,
                "flops": t * ((hq + hkv) * (4 * dim + 3 * case["rot"]) + 4 * hkv * dim)}
    if op == "attention8":
        new, cached = _lengths(case)
        pairs = read = 0
        for i, (n, c) in enumerate(zip(new, cached)):
            if i == _refused(case):
                continue
            w = case["window"] or n + c
            pairs += sum(min(w, p + 1) for p in range(c, c + n))
            read += min(n + c, w + n - 1)
        e, dim, heads = BYTES[case["dtype"]], case["dim"], case["kv_heads"]
        return {"bytes": 2 * sum(new) * case["q_heads"] * dim * e + 2 * read * heads * (dim + 4 / case["block"]) + 4 * sum(new) * case["q_heads"],
                "flops": 4 * pairs * case["q_heads"] * dim}
    size = case["rows"] * case["vocab"]
    return {"bytes": size * BYTES[case["dtype"]] + case["rows"] * (20 + 12 * case["top"]), "flops": 6 * size}
