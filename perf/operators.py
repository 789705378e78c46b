"""Measured cases of the reading step: what a language model does with the passages that a search has found.

Four operators, in the order in which one step of a serving program calls them: the plan of a paged cache of keys and
values (block tables, positions and slots from the requests' lengths), the append (norm and position rotation of
queries and keys, written into the cache), the attention of the new tokens over the cache, and the draw of the next
tokens from the logits.

``listed`` holds the measured cases, ``draw`` gives further ones of the same ranges, ``prepare`` makes a case's inputs
from a seed, ``run`` is one pass: with ``own`` the library's entry points, else the same result from elementary torch
operations in 32 bits.  ``exact`` computes it from the definition in 64 bits, ``work`` says what a pass has to move and
compute.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
MAX_POSITIONS = 32768   # rows of the rotation tables
EPS = 1e-6

_context = None


def listed():
    return [
        # one decoding step of a small batch: every request adds one token, most need no fresh block
        dict(name="plan, 64 single tokens", op="plan", requests=64, new_low=1, new_high=1, cached=8191, block=16),
        # admission of a full queue: prompts of all lengths on top of cached passages
        dict(name="plan, 1777 mixed", op="plan", requests=1777, new_low=1, new_high=611, cached=4000, block=16),
        # the projections of a decoding step
        dict(name="append, 64 tokens", op="append", tokens=64, q_heads=32, kv_heads=8, dim=128, rot=128, pairs=False, block=16,
             dtype="bf16", norm=True),
        # a chunk of prompt tokens of several requests
        dict(name="append, 16384 tokens", op="append", tokens=16384, q_heads=32, kv_heads=8, dim=128, rot=128, pairs=False, block=16,
             dtype="bf16", norm=True),
        # a model that rotates a part of each head, in neighbouring pairs, kept in 32 bits; an odd number of tokens
        dict(name="append, 4099 part", op="append", tokens=4099, q_heads=12, kv_heads=12, dim=80, rot=32, pairs=True, block=24,
             dtype="f32", norm=True),
        # decoding for a ragged batch of long contexts
        dict(name="attention, 64 single tokens", op="attention", requests=64, new_low=1, new_high=1, cached=8191, q_heads=32, kv_heads=8,
             dim=128, block=16, window=0, dtype="bf16"),
        # decoding for one request whose context is a whole collection of passages
        dict(name="attention, one long", op="attention", requests=1, new_low=1, new_high=1, cached=131037, q_heads=32, kv_heads=8,
             dim=128, block=64, window=0, dtype="bf16"),
        # single tokens and prompt chunks in one call, a window, odd pages, one request that got no memory
        dict(name="attention, mixed chunks", op="attention", requests=23, new_low=1, new_high=517, cached=3001, q_heads=16, kv_heads=16,
             dim=64, block=24, window=1024, dtype="f16"),
        # prompt chunks behind long cached contexts
        dict(name="attention, two chunks of 2048", op="attention", requests=2, new_low=2048, new_high=2048, cached=14336, q_heads=32,
             kv_heads=8, dim=128, block=16, window=0, dtype="bf16"),
        # the draw of a small batch with the usual filters, each request its own
        dict(name="sample, 8 of 32000", op="sample", rows=8, vocab=32000, filters="mixed", dtype="bf16"),
        # plain softmax draws, an odd vocabulary
        dict(name="sample, 33 of 50021 all", op="sample", rows=33, vocab=50021, filters="none", dtype="f16"),
        # a large batch over a large vocabulary
        dict(name="sample, 256 of 131072", op="sample", rows=256, vocab=131072, filters="mixed", dtype="f32"),
    ]


def _between(rng, low, high):
    """A whole number of low ... high, spread over the logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["plan", "append", "attention", "attention", "sample"])
    if op == "plan":
        requests = _between(rng, 1, 1777)
        return dict(op=op, requests=requests, new_low=1, new_high=_between(rng, 1, 600), cached=_between(rng, 16, 8191),
                    block=rng.choice([8, 16, 24, 64]))
    if op == "append":
        dim = rng.choice([64, 80, 96, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8])
        return dict(op=op, tokens=_between(rng, 1, 8191), q_heads=kv_heads * rng.choice([1, 4, 7]), kv_heads=kv_heads, dim=dim,
                    rot=rng.choice([dim, dim // 2]), pairs=rng.random() < 0.5, block=rng.choice([8, 16, 24, 64]),
                    dtype=rng.choice(["bf16", "f16", "f32"]), norm=rng.random() < 0.8)
    if op == "attention":
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
    return dict(op=op, rows=max(1, min(_between(rng, 1, 256), 2 ** 25 // vocab)), vocab=vocab, filters=rng.choice(["mixed", "mixed", "none"]),
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


def _shuffled_lengths(case, seed):
    new, cached = _lengths(case)
    order = list(range(len(new)))
    random.Random(seed).shuffle(order)
    return [new[i] for i in order], [cached[i] for i in order], order


def _tables(block_counts, width, gen):
    """Block tables of requests that hold so many blocks each, at places of a pool in no order; the pool's size."""
    counts = _whole(block_counts, torch.int64)
    total = sum(block_counts)
    pool = torch.randperm(total + 8, device="cuda", generator=gen).to(torch.int32)
    column = torch.arange(width, device="cuda")
    at = (counts.cumsum(0) - counts)[:, None] + column[None, :]
    held = column[None, :] < counts[:, None]
    return torch.where(held, pool[at.clamp(max=total + 7)], -1).contiguous(), pool[total:], total + 8


def _prepare_plan(case, seed, gen, state):
    new, cached, _ = _shuffled_lengths(case, seed)
    block = case["block"]
    have = [-(-c // block) for c in cached]
    fresh = sum(-(-(c + n) // block) - h for c, n, h in zip(cached, new, have))
    width = -(-(case["cached"] + case["new_high"]) // block)
    table, _, pool = _tables(have, width, gen)
    state.update(ntokens=sum(new), new_lens=_whole(new), cached_lens=_whole(cached), block_tables=table,
                 free_blocks=(pool + torch.randperm(fresh + 5, device="cuda", generator=gen)).to(torch.int32))
    r, t = case["requests"], state["ntokens"]
    state["out"] = (torch.empty(r + 1, dtype=torch.int32, device="cuda"), torch.empty(r, dtype=torch.int32, device="cuda"),
                    torch.empty(t, dtype=torch.int32, device="cuda"), torch.empty(t, dtype=torch.int64, device="cuda"),
                    torch.empty(1, dtype=torch.int32, device="cuda"))


def _prepare_append(case, seed, gen, state):
    t, hq, hkv, dim, block, dtype = (case[k] for k in ("tokens", "q_heads", "kv_heads", "dim", "block", "dtype"))
    # one projection's output holds queries, keys and values side by side; a few of the dimensions are much larger
    loud = 1 + 7 * (torch.rand((hq + 2 * hkv) * dim, device="cuda", generator=gen) > 0.98)
    qkv = (_normal(gen, t, (hq + 2 * hkv) * dim) * loud).to(DTYPES[dtype])
    state["q"], state["k"], state["v"] = (x.unflatten(1, (-1, dim)) for x in qkv.split([hq * dim, hkv * dim, hkv * dim], dim=1))
    blocks = -(-t // block) + 2
    state["slots"] = torch.randperm(blocks * block, device="cuda", generator=gen)[:t].contiguous()
    state["positions"] = torch.randint(0, MAX_POSITIONS, (t,), device="cuda", generator=gen, dtype=torch.int32)
    half = case["rot"] // 2
    angle = torch.arange(MAX_POSITIONS, device="cuda", dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    state["cos"], state["sin"] = angle.cos().float(), angle.sin().float()
    state["q_weight"] = 1 + 0.2 * _normal(gen, dim) if case["norm"] else None
    state["k_weight"] = 1 + 0.2 * _normal(gen, dim) if case["norm"] else None
    state["key_cache"] = _normal(gen, blocks, block, hkv, dim).to(DTYPES[dtype])
    state["value_cache"] = _normal(gen, blocks, block, hkv, dim).to(DTYPES[dtype])
    state["out"] = torch.empty((t, hq, dim), dtype=DTYPES[dtype], device="cuda")


def _prepare_attention(case, seed, gen, state):
    new, cached, order = _shuffled_lengths(case, seed)
    hq, hkv, dim, block, dtype = (case[k] for k in ("q_heads", "kv_heads", "dim", "block", "dtype"))
    kv = [n + c for n, c in zip(new, cached)]
    table, _, pool = _tables([-(-x // block) for x in kv], -(-max(kv) // block), gen)
    # queries of all sharpness: some spread over all keys, for others a few keys matter
    key_cache, value_cache = _normal(gen, pool, block, hkv, dim), _normal(gen, pool, block, hkv, dim)
    state["key_cache"], state["value_cache"] = key_cache.to(DTYPES[dtype]), value_cache.to(DTYPES[dtype])
    del key_cache, value_cache
    t = sum(new)
    gain = 0.5 + 2 * torch.rand((t, hq, 1), device="cuda", generator=gen)
    state["q"] = (_normal(gen, t, hq, dim) * gain).to(DTYPES[dtype])
    if _refused(case) >= 0:
        kv[order.index(_refused(case))] = -1
    state.update(block_tables=table, max_new=max(new), max_kv=max(kv), kv_lens=_whole(kv), scale=dim ** -0.5,
                 cu_new=_whole([0] + torch.tensor(new).cumsum(0).tolist()))
    state["out"] = torch.empty((t, hq, dim), dtype=DTYPES[dtype], device="cuda")
    state["lse"] = torch.empty((t, hq), dtype=torch.float32, device="cuda")


def _prepare_sample(case, seed, gen, state):
    rows, vocab = case["rows"], case["vocab"]
    # a bulk of unlikely tokens, a head of likely ones, some that a grammar rules out
    logits = 2 * _normal(gen, rows, vocab)
    head = torch.rand((rows, vocab), device="cuda", generator=gen) < 40 / vocab
    logits += head * (4 + 3 * _normal(gen, rows, vocab).abs())
    logits[torch.rand((rows, vocab), device="cuda", generator=gen) < 0.01] = -math.inf
    state["logits"] = logits.to(DTYPES[case["dtype"]])
    state["noise"] = torch.rand((rows, vocab), device="cuda", generator=gen)

    def pick(choices, dtype):
        return _whole(choices, dtype)[torch.randint(0, len(choices), (rows,), device="cuda", generator=gen)]

    if case["filters"] == "mixed":
        state["temperature"] = pick([0.0, 0.3, 0.6, 0.7, 0.8, 1.0, 1.0, 1.3], torch.float32)
        state["top_k"] = pick([0, 0, 1, 20, 40, 50, 200, 1000], torch.int32)
        state["top_p"] = pick([0.5, 0.8, 0.9, 0.9, 0.95, 0.99, 1.0, 1.0], torch.float32)
        state["min_p"] = pick([0.0, 0.0, 0.0, 0.02, 0.05, 0.1], torch.float32)
    else:
        state["temperature"] = pick([0.7, 1.0, 1.3], torch.float32)
        state["top_k"] = state["top_p"] = state["min_p"] = None
    state["out"] = (torch.empty(rows, dtype=torch.int64, device="cuda"), torch.empty(rows, dtype=torch.float32, device="cuda"))


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["op"]](state)


# -- the library's entry points ---------------------------------------------------------------------------------------
def _own_plan(s):
    out = s["ctx"].pq_kv_plan(s["new_lens"], s["cached_lens"], s["block_tables"], s["free_blocks"], s["block"], s["ntokens"],
                              out=s["out"])
    return (s["block_tables"],) + tuple(out)


def _own_append(s):
    q = s["ctx"].pq_kv_append(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["key_cache"], s["value_cache"], s["cos"],
                              s["sin"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, norm=s["norm"], pairs=s["pairs"],
                              out=s["out"])
    return q, s["key_cache"], s["value_cache"]


def _own_attention(s):
    return s["ctx"].pq_kv_attention(s["q"], s["key_cache"], s["value_cache"], s["block_tables"], s["cu_new"], s["kv_lens"],
                                    s["max_new"], scale=s["scale"], window=s["window"], out=s["out"], lse=s["lse"])


def _own_sample(s):
    return s["ctx"].pq_sample_tokens(s["logits"], s["noise"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                     min_p=s["min_p"], out=s["out"])


# -- the plain forms --------------------------------------------------------------------------------------------------
def _plain_plan(s):
    new, cached, table, block = s["new_lens"], s["cached_lens"], s["block_tables"], s["block"]
    width = table.shape[1]
    have, full = (cached + block - 1) // block, (cached + new + block - 1) // block
    fits = full <= width
    need = torch.where(fits, full - have, 0)
    upto = need.cumsum(0)
    served = fits & (upto <= s["free_blocks"].shape[0])
    column = torch.arange(width, device="cuda")
    fresh = served[:, None] & (column >= have[:, None]) & (column < full[:, None])
    source = (upto - need)[:, None] + column - have[:, None]
    table.copy_(torch.where(fresh, s["free_blocks"][torch.where(fresh, source, 0)], table))
    ends = new.cumsum(0)
    cu = torch.cat([ends.new_zeros(1), ends])
    request = torch.repeat_interleave(torch.arange(new.shape[0], device="cuda"), new, output_size=s["ntokens"])
    position = cached[request] + torch.arange(s["ntokens"], device="cuda") - cu[request]
    slot = table[request, position // block].long() * block + position % block
    ok = served[request]
    return (table, cu.int(), torch.where(served, cached + new, -1).int(), torch.where(ok, position, -1).int(),
            torch.where(ok, slot, -1), torch.where(served, need, 0).sum().int().reshape(1))


def _plain_turn(x, weight, s):
    """Norm and rotation of heads [t][h][dim]."""
    x = x.float()
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


def _plain_append(s):
    dtype = s["q"].dtype
    q = _plain_turn(s["q"], s["q_weight"], s).to(dtype)
    s["key_cache"].flatten(0, 1)[s["slots"]] = _plain_turn(s["k"], s["k_weight"], s).to(dtype)
    s["value_cache"].flatten(0, 1)[s["slots"]] = s["v"]
    return q, s["key_cache"], s["value_cache"]


def _plain_attention(s):
    t, hq, dim = s["q"].shape
    hkv, block = s["kv_heads"], s["block"]
    group, requests, max_new, max_kv = hq // hkv, s["requests"], s["max_new"], s["max_kv"]
    new, kv = s["cu_new"][1:] - s["cu_new"][:-1], s["kv_lens"]
    # queries padded to [request][kv head][head of the group, token][dim], keys and values to [request][kv head][key][dim]
    step = torch.arange(max_new, device="cuda")
    row = (s["cu_new"][:-1, None] + step).clamp(max=t - 1)
    q = s["q"][row].float().unflatten(2, (hkv, group)).permute(0, 2, 3, 1, 4).reshape(requests, hkv, group * max_new, dim)
    place = torch.arange(max_kv, device="cuda")
    slot = (s["block_tables"][:, place // block].long() * block + place % block).clamp(min=0)
    keys = s["key_cache"].flatten(0, 1)[slot].float().permute(0, 2, 3, 1)
    values = s["value_cache"].flatten(0, 1)[slot].float().permute(0, 2, 1, 3)
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


def _plain_sample(s):
    logits, noise = s["logits"].float(), s["noise"]
    rows, vocab = logits.shape
    temperature = s["temperature"]
    greedy = temperature <= 0
    top = logits.amax(dim=1, keepdim=True)
    x = (logits - top) / torch.where(greedy, 1, temperature)[:, None]
    weight = torch.exp(x)
    if s["top_k"] is None:
        keep = weight > 0
    else:
        order = torch.sort(logits, dim=1, descending=True, stable=True)[1]
        ranked = weight.gather(1, order)
        place = torch.arange(vocab, device="cuda")
        first = torch.where(s["top_k"] > 0, s["top_k"], vocab)[:, None]
        ranked = torch.where(place < first, ranked, 0)
        before = ranked.cumsum(1) - ranked
        p = s["top_p"][:, None]
        kept = (ranked > 0) & ((p >= 1) | (before < p * ranked.sum(1, keepdim=True))) & (ranked >= s["min_p"][:, None])
        keep = torch.zeros_like(kept).scatter(1, order, kept)
    race = torch.where(keep, x - torch.log(-torch.log(noise)), -math.inf)
    race = torch.where(greedy[:, None], logits, race)
    place = torch.arange(vocab, device="cuda")
    token = torch.where(race == race.amax(dim=1, keepdim=True), place, vocab).amin(dim=1)
    mass = torch.where(keep, weight, 0).sum(1)
    logprob = x.gather(1, token[:, None])[:, 0] - torch.log(mass)
    return token, torch.where(greedy, 0, logprob)


# -- from the definitions, in 64 bits ---------------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    return globals()["_exact_" + case["op"]](state)


def _exact_plan(s):
    new, cached = s["new_lens"].tolist(), s["cached_lens"].tolist()
    table, free, block = s["block_tables"].tolist(), s["free_blocks"].tolist(), s["block"]
    cu, kv, positions, slots, counted, taken = [0], [], [], [], 0, 0
    for r, (n, c) in enumerate(zip(new, cached)):
        have, full = -(-c // block), -(-(c + n) // block)
        need = full - have if full <= len(table[r]) else 0
        served = full <= len(table[r]) and counted + need <= len(free)
        if served:
            table[r][have:full] = free[counted:counted + need]
            taken += need
        counted += need
        kv.append(c + n if served else -1)
        for p in range(c, c + n):
            positions.append(p if served else -1)
            slots.append(table[r][p // block] * block + p % block if served else -1)
        cu.append(cu[-1] + n)
    whole = torch.int32
    return (torch.tensor(table, dtype=whole), torch.tensor(cu, dtype=whole), torch.tensor(kv, dtype=whole),
            torch.tensor(positions, dtype=whole), torch.tensor(slots, dtype=torch.int64), torch.tensor([taken], dtype=whole))


def _exact_append(s):
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
    caches = []
    for cache, fresh in ((s["key_cache"], found[1]), (s["value_cache"], s["v"].double())):
        cache = cache.double()
        cache.view(-1, *cache.shape[2:]).index_copy_(0, s["slots"], fresh)
        caches.append(cache)
    return found[0], caches[0], caches[1]


def _exact_attention(s):
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
        keys, values = (c[blocks].reshape(-1, s["kv_heads"], dim)[:n].double() for c in (s["key_cache"], s["value_cache"]))
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


def _exact_sample(s):
    """The log-probabilities of the tokens: those of the plain definition, token by token from the sorted row."""
    tokens, logprobs = [], []
    for r in range(s["rows"]):
        logits = s["logits"][r].double()
        t = float(s["temperature"][r])
        if t <= 0:
            tokens.append(int((logits == logits.max()).nonzero()[0]))
            logprobs.append(0.0)
            continue
        x = (logits - logits.max()) / t
        value, order = torch.sort(x, descending=True, stable=True)
        n = int((value > -math.inf).sum())
        if s["top_k"] is not None:
            k, p, least = int(s["top_k"][r]), float(s["top_p"][r]), float(s["min_p"][r])
            n = min(n, k) if k > 0 else n
            mass = value[:n].exp()
            if p < 1:
                n = min(n, int((mass.cumsum(0) - mass < p * mass.sum()).sum()))
            n = max(1, min(n, int((value[:n].exp() >= least).sum())))
        kept, index = value[:n], order[:n]
        race = kept - torch.log(-torch.log(s["noise"][r].double()[index]))
        best = int(race.argmax())
        tokens.append(int(index[best]))
        logprobs.append(float(kept[best] - torch.logsumexp(kept, 0)))
    return torch.tensor(tokens), torch.tensor(logprobs, dtype=torch.float64)


# -- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "plan":
        new, cached = _lengths(case)
        fresh = sum(-(-(c + n) // case["block"]) + -c // case["block"] for n, c in zip(new, cached))
        return {"bytes": 16 * len(new) + 8 * fresh + 12 * sum(new), "flops": 0}
    if op == "append":
        t, heads, dim = case["tokens"], case["q_heads"] + 2 * case["kv_heads"], case["dim"]
        return {"bytes": t * (2 * heads * dim * BYTES[case["dtype"]] + 4 * case["rot"] + 12),
                "flops": t * (case["q_heads"] + case["kv_heads"]) * (4 * dim + 3 * case["rot"])}
    if op == "attention":
        new, cached = _lengths(case)
        pairs = read = 0
        for i, (n, c) in enumerate(zip(new, cached)):
            if i == _refused(case):
                continue
            w = case["window"] or n + c
            pairs += sum(min(w, p + 1) for p in range(c, c + n))
            read += min(n + c, w + n - 1)
        e, dim = BYTES[case["dtype"]], case["dim"]
        return {"bytes": 2 * sum(new) * case["q_heads"] * dim * e + 2 * read * case["kv_heads"] * dim * e + 4 * sum(new) * case["q_heads"],
                "flops": 4 * pairs * case["q_heads"] * dim}
    noise = 4 if case["filters"] == "none" else 0   # (with filters only that of the tokens that stay)
    size = case["rows"] * case["vocab"]
    return {"bytes": size * (BYTES[case["dtype"]] + noise), "flops": 4 * size}
