"""The reading step over a cache of 8 bits and the log-probabilities of tokens at the ends of their ranges: bounds that know what of a row
counts, scales and sizes next to the limits, against the oracles in 64 bits."""
import gc

import numpy as np
import pytest
import torch

from oracle import read8_oracle as orc
from oracle import read_oracle
from paper_1712_02912_amd import binding
from test_gpu_read8 import BF16, E4M3, F16, F32, UNIT, attention_bound, dev, host, make_cache, whole

pytestmark = pytest.mark.gpu

HALF_UNIT = 2.0 ** -24   # of fp32, relative


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()
    gc.collect()


# ---- append -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype,dim,q_heads,heads,tokens", [(BF16, 128, 192, 1, 1365), (F16, 80, 192, 2, 2184), (F32, 64, 192, 1, 1365), (BF16, 512, 96, 2, 682)])
@pytest.mark.parametrize("more", [0, 1, 70])
def test_append_of_queries_about_64_mib(ctx, dtype, pairs, dim, q_heads, heads, tokens, more):
    """Up to 64 MiB of queries go with the keys and values, more of them by themselves: either way as the same tokens in two calls, with
    tokens without a position, and as the definition."""
    assert tokens * q_heads * dim * dtype.itemsize <= 64 * 2 ** 20 < (tokens + 1) * q_heads * dim * dtype.itemsize
    tokens += more
    r = np.random.default_rng(dim + more)
    gen = torch.Generator(device="cuda").manual_seed(dim + more)
    q, k, v = (torch.randn((tokens, n, dim), device="cuda", generator=gen).mul_(3).to(dtype) for n in (q_heads, heads, heads))
    positions = r.integers(0, 50, tokens).astype(np.int32)
    # requests of 1 to 300 tokens, each from the beginning of a block on
    slots, at = np.empty(tokens, np.int64), 0
    begins = []
    while at < tokens:
        n = min(tokens - at, int(r.integers(1, 301)))
        begins.append(at)
        slots[at:at + n] = (max(slots[:at], default=-16) // 16 + 1) * 16 + np.arange(n)
        at += n
    cut = begins[len(begins) // 2]
    unplaced = np.array([begins[1], begins[2], cut, tokens]) - 1   # (the last tokens of requests: a run ends before them)
    positions[unplaced] = [-1, 50, 2 ** 31 - 1, -2 ** 31]
    blocks = int(slots.max()) // 16 + 1
    rot = dim // 2
    angle = r.uniform(-3, 3, (50, rot // 2))
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    qw, kw = (r.uniform(0.5, 2, dim).astype(np.float32) for _ in range(2))

    def append(parts):
        cache = [torch.full((blocks, 16, heads, dim), 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
        scales = [torch.full((blocks, heads), float("nan"), device="cuda") for _ in range(2)]
        out = torch.full((tokens, q_heads, dim), 7.0, dtype=dtype, device="cuda")
        for a, b in parts:
            ctx.pq_kv_append8(q[a:b], k[a:b], v[a:b], dev(positions[a:b]), dev(slots[a:b]), *cache, *scales, dev(cos), dev(sin), q_weight=dev(qw),
                              k_weight=dev(kw), pairs=pairs, out=out[a:b])
        return [out] + [c.view(torch.uint8) for c in cache] + [s.view(torch.int32) for s in scales]

    whole_call, halves = append([(0, tokens)]), append([(0, cut), (cut, tokens)])
    assert all(torch.equal(a, b) for a, b in zip(whole_call, halves))
    # of the queries some tokens, against the definition
    some = np.unique(np.concatenate([unplaced, [1, tokens - 1], r.integers(0, tokens, 5)]))
    p = np.where((positions >= 0) & (positions < 50), positions, 0)
    want = read_oracle.turn(host(q[some]), p[some], cos, sin, qw, 1e-6, True, pairs)
    size = np.abs(read_oracle.turn(host(q[some]), p[some], None, None, qw, 1e-6, True, pairs)).max(axis=2, keepdims=True)
    placed = ~np.isin(some, unplaced)[:, None, None]
    bound = UNIT[dtype] * np.abs(want) * 1.01 + (8 + dim / 64) * HALF_UNIT * 2 * size + 2.0 ** -25 * (dtype == F16)
    assert (np.abs(host(whole_call[0][some]) - np.where(placed, want, 0)) <= np.where(placed, bound, 0)).all()
    # codes and scales, all of them
    keys = read_oracle.turn(host(k), p, cos, sin, kw, float(np.float32(1e-6)), True, pairs).astype(np.float32)
    for rows, codes, scale in zip((keys, host(v)), whole_call[1:3], whole_call[3:]):
        values, held = np.full((blocks, 16, heads, dim), np.nan), np.full((blocks, heads), np.nan)
        orc.store(values, held, rows, slots, ~np.isin(np.arange(tokens), unplaced))
        assert np.array_equal(host(scale.view(F32)), held, equal_nan=True) and np.array_equal(host(codes.view(E4M3)), values, equal_nan=True)


# ---- attention --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype,dim", [(F32, 64), (F32, 80), (BF16, 64), (BF16, 80)])
def test_attention_of_keys_of_the_least_scale(ctx, new, dtype, dim):
    """Large queries and small keys: products of a query with the keys' codes alone would leave fp32."""
    r = np.random.default_rng(new)
    tables, kc, vc, _, vs, keys, values = make_cache(r, [new + 77, new], 2, dim, 16, 0)
    ks = torch.full_like(vs, 2.0 ** -126)
    keys = host(kc) * 2.0 ** -126
    q = dev(r.standard_normal((2 * new, 4, dim)) * 1e37, dtype)
    scale, cu, kv = 0.1 * dim ** -0.5, np.array([0, new, 2 * new]), np.array([new + 77, new])
    out, lse = ctx.pq_kv_attention8(q, kc, vc, ks, vs, dev(tables), whole(cu), whole(kv), new, scale=scale)
    want, want_lse, spread = read_oracle.attention(host(q), keys, values, tables, cu, kv, scale, 0)
    bound, fp32 = attention_bound(dtype, host(q), keys, spread, want, scale, 0, dim)
    assert (np.abs(host(out) - want) <= bound).all()
    assert (np.abs(host(lse) - want_lse) <= 2 * fp32 + 1e-6 * np.abs(want_lse)).all()


@pytest.mark.parametrize("dtype,dim", [(F32, 64), (F32, 80), (BF16, 80)])
def test_attention_adds_up_small_weights_of_a_small_scale(ctx, dtype, dim):
    """One key of a large weight and value 0, thousands of exp(-18) of it whose values are 256 times 2^-120: a weight times the scale alone has
    three bits left in fp32."""
    count, scale = 8191, 2.0 ** -120
    tables = np.arange(512, dtype=np.int32)[None]
    keys, values = (np.zeros((512, 16, 1, dim)) for _ in range(2))
    keys.reshape(-1, dim)[1:, 0], values.reshape(-1, dim)[1:] = -18.0, 256.0
    q = np.zeros((1, 1, dim))
    q[0, 0, 0] = 1.0
    ones, small = torch.ones((512, 1), device="cuda"), torch.full((512, 1), scale, device="cuda")
    out, _ = ctx.pq_kv_attention8(dev(q, dtype), dev(keys, F32).to(E4M3), dev(values, F32).to(E4M3), ones, small, dev(tables), whole([0, 1]), whole([8192]),
                                  1, scale=1.0)
    term = np.exp(-18.0) * 256 * scale
    want = count * term / (1 + count * np.exp(-18.0))
    # each addition of a term is off by half a unit of the sum, or half of fp32's least step; rounding of the result
    assert (np.abs(host(out) - want) <= want * (8192 * HALF_UNIT + 2.0 ** -150 / term + (2.0 ** -8 if dtype == BF16 else 0.0))).all()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("requests", [2 ** 24 - 2, 2 ** 24 - 2 ** 19])
def test_attention_of_as_many_requests_as_a_launch_takes(ctx, eight, requests):
    """Chunks of so many requests, all but one of them empty: 2^32 threads are not passed, so the rows are written."""
    new, dim, heads = 40, 64, 1
    r = np.random.default_rng(1)
    tables, *cache, keys, values = make_cache(r, [new + 9], heads, dim, 16)
    q = dev(r.standard_normal((new, 2, dim)), BF16)
    if not eight:
        cache = [dev(np.nan_to_num(x), BF16) for x in (keys, values)]
        keys, values = (host(x) for x in cache)
    cu = torch.zeros(requests + 1, dtype=torch.int32, device="cuda")
    cu[-1] = new
    kv = torch.zeros(requests, dtype=torch.int32, device="cuda")
    kv[-1] = new + 9
    table = torch.full((requests, tables.shape[1]), -1, dtype=torch.int32, device="cuda")
    table[-1] = dev(tables[0])
    out, lse = (ctx.pq_kv_attention8 if eight else ctx.pq_kv_attention)(q, *cache, table, cu, kv, new)
    want, want_lse, spread = read_oracle.attention(host(q), keys, values, tables, np.array([0, new]), np.array([new + 9]), dim ** -0.5, 0)
    bound, fp32 = attention_bound(BF16, host(q), np.nan_to_num(keys), spread, want, dim ** -0.5, new + 9, dim)
    assert (np.abs(host(out) - want) <= bound).all() and (np.abs(host(lse) - want_lse) <= 2 * fp32 + 1e-6 * np.abs(want_lse)).all()


# ---- log-probabilities ------------------------------------------------------------------------------------------------
def least_time(f, calls=3, tries=5):
    """Milliseconds of a call, the least of some tries."""
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    found = []
    for _ in range(tries + 1):   # (the first one loads the kernel)
        begin.record()
        for _ in range(calls):
            f()
        end.record()
        torch.cuda.synchronize()
        found.append(begin.elapsed_time(end) / calls)
    return min(found[1:])


@pytest.mark.parametrize("dtype,mask", [(F16, -65504.0), (BF16, -9984.0), (F32, -1e4)])
def test_logprobs_of_masked_rows_take_no_pass_for_each_token(ctx, dtype, mask):
    """Twenty logits, all different, over 131 052 equal ones take as long where the equal ones are negative as where they are zero: what is
    above the limit is listed by one pass.  (A pass for each of the twenty would be ten times the whole call.)"""
    r = np.random.default_rng(1)
    found = []
    for rest in (mask, 0.0):
        l = np.full((512, 131072), rest, np.float32)
        for row in l:
            row[r.permutation(131072)[:20]] = 1 + np.arange(20) / 16
        logits = dev(l, dtype)
        first, lp = (host(x)[::101] for x in ctx.pq_token_logprobs(logits, top=50)[3:])
        for i, row in enumerate(host(logits[::101])):
            _, _, _, want, want_lp = orc.logprobs(row, 0, 50)
            assert np.array_equal(first[i], want) and (np.abs(lp[i] - want_lp) <= 3e-6 * (1 + np.abs(want_lp))).all()
        found.append(least_time(lambda: ctx.pq_token_logprobs(logits, top=50)))
    assert found[0] <= 2.5 * found[1], found


def check_closely(ctx, logits, tokens, top, rows=None):
    """As the definition has it, with bounds that masks and the size of a row's logits do not widen.

    A row's sum S of weights w = exp(-d), d = distance from the largest, and M of d w: terms are off by 2 + d units (power, distance), chains
    of up to n additions by n.  n: 64 and one for each 4096 logits; rows whose largest is beyond 2^19 are summed in more bits.  So log S is off by
    n + 2 + D, D = M / S the mean distance, and M / S by (2 n + 4) D + D2, D2 the mean square; then come roundings of what is
    put together."""
    lp, ranks, entropy, first, top_lp = (None if x is None else host(x) for x in ctx.pq_token_logprobs(logits, whole(tokens, np.int64), top))
    for r in range(len(tokens)) if rows is None else rows:
        l = host(logits[r])
        want_lp, rank, want_entropy, want_first, want_top = orc.logprobs(l, int(tokens[r]), top)
        assert ranks[r] == rank and np.array_equal(first[r], want_first), r
        high = l[~np.isnan(l)].max()
        d = high - l[l >= high - 200]
        w = np.exp(-d)
        mean, square = (w @ d) / w.sum(), (w @ d ** 2) / w.sum()
        n = 4 if abs(high) >= 2 ** 19 else 64 + len(l) / 4096
        sure = n + 4 + mean + 2 * np.log(w.sum())
        assert lp[r] == want_lp or abs(lp[r] - want_lp) <= HALF_UNIT * (sure + 2 * abs(want_lp)), (r, lp[r], want_lp)
        assert abs(entropy[r] - want_entropy) <= HALF_UNIT * (sure + (2 * n + 4) * mean + square + 2 * want_entropy), (r, entropy[r], want_entropy)
        some = np.isfinite(want_top)
        assert np.array_equal(top_lp[r][~some], want_top[~some])
        assert (np.abs(top_lp[r][some] - want_top[some]) <= HALF_UNIT * (sure + 2 * np.abs(want_top[some]))).all(), r


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("vocab", [9, 3000, 40000, 2 ** 20 - 1])
@pytest.mark.parametrize("base", [21.0, -300.0, 30003.0, -500000.0])
def test_logprobs_of_rows_away_from_zero(ctx, rows, vocab, base):
    """One logit over equal ones, and logits of all distances, away from zero: as exact as rows next to it."""
    r = np.random.default_rng(vocab)
    for low in (np.full(vocab, 9.875), np.full(vocab, 2.375), r.integers(0, 200, vocab) / 8):
        l = base - low
        l[vocab // 2] = base
        logits = dev(l[None], F32).expand(rows, vocab)
        check_closely(ctx, logits, np.full(rows, vocab - 1), 3, rows=[0, rows - 1])


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("vocab", [9, 3000, 40000, 2 ** 20 - 1])
@pytest.mark.parametrize("base", [2.0 ** 20, -2.0 ** 20 + 64, 2.0 ** 19, -2.0 ** 19 - 8])
def test_logprobs_of_rows_far_from_zero(ctx, rows, vocab, base):
    """The same a million from zero, where rows are summed a second time."""
    test_logprobs_of_rows_away_from_zero(ctx, rows, vocab, base)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [7, 600, 40000])
@pytest.mark.parametrize("mask", [-3e4, -6e5, -1.1e6, -1e9, -1e30, -3e38])
def test_logprobs_of_logits_beside_a_mask(ctx, dtype, vocab, mask):
    """A mask's size, which the results do not depend on, is not in the bounds either."""
    if dtype == F16:
        mask = max(mask, -65504.0)
    r = np.random.default_rng(vocab)
    l = r.standard_normal((6, vocab)) * 3
    l[0, : vocab // 2] = mask
    l[1, vocab // 3:] = mask
    l[2, r.random(vocab) < 0.9] = mask
    l[3, r.random(vocab) < 0.5] = -np.inf
    l[3, r.random(vocab) < 0.5] = mask
    l[4] += 100
    l[4, ::2] = mask
    l[5, 1:] = mask
    logits = dev(l, dtype)
    for tokens in ([0, vocab - 1, 3, 5, 1, 0], [vocab - 1, 0, 1, 2, 3, 1]):
        check_closely(ctx, logits, tokens, 5)
