"""The reading step over a cache of 8 bits, and the log-probabilities of tokens (include/pq_read.h), against their oracles in 64 bits."""
import gc

import numpy as np
import pytest
import torch

from oracle import read8_oracle as orc
from oracle import read_oracle
from paper_1712_02912_amd import binding

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}   # half a unit in the last place, relative


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()
    gc.collect()   # tensors that errors' frames hold: later tests watch the memory that is allocated


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    """Values of a tensor in double (whole numbers as they are)."""
    if t.dtype == E4M3:
        return orc.numbers()[t.contiguous().view(torch.uint8).cpu().numpy()]
    return (t.double() if t.is_floating_point() else t).cpu().numpy()


def whole(x, dtype=np.int32):
    return dev(np.asarray(x, dtype))


def laid_out(x, layout):
    """A cache [blocks][block size][heads][dim] of 8 bits with other strides."""
    if layout == "heads first":
        return x.view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(E4M3)
    if layout == "odd":                  # rows that begin at odd bytes
        wide = torch.zeros(x.shape[:-1] + (x.shape[-1] + 1,), dtype=torch.uint8, device="cuda")
        wide[..., 1:] = x.view(torch.uint8)
        return wide[..., 1:].view(E4M3)
    return x


# ---- append -----------------------------------------------------------------------------------------------------------
def chunks(r, tokens, requests, block_size, pool):
    """Slots of requests' tokens, one request after the other, each from a place within its first block on."""
    cuts = np.concatenate([[0], np.sort(r.choice(np.arange(1, tokens), requests - 1, replace=False)), [tokens]]) if requests > 1 else np.array([0, tokens])
    slots, at = [], 0
    for n in np.diff(cuts):
        place = r.integers(0, block_size) + np.arange(n)
        slots.append(pool[at + place // block_size].astype(np.int64) * block_size + place % block_size)
        at += int(place[-1]) // block_size + 1
    return np.concatenate(slots)


def check_append(ctx, tokens, requests, q_heads, heads, dim, rot, pairs, dtype, norm=True, weights=True, layout="plain", block_size=16, eps=1e-6,
                 gain=3.0, seed=0, spoil=True):
    r = np.random.default_rng(seed)
    sizes = gain * 2.0 ** r.integers(-3, 4, (tokens, 1, 1))      # rows of all sizes: scales grow within blocks
    qkv = dev(r.standard_normal((tokens, q_heads + 2 * heads, dim)) * sizes, dtype)
    if layout == "odd":
        wide = torch.zeros((tokens, q_heads + 2 * heads, dim + 3), dtype=dtype, device="cuda")
        wide[:, :, 1:dim + 1] = qkv
        qkv = wide[:, :, 1:dim + 1]
    q, k, v = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
    blocks = sum(-(-(block_size + n) // block_size) for n in [tokens]) + 2 * requests + 1
    pool = r.permutation(blocks)
    slots = chunks(r, tokens, requests, block_size, pool)
    caches, scales = [], []
    for _ in range(2):
        caches.append(laid_out(dev(r.integers(0, 127, (blocks, block_size, heads, dim)).astype(np.uint8)).view(E4M3), layout))
        scales.append(dev(2.0 ** r.integers(-9, -3, (blocks, heads)), F32))
    positions = r.integers(0, 50, tokens).astype(np.int32)
    runs = orc.runs(slots, block_size, np.ones(tokens, bool))
    if spoil and len(runs) >= 5:         # ends of runs without a position, with one behind the tables, without a slot, with one behind the cache
        ends = [slice(t + r.integers(0, n), t + n) for t, n in (runs[i] for i in r.choice(len(runs), 4, replace=False))]
        positions[ends[0]], positions[ends[1]], slots[ends[2]], slots[ends[3]] = -1, 50, -1, blocks * block_size
    angle = r.uniform(-3, 3, (50, rot // 2))
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    qw, kw = (r.uniform(0.5, 2, dim).astype(np.float32) if norm and weights else None for _ in range(2))
    before = [(host(c), host(s)) for c, s in zip(caches, scales)]
    out = ctx.pq_kv_append8(q if q_heads else None, k, v, dev(positions), dev(slots), *caches, *scales, dev(cos) if rot else None,
                            dev(sin) if rot else None, q_weight=None if qw is None else dev(qw), k_weight=None if kw is None else dev(kw),
                            eps=eps, norm=norm, pairs=pairs)
    placed = (positions >= 0) & ((positions < 50) if rot else True)
    p = np.where(placed, positions, 0)
    written = placed & (slots >= 0) & (slots < blocks * block_size)
    tables = (cos, sin) if rot else (None, None)
    if q_heads:
        want = read_oracle.turn(host(q), p, *tables, qw, eps, norm, pairs)
        # rounding of the result, and the fp32 steps before it (sum of squares, root, weight, two products and their sum, each in
        # proportion to the size of a pair, at most twice the larger of the two)
        size = np.abs(read_oracle.turn(host(q), p, None, None, qw, eps, norm, pairs)).max(axis=2, keepdims=True)
        bound = UNIT[dtype] * np.abs(want) * 1.01 + (8 + dim / 64) * 2.0 ** -24 * 2 * size + 2.0 ** -25 * (dtype == F16)
        assert (np.abs(host(out) - np.where(placed[:, None, None], want, 0)) <= np.where(placed[:, None, None], bound, 0)).all()
    else:
        assert out is None
    keys = read_oracle.turn(host(k), p, *tables, kw, float(np.float32(eps)), norm, pairs).astype(np.float32)
    for rows, cache, scale, (values, held) in zip((keys, host(v)), caches, scales, before):
        orc.store(values, held, rows, slots, written)
        # (keys are computed in 64 bits on both sides: nothing is left that a border could turn)
        assert np.array_equal(host(scale), held)
        assert np.array_equal(host(cache), values, equal_nan=True)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (64, 32), (80, 32), (96, 96), (256, 64), (2, 2), (10, 6), (512, 512), (130, 0), (1024, 26)])
def test_append(ctx, dtype, pairs, dim, rot):
    check_append(ctx, 61, 4, 5, 2, dim, rot, pairs, dtype, seed=dim)


@pytest.mark.parametrize("block_size", [1, 3, 8, 16, 24, 64, 100, 256])
@pytest.mark.parametrize("tokens,requests", [(1, 1), (9, 9), (333, 3), (700, 1)])
def test_append_block_sizes(ctx, block_size, tokens, requests):
    check_append(ctx, tokens, requests, 4, 2, 128, 128, False, BF16, block_size=block_size, seed=block_size + tokens)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128, 256, 512])
def test_append_of_large_blocks(ctx, dtype, dim):
    check_append(ctx, 900, 2, 2, 1, dim, dim, False, dtype, block_size=400, seed=dim)


@pytest.mark.parametrize("dim,heads", [(64, 40), (128, 24), (256, 12), (512, 8)])
def test_append_of_many_heads_of_large_blocks(ctx, dim, heads):
    check_append(ctx, 1900, 3, 2, heads, dim, dim, False, BF16, block_size=400, seed=dim)


@pytest.mark.parametrize("tokens,requests", [(1, 1), (6, 6), (1031, 300), (9000, 11)])
def test_append_of_many_tokens(ctx, tokens, requests):
    check_append(ctx, tokens, requests, 8, 2, 64, 64, False, BF16, block_size=24, seed=tokens)


@pytest.mark.parametrize("layout", ["odd", "heads first"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_append_layouts(ctx, dtype, layout):
    check_append(ctx, 39, 3, 4, 4, 128, 64, False, dtype, layout=layout)


def test_append_without_norm_weights_queries(ctx):
    check_append(ctx, 39, 3, 4, 2, 64, 64, False, BF16, norm=False)
    check_append(ctx, 39, 3, 4, 2, 64, 64, True, F32, weights=False)
    check_append(ctx, 39, 3, 0, 2, 64, 64, False, F16)
    check_append(ctx, 39, 3, 3, 1, 64, 0, False, F32, norm=False)


@pytest.mark.parametrize("dim", [64, 80, 128])
def test_append_step_by_step(ctx, dim):
    """Tokens that come one by one, and in chunks, to the same blocks: the scale is that of the largest so far, and what was there is kept."""
    r = np.random.default_rng(dim)
    caches = [torch.full((3, 16, 2, dim), 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
    scales = [torch.full((3, 2), float("nan"), device="cuda") for _ in range(2)]
    values, held = [host(c) for c in caches], [np.full((3, 2), 1.0) for _ in range(2)]
    at = 0
    for n in [1, 1, 3, 1, 11, 1, 5, 16, 9]:
        x = dev(r.standard_normal((n, 4, dim)) * 10 * r.random(), F32)
        slots = np.arange(at, at + n)
        ctx.pq_kv_append8(None, x[:, :2], x[:, 2:], whole(np.zeros(n)), dev(slots), *caches, *scales, norm=False)
        for i in range(2):
            orc.store(values[i], held[i], host(x)[:, 2 * i:2 * i + 2], slots, np.ones(n, bool))
            touched = -(-(at + n) // 16)
            assert np.array_equal(host(scales[i])[:touched], held[i][:touched]) and np.isnan(host(scales[i])[touched:]).all()
            assert np.array_equal(host(caches[i]), values[i], equal_nan=True)
        at += n


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [64, 10])
def test_append_of_special_values(ctx, dtype, dim):
    """Zeros, the largest and smallest numbers, infinities and NaN, each in a block of its own."""
    largest = torch.finfo(dtype).max
    rows = [np.zeros((4, dim)), np.full((4, dim), largest), np.full((4, dim), float(torch.finfo(dtype).tiny)), np.full((4, dim), 448.0), np.full((4, dim), 1.0)]
    rows[3][2, 1], rows[3][3, 0] = 449.0 if dtype == F32 else 450.0, -np.inf
    rows[4][0], rows[4][1, 3], rows[4][2, 2] = np.nan, np.inf, np.nan
    x = dev(np.stack(rows).reshape(20, 1, dim), dtype)
    caches = [torch.zeros((6, 4, 1, dim), dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
    scales = [torch.zeros((6, 1), device="cuda") for _ in range(2)]
    slots = np.arange(4, 24)
    ctx.pq_kv_append8(None, x, x, whole(np.zeros(20)), dev(slots), *caches, *scales, norm=False)
    values, held = np.zeros((6, 4, 1, dim)), np.zeros((6, 1))
    orc.store(values, held, host(x), slots, np.ones(20, bool))
    for cache, scale in zip(caches, scales):
        assert np.array_equal(host(scale), held) and np.array_equal(host(cache), values, equal_nan=True)
    assert held[1, 0] == 2.0 ** -126 and np.isnan(values[5]).sum() == dim + 1


@pytest.mark.parametrize("dim", [64, 80, 10])
def test_append_counts_the_exponents_of_scales(ctx, dim):
    """A block's scale from before that is no power of two is taken as the one below; a run that keeps it writes that."""
    x = dev(np.random.default_rng(dim).standard_normal((2, 1, dim)), F32)
    found = []
    for scale in (4.0, 7.9):
        caches = [torch.full((1, 16, 1, dim), 0x51, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
        scales = [torch.full((1, 1), scale, device="cuda") for _ in range(2)]
        ctx.pq_kv_append8(None, x, x, whole([0, 0]), dev(np.array([3, 4])), *caches, *scales, norm=False)
        assert all(float(s) == 4.0 for s in scales)
        found.append([host(c) for c in caches])
    assert np.array_equal(found[0], found[1])


@pytest.mark.parametrize("dim", [64, 10])
def test_append_of_rows_without_a_size(ctx, dim):
    """Keys of zeros under a norm: zeros with eps, no numbers without it; values are not touched by that."""
    x = torch.zeros((2, 1, dim), device="cuda")
    for eps in (1e-6, 0.0):
        caches = [torch.full((1, 4, 1, dim), 0x51, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
        scales = [torch.ones((1, 1), device="cuda") for _ in range(2)]
        ctx.pq_kv_append8(None, x, x, whole([0, 0]), dev(np.array([0, 1])), *caches, *scales, eps=eps)
        assert np.array_equal(np.isnan(host(caches[0])[0, :2]), np.full((2, 1, dim), eps == 0)) and (host(caches[1])[0, :2] == 0).all()
        assert all(float(s) == 2.0 ** -126 for s in scales) and (host(caches[0])[0, 2:] == 9.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens", [1100, 20000])
def test_append_of_single_tokens_of_many_requests(ctx, dtype, tokens):
    check_append(ctx, tokens, tokens, 2, 2, 64, 64, False, dtype, block_size=4, seed=tokens)


def test_append_refusals(ctx):
    x = torch.zeros((4, 2, 64), device="cuda")
    cache, scales = torch.zeros((2, 4, 2, 64), dtype=torch.uint8, device="cuda").view(E4M3), torch.ones((2, 2), device="cuda")
    rest = (torch.zeros(4, dtype=torch.int32, device="cuda"), torch.arange(4, device="cuda"), cache, cache, scales, scales)
    table = torch.zeros((8, 40), device="cuda")
    for bad in (dict(cos=table, sin=table), dict(eps=-1.0)):
        with pytest.raises(binding.PqError, match="kv_append8"):
            ctx.pq_kv_append8(x, x, x, *rest, **bad)
    odd, odd_cache = torch.zeros((4, 2, 63), device="cuda"), cache[..., :63]
    with pytest.raises(binding.PqError) as e:
        ctx.pq_kv_append8(odd, odd, odd, *rest[:2], odd_cache, odd_cache, scales, scales)
    assert e.value.code == -3
    for bad in (cache.view(torch.uint8), cache.float()):
        with pytest.raises(TypeError):
            ctx.pq_kv_append8(x, x, x, *rest[:2], bad, bad, scales, scales)
    with pytest.raises(TypeError):
        ctx.pq_kv_append8(x.half(), x, x, *rest)
    with pytest.raises(TypeError):
        ctx.pq_kv_append8(x.double(), x.double(), x.double(), *rest)
    with pytest.raises(TypeError):
        ctx.pq_kv_append8(x, x, x, *rest[:4], scales.double(), scales)
    for bad in (scales[:1], scales[:, :1], scales.T):
        with pytest.raises(ValueError):
            ctx.pq_kv_append8(x, x, x, *rest[:5], bad if bad is not scales.T else torch.ones((2, 4), device="cuda")[:, ::2])
    with pytest.raises(ValueError):
        ctx.pq_kv_append8(x, x, x, *rest, cos=table)
    assert bool((cache.view(torch.uint8) == 0).all()) and bool((scales == 1).all())


# ---- attention --------------------------------------------------------------------------------------------------------
def attention_bound(dtype, q, keys, spread, out, scale, most, dim):
    """Rounding of the result, of the weights to 16 bits, and of the fp32 products, sums and powers: scores are sums of
    dim products, off by up to dim units of their terms' sizes, and a weight's relative error is its score's absolute one."""
    u = UNIT[dtype]
    size = np.abs(q).max() * np.abs(keys[np.isfinite(keys)]).max(initial=0.0) * scale * dim ** 0.5 * 4
    fp32 = 2.0 ** -24 * (4 * dim ** 0.5 * max(1.0, size) + 64)
    # (f16 weights below 2^-14 are rounded to multiples of 2^-24)
    return u * np.abs(out) * 1.01 + (u * (dtype != F32) + fp32) * 2 * spread + (2.0 ** -24 * most if dtype == F16 else 0.0), fp32


def make_cache(r, kv, heads, dim, block_size, fill=0x7f, layout="plain"):
    """A cache with the requests' blocks in no order; places that hold no key have the code `fill`, blocks that hold none NaN as scales.
    Returns (tables, key codes, value codes, key scales, value scales, keys, values), the last two in double."""
    counts = [-(-max(k, 0) // block_size) for k in kv]
    width = max(counts + [1]) + 1
    total = sum(counts) + 2
    pool = r.permutation(total).astype(np.int32)
    tables = np.full((len(kv), width), -1, np.int32)
    held, at = np.zeros((total, block_size), bool), 0
    for i, (k, n) in enumerate(zip(kv, counts)):
        tables[i, :n] = pool[at:at + n]
        at += n
        j = np.arange(max(k, 0))
        held[tables[i, j // block_size], j % block_size] = True
    codes, scales, values = [], [], []
    for shift in (0.0, 0.5):
        x = (r.standard_normal((total, block_size, heads, dim)) + shift) * 2.0 ** r.integers(-2, 3, (total, 1, heads, 1))
        s = np.vectorize(orc.scale_for)(np.abs(x).max(axis=(1, 3))) if total else np.ones((total, heads))
        code = dev((x / s[:, None, :, None]).astype(np.float32)).to(E4M3).view(torch.uint8)
        code[~dev(held)] = fill
        s[~held.any(axis=1)] = np.nan
        codes.append(laid_out(code.view(E4M3), layout))
        scales.append(dev(s, F32))
        values.append(host(code.view(E4M3)) * s[:, None, :, None])
    return tables, *codes, *scales, *values


def check_attention(ctx, new, kv, q_heads, heads, dim, dtype, block_size=16, window=0, fill=0x7f, layout="plain", gain=1.0, seed=0,
                    extra=0, scale=None, max_new=None):
    r = np.random.default_rng(seed)
    tables, *cache, keys, values = make_cache(r, kv, heads, dim, block_size, fill, layout)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = int(cu[-1]) + extra
    q = dev(r.standard_normal((t, q_heads, dim)) * gain, dtype)
    if layout == "odd":
        wide = torch.zeros((t, q_heads, dim + 1), dtype=dtype, device="cuda")
        wide[..., 1:] = q
        q = wide[..., 1:]
    kv = np.array(kv, np.int32)
    out = torch.full((t, q_heads, dim), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((t, q_heads), 7.0, device="cuda")
    ctx.pq_kv_attention8(q, *cache, dev(tables), dev(cu), dev(kv), max(new) if max_new is None else max_new, scale=scale, window=window,
                         out=out, lse=lse)
    scale = dim ** -0.5 if scale is None else scale
    want, want_lse, spread = read_oracle.attention(host(q), keys, values, tables, cu, kv, scale, window)
    got, got_lse = host(out), host(lse)
    end = int(cu[-1])
    assert (got[end:] == 7).all() and (got_lse[end:] == 7).all()
    if end == 0:
        return
    got, got_lse, want, want_lse, spread = got[:end], got_lse[:end], want[:end], want_lse[:end], spread[:end]
    empty = np.isneginf(want_lse)
    assert np.array_equal(empty, np.isneginf(got_lse)) and (got[empty] == 0).all()
    bound, fp32 = attention_bound(dtype, host(q), keys, spread, want, abs(scale), max(1, kv.max()), dim)
    assert (np.abs(got - want) <= bound).all(), np.nanmax(np.abs((got - want) / bound))
    assert (np.abs(got_lse - want_lse)[~empty] <= 2 * fp32 + 1e-6 * np.abs(want_lse[~empty])).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [64, 96, 128, 256, 80, 2, 512])
def test_attention_of_single_tokens(ctx, dtype, dim):
    check_attention(ctx, [1] * 7, [1, 2, 31, 64, 65, 300, 1], 8, 2, dim, dtype, seed=dim)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [64, 96, 128, 256, 80])
def test_attention_of_chunks(ctx, dtype, dim):
    check_attention(ctx, [33, 1, 70, 5], [33, 200, 129, 64], 4, 2, dim, dtype, seed=dim)


@pytest.mark.parametrize("q_heads,heads", [(1, 1), (3, 3), (6, 2), (7, 1), (16, 2), (24, 1), (40, 1)])
@pytest.mark.parametrize("new", [1, 2, 3, 19])
def test_attention_head_layouts(ctx, q_heads, heads, new):
    check_attention(ctx, [new, 1, new], [new, 90, 150], q_heads, heads, 64, BF16, seed=q_heads + new)


@pytest.mark.parametrize("block_size", [1, 3, 8, 16, 24, 64, 100])
@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_pages(ctx, block_size, new, dtype):
    check_attention(ctx, [new, 1, new], [new + 60, 131, new + 190], 4, 2, 128, dtype, block_size=block_size, seed=block_size)


@pytest.mark.parametrize("window", [1, 2, 17, 64, 65, 200, 100000, 2 ** 31 - 1])
@pytest.mark.parametrize("new", [1, 90])
def test_attention_windows(ctx, window, new):
    check_attention(ctx, [new, 1, new], [new, 131, new + 190], 4, 2, 64, BF16, window=window, seed=window % 1000)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_rows_that_see_nothing(ctx, new, dtype):
    """Refused requests, empty ones, and lengths below the number of new tokens, whose first rows see nothing."""
    check_attention(ctx, [new, new, 0, new, new], [-1, new + 5, 9, 0, new - 1 if new > 1 else 7], 4, 2, 64, dtype, extra=3)
    check_attention(ctx, [new], [-1], 4, 2, 128, dtype)
    check_attention(ctx, [0, 0], [5, 0], 4, 2, 128, dtype, extra=2, max_new=1)


@pytest.mark.parametrize("layout", ["heads first", "odd"])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_layouts(ctx, layout, new, dtype):
    check_attention(ctx, [new, 2], [new + 100, 77], 8, 2, 128, dtype, layout=layout)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("fill", [0x7f, 0xff, 0x7e, 0])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_ignores_what_no_row_sees(ctx, new, dtype, fill, dim):
    """Not to the last bits: NaN, the largest code or zero in places that hold no key give one result."""
    found = []
    for code in (fill, 0):
        r = np.random.default_rng(dim)
        tables, *cache, keys, values = make_cache(r, [new, 33 + new, 1], 1, dim, 64, code)
        q = dev(np.random.default_rng(1).standard_normal((2 * new + 1, 4, dim)), dtype)
        found.append(ctx.pq_kv_attention8(q, *cache, dev(tables), whole([0, new, 2 * new, 2 * new + 1]), whole([new, 33 + new, 1]), new))
    assert all(torch.equal(a, b) for a, b in zip(*found))
    check_attention(ctx, [new, new, 1], [new, 33 + new, 1], 4, 1, dim, dtype, block_size=64, fill=fill)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new,window", [(3, 0), (3, 20), (70, 0), (70, 40), (300, 0), (300, 130)])
def test_attention_of_numbers_that_are_none(ctx, dtype, dim, new, window):
    """Keys and values of NaN reach the rows that see them, and no other row of their chunk."""
    r = np.random.default_rng(new + dim)
    kv = [new + 150, new]
    tables, *cache, keys, values = make_cache(r, kv, 2, dim, 16)

    def spoil(which, request, j, head, d):
        at = int(tables[request, j // 16]), j % 16, head, d
        cache[which].view(torch.uint8)[at] = 0x7f if d % 2 else 0xff
        (keys, values)[which][at] = np.nan
    spoil(1, 0, kv[0] - 2, 0, 3)
    spoil(1, 0, kv[0] - new + 1, 1, dim - 1)
    spoil(1, 0, 149, 0, 40)
    spoil(0, 1, new - 1, 1, 5)
    spoil(0, 0, kv[0] - 1, 0, 8)
    cu = np.array([0, new, 2 * new], np.int32)
    q = dev(r.standard_normal((2 * new, 4, dim)), dtype)
    out, lse = ctx.pq_kv_attention8(q, *cache, dev(tables), dev(cu), whole(kv), new, window=window)
    with np.errstate(invalid="ignore"):
        want, want_lse, spread = read_oracle.attention(host(q), keys, values, tables, cu, np.array(kv), dim ** -0.5, window)
    got, got_lse = host(out), host(lse)
    fine = np.isfinite(want)
    assert fine.mean() > 0.5 and not fine.all()
    assert np.array_equal(np.isfinite(got), fine) and np.array_equal(np.isfinite(got_lse), np.isfinite(want_lse))
    bound, fp32 = attention_bound(dtype, host(q), keys, spread, want, dim ** -0.5, max(kv), dim)
    assert (np.abs(got - want)[fine] <= bound[fine]).all()
    sure = np.isfinite(want_lse)
    assert (np.abs(got_lse - want_lse)[sure] <= 2 * fp32 + 1e-6 * np.abs(want_lse[sure])).all()


@pytest.mark.parametrize("new", [1, 33])
def test_attention_of_sharp_scores(ctx, new):
    """Scores of some hundreds: one key takes all the weight, and running maxima jump."""
    check_attention(ctx, [new, 1], [new + 500, 400], 4, 2, 64, BF16, gain=30.0)
    check_attention(ctx, [new, 1], [new + 500, 400], 4, 2, 64, F16, gain=30.0)
    check_attention(ctx, [new, 1], [new + 500, 400], 4, 2, 64, BF16, scale=0.0)
    check_attention(ctx, [new, 1], [new + 500, 400], 4, 2, 64, F16, scale=-0.2)


@pytest.mark.parametrize("new", [1, 4, 130])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_of_long_contexts(ctx, new, dtype):
    check_attention(ctx, [new, 1, new], [9000 + new, 5000, 301 + new], 4, 1, 128, dtype, block_size=48, seed=new)


def test_attention_of_many_requests(ctx):
    r = np.random.default_rng(5)
    kv = r.integers(1, 40, 2500)
    check_attention(ctx, [1] * 2500, kv.tolist(), 2, 1, 64, BF16)
    new = np.minimum(r.integers(0, 4, 600), 3)
    check_attention(ctx, new.tolist(), (r.integers(4, 40, 600)).tolist(), 24, 2, 64, BF16)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("new,kv", [([1, 2, 1], [1, 35, 700]), ([1, 3], [9000, 20000]), ([40, 40, 1], [40, 73, 1]), ([300, 200], [9000, 500]),
                                    ([90, 1, 1, 7], [4400, 4300, 60, 9000])])
def test_attention_repeats_itself_exactly(ctx, dtype, new, kv):
    r = np.random.default_rng(len(new))
    tables, *cache, _, _ = make_cache(r, kv, 2, 128, 16)
    args = (dev(r.standard_normal((sum(new), 8, 128)), dtype), *cache, dev(tables), whole(np.concatenate([[0], np.cumsum(new)])), whole(kv), max(new))
    first = ctx.pq_kv_attention8(*args)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(first, ctx.pq_kv_attention8(*args)))


# few rows, whole and in parts; chunks, whole and in parts; both; the general kernel takes f32
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("new,kv,max_new", [([5, 3, 1], [200, 3, 90], 2), ([40, 3, 1, 9], [700, 90, 1, 9], 2), ([7, 40], [9000, 8000], 3),
                                            ([300, 40, 0, 1], [310, 90, 7, 60], 100), ([90, 130], [3000, 2900], 60),
                                            ([90, 1, 1, 30], [4400, 4300, 60, -1], 70), ([90, 9, 1, 30], [9000, 4300, 60, 30], 29),
                                            ([1, 1], [100, 200], 0)])
def test_attention_of_more_tokens_than_the_call_says(ctx, dtype, window, new, kv, max_new):
    """Rows of a request behind max_new are left, those before it are as without the limit."""
    r = np.random.default_rng(max_new)
    tables, *cache, keys, values = make_cache(r, kv, 2, 64, 16)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = int(cu[-1])
    q = dev(r.standard_normal((t, 4, 64)), dtype)
    out, lse = torch.full((t, 4, 64), 7.0, dtype=dtype, device="cuda"), torch.full((t, 4), 7.0, device="cuda")
    ctx.pq_kv_attention8(q, *cache, dev(tables), dev(cu), whole(kv), max_new, window=window, out=out, lse=lse)
    want, want_lse, spread = read_oracle.attention(host(q), keys, values, tables, cu, np.array(kv), 0.125, window)
    got, got_lse = host(out), host(lse)
    held = np.concatenate([np.arange(n) < max_new for n in new])
    assert (got[~held] == 7).all() and (got_lse[~held] == 7).all()
    bound, fp32 = attention_bound(dtype, host(q), keys, spread, want, 0.125, max(kv), 64)
    assert (np.abs(got - want) <= bound)[held].all()
    seen = held[:, None] & np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(got_lse)[held], np.isneginf(want_lse)[held])
    assert (np.abs(got_lse[seen] - want_lse[seen]) <= 2 * fp32 + 1e-6 * np.abs(want_lse[seen])).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_heads,heads,dim", [(2, 2, 64), (4, 2, 64), (8, 2, 96), (4, 1, 128), (2, 1, 256)])
@pytest.mark.parametrize("new", [[1, 40, 2, 17, 1, 3], [1] * 9 + [300], [5, 700, 1]])
def test_attention_of_single_tokens_beside_chunks(ctx, dtype, q_heads, heads, dim, new):
    kv = [4300 + 7 * i if i % 3 == 0 else 60 + n + 31 * i for i, n in enumerate(new)]
    kv[1] = -1 if len(new) > 6 else kv[1]
    check_attention(ctx, new, kv, q_heads, heads, dim, dtype, extra=2)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("window", [0, 30])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_of_lengths_that_no_plan_gives(ctx, new, window, dtype):
    """The least of all lengths sees nothing; keys behind the end of the table are not seen; blocks outside the cache are not read."""
    r = np.random.default_rng(new)
    tables, *cache, keys, values = make_cache(r, [90, 90, 90, 90], 2, 64, 16, 0)
    tables = tables[:, :5]                                  # 80 positions
    tables[3, 2], tables[3, 4] = -5, 10 ** 9
    cu = (np.arange(5) * new).astype(np.int32)
    q = dev(r.standard_normal((4 * new, 4, 64)), dtype)
    kv = np.array([-2 ** 31, 75, 85, 80], np.int32)
    out, lse = ctx.pq_kv_attention8(q, *cache, dev(tables), dev(cu), dev(kv), new, window=window)
    got, got_lse = host(out), host(lse)
    assert (got[:new] == 0).all() and np.isneginf(got_lse[:new]).all()
    for i in (1, 2):
        for t in range(new):
            at = kv[i] - new + t
            upto, first = min(at, 79), max(0, at - window + 1) if window else 0
            # (as one token whose last key is the last seen)
            row = i * new + t
            want, _, spread = read_oracle.attention(host(q)[row:row + 1], keys, values, tables[i:i + 1], np.array([0, 1]),
                                                    np.array([upto + 1]), 0.125, upto - first + 1)
            bound, _ = attention_bound(dtype, host(q), keys, spread, want, 0.125, 90, 64)
            assert (np.abs(got[row] - want[0]) <= bound[0]).all()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype,exponents", [(F32, (-100, 60)), (BF16, (-100, 60)), (F16, (-16, 7))])
def test_attention_of_scales_of_all_sizes(ctx, new, dtype, exponents):
    """One scale for all blocks, from very small to very large, for keys and values."""
    r = np.random.default_rng(new)
    for ke in exponents:
        for ve in exponents:
            tables, kc, vc, _, _, _, _ = make_cache(r, [new + 77, new], 2, 64, 16, 0)
            scales = [torch.full((kc.shape[0], 2), 2.0 ** e, device="cuda") for e in (ke, ve)]
            keys, values = host(kc) * 2.0 ** ke, host(vc) * 2.0 ** ve
            q = dev(r.standard_normal((2 * new, 4, 64)), dtype)
            scale, cu, kv = float(2.0 ** -(ke + 9)), np.array([0, new, 2 * new]), np.array([new + 77, new])
            out, lse = ctx.pq_kv_attention8(q, kc, vc, *scales, dev(tables), whole(cu), whole(kv), new, scale=scale)
            want, want_lse, spread = read_oracle.attention(host(q), keys, values, tables, cu, kv, scale, 0)
            bound, fp32 = attention_bound(dtype, host(q), keys, spread, want, scale, 0, 64)
            if dtype == F16:   # weights, and results, next to the type's least numbers; values are held to multiples of 2^-25
                bound += 2.0 ** -24 * 512 * 2.0 ** ve + 2.0 ** -24
            assert (np.abs(host(out) - want) <= bound).all()
            assert (np.abs(host(lse) - want_lse) <= 2 * fp32 + 1e-6 * np.abs(want_lse)).all()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [64, 80])
def test_attention_counts_the_exponents_of_scales(ctx, new, dtype, dim):
    """Scales between powers of two give the result of the power below, to the last bit."""
    r = np.random.default_rng(new)
    tables, kc, vc, ks, vs, _, _ = make_cache(r, [new + 77, new], 2, dim, 16, 0)
    q = dev(r.standard_normal((2 * new, 4, dim)), dtype)
    rest = (dev(tables), whole([0, new, 2 * new]), whole([new + 77, new]), new)
    want = ctx.pq_kv_attention8(q, kc, vc, ks, vs, *rest)
    got = ctx.pq_kv_attention8(q, kc, vc, ks * 1.75, vs * 1.25, *rest)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_attention_of_the_largest_values_of_f16(ctx, new, dtype):
    """Keys and values of 65504, which e4m3 holds as 2^16: weights add up to one, nothing overflows on the way."""
    kc = torch.full((4, 16, 1, 64), 256.0, device="cuda").to(E4M3)
    scales = torch.full((4, 1), 256.0, device="cuda")
    q = torch.full((new, 2, 64), 2.0 ** -20, device="cuda").to(dtype)
    small = kc.float().mul(2.0 ** -1).to(E4M3)
    out, lse = ctx.pq_kv_attention8(q, kc, small, scales, scales, whole([[0, 1, 2, 3]]), whole([0, new]), whole([60]), new, scale=1.0)
    # (a sum of equal weights over themselves, rounded: two units in fp32, one in the type)
    assert (np.abs(host(out) - 2.0 ** 15) <= 2.0 ** 15 * (2 * UNIT[dtype] + 2.0 ** -20)).all()
    want = 64 * 2.0 ** 16 * host(q)[0, 0, 0] + np.log(60.0 - new + 1 + np.arange(new))
    assert (np.abs(host(lse) - want[:, None]) <= 2e-5).all()


@pytest.mark.parametrize("new", [1, 40])
def test_attention_of_a_cache_with_a_wide_stride(ctx, new):
    """One block whose stride passes 32 bits."""
    r = np.random.default_rng(new)
    tables, kc, vc, ks, vs, keys, values = make_cache(r, [60], 2, 64, 64)
    block = int(tables[0, 0])
    kc, vc, ks, vs = kc[block:block + 1].contiguous(), vc[block:block + 1], ks[block:block + 1], vs[block:block + 1]
    wide = kc.as_strided(kc.shape, (2 ** 32,) + kc.stride()[1:])
    q = dev(r.standard_normal((new, 4, 64)), BF16)
    table, cu, kv = np.zeros((1, 1), np.int32), np.array([0, new], np.int32), np.array([60], np.int32)
    out, _ = ctx.pq_kv_attention8(q, wide, vc, ks, vs, dev(table), dev(cu), dev(kv), new)
    want, _, spread = read_oracle.attention(host(q), keys[block:block + 1], values[block:block + 1], table, cu, kv, 0.125, 0)
    bound, _ = attention_bound(BF16, host(q), keys, spread, want, 0.125, 60, 64)
    assert (np.abs(host(out) - want) <= bound).all()


@pytest.mark.parametrize("new", [1, 40])
def test_attention_adds_up_small_weights(ctx, new):
    """One key of a large weight and value 0, thousands of 2^-25.5 of it whose values are large: in f16 those weights count."""
    kv, count = 8192 + new, 8191
    tables = np.arange(-(-kv // 16), dtype=np.int32)[None]
    keys, values = (np.zeros((tables.shape[1], 16, 1, 64)) for _ in range(2))
    keys.reshape(-1, 64)[1:8192, 0], values.reshape(-1, 64)[1:8192] = -18.0, 256.0
    keys.reshape(-1, 64)[8192:, 0] = -448.0               # (the new tokens themselves)
    q = np.zeros((new, 1, 64))
    q[:, 0, 0] = 1.0
    ones, fours = torch.ones((tables.shape[1], 1), device="cuda"), torch.full((tables.shape[1], 1), 4.0, device="cuda")
    out, _ = ctx.pq_kv_attention8(dev(q, F16), dev(keys, F32).to(E4M3), dev(values, F32).to(E4M3), ones, fours, dev(tables), whole([0, new]), whole([kv]),
                                  new, scale=1.0)
    want = count * np.exp(-18.0) * 1024 / (1 + count * np.exp(-18.0))
    # half of the least weight, 2^-24 of 2^7 of the largest, for each of them; rounding of the result
    assert (np.abs(host(out) - want) <= count * 1024 * 2.0 ** -32 + 2.0 ** -10 * want).all()


def test_attention_refusals(ctx):
    i32 = dict(dtype=torch.int32, device="cuda")
    q, cache = torch.zeros((2, 4, 64), dtype=BF16, device="cuda"), torch.zeros((3, 16, 2, 64), device="cuda").to(E4M3)
    scales = torch.ones((3, 2), device="cuda")
    c = (cache, cache, scales, scales)
    table, cu, kv = torch.zeros((2, 1), **i32), torch.tensor([0, 1, 2], **i32), torch.tensor([4, 5], **i32)
    with pytest.raises(binding.PqError, match="kv_attention8") as e:
        ctx.pq_kv_attention8(q[:, :3], *c, table, cu, kv, 1)
    assert e.value.code == -2
    for bad in (dict(window=-1), dict(scale=float("nan"))):
        with pytest.raises(binding.PqError):
            ctx.pq_kv_attention8(q, *c, table, cu, kv, 1, **bad)
    with pytest.raises(binding.PqError):
        ctx.pq_kv_attention8(q, *c, torch.zeros((2, 0), **i32), cu, kv, 1)
    wide, wide_cache = torch.zeros((2, 4, 514), dtype=BF16, device="cuda"), torch.zeros((3, 16, 2, 514), device="cuda").to(E4M3)
    with pytest.raises(binding.PqError) as e:
        ctx.pq_kv_attention8(wide, wide_cache, wide_cache, scales, scales, table, cu, kv, 1)
    assert e.value.code == -3
    with pytest.raises(TypeError):
        ctx.pq_kv_attention8(q.double(), *c, table, cu, kv, 1)
    with pytest.raises(TypeError):
        ctx.pq_kv_attention8(q, cache.to(BF16), cache, scales, scales, table, cu, kv, 1)
    with pytest.raises(TypeError):
        ctx.pq_kv_attention8(q, cache, cache.view(torch.uint8), scales, scales, table, cu, kv, 1)
    with pytest.raises(TypeError):
        ctx.pq_kv_attention8(q, *c, table, cu, kv, 1, out=q.half())
    with pytest.raises(ValueError):
        ctx.pq_kv_attention8(q, cache, cache, scales[:2], scales, table, cu, kv, 1)
    with pytest.raises(ValueError):
        ctx.pq_kv_attention8(q, *c, table, cu[:2], kv, 1)
    with pytest.raises(ValueError):
        ctx.pq_kv_attention8(q, cache, cache.transpose(2, 3), scales, scales, table, cu, kv, 1)


@pytest.mark.parametrize("dim,dtype,tokens", [(2, F32, 2 ** 25 + 4), (64, BF16, 2 ** 29)])
def test_append_of_more_tokens_than_a_launch_takes(ctx, dim, dtype, tokens):
    x = torch.ones((1, 1, dim), dtype=dtype, device="cuda").expand(tokens, 1, dim)
    positions, slots = torch.zeros(tokens, dtype=torch.int32, device="cuda"), torch.full((tokens,), -1, dtype=torch.int64, device="cuda")
    cache = torch.zeros((2, 4, 1, dim), device="cuda").to(E4M3)
    with pytest.raises(binding.PqError, match="kv_append8") as e:
        ctx.pq_kv_append8(None, x, x, positions, slots, cache, cache, *torch.ones((2, 2, 1), device="cuda"))
    assert e.value.code == -3
    with pytest.raises(binding.PqError, match="kv_append") as e:
        ctx.pq_kv_append(None, x, x, positions, slots, *torch.zeros((2, 2, 4, 1, dim), dtype=dtype, device="cuda"))
    assert e.value.code == -3


@pytest.mark.parametrize("dim,dtype,tokens,requests", [(2, F32, 2 ** 24, 1), (64, BF16, 1, 2 ** 24), (64, BF16, 40, 2 ** 24)])
def test_attention_of_more_rows_than_a_launch_takes(ctx, dim, dtype, tokens, requests):
    i32 = dict(dtype=torch.int32, device="cuda")
    q, cache, ones = torch.ones((tokens, 1, dim), dtype=dtype, device="cuda"), torch.zeros((2, 16, 1, dim), device="cuda"), torch.ones((2, 1), device="cuda")
    where = (torch.zeros((requests, 1), **i32), torch.zeros(requests + 1, **i32), torch.zeros(requests, **i32), tokens)
    with pytest.raises(binding.PqError, match="kv_attention") as e:
        ctx.pq_kv_attention8(q, cache.to(E4M3), cache.to(E4M3), ones, ones, *where)
    assert e.value.code == -3
    with pytest.raises(binding.PqError, match="kv_attention") as e:
        ctx.pq_kv_attention(q, cache.to(dtype), cache.to(dtype), *where)
    assert e.value.code == -3


# ---- log-probabilities ------------------------------------------------------------------------------------------------
def check_logprobs(ctx, logits, tokens, top):
    """fp32 sums of up to 2^20 terms in parts of at most 2^12, each term off by a few units and by its distance from the maximum (up
    to about 100, where its weight ends) times one; logarithm and difference: some units of numbers up to the result's size."""
    lp, ranks, entropy, first, top_lp = (host(x) for x in ctx.pq_token_logprobs(logits, whole(tokens, np.int64), top))
    for r, l in enumerate(host(logits)):
        want_lp, rank, want_entropy, want_first, want_top = orc.logprobs(l, int(tokens[r]), top)
        assert ranks[r] == rank and np.array_equal(first[r], want_first), r
        sure = max(abs(x) for x in [0.0, *l[np.isfinite(l)]]) * 2.0 ** -23       # (differences of logits of that size)
        assert lp[r] == want_lp or abs(lp[r] - want_lp) <= 3e-6 * (1 + abs(want_lp)) + sure, (r, lp[r], want_lp)
        assert abs(entropy[r] - want_entropy) <= 5e-6 * (1 + want_entropy) + sure, (r, entropy[r], want_entropy)
        assert entropy[r] >= 0
        some = np.isfinite(want_top)
        assert np.array_equal(top_lp[r][~some], want_top[~some])
        assert (np.abs(top_lp[r] - want_top)[some] <= 3e-6 * (1 + np.abs(want_top[some])) + sure).all()
    return lp, ranks, entropy, first, top_lp


def rows_of(r, rows, vocab, dtype, spread=3.0):
    l = r.standard_normal((rows, vocab)) * spread
    l[:, r.integers(0, vocab, max(1, vocab // 50))] = -np.inf
    if vocab > 1:
        l[:, r.integers(0, vocab)] = 0.5
    return dev(l, dtype)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 500, 1000, 4099, 32000, 50021, 131072])
@pytest.mark.parametrize("top", [0, 1, 20, 128])
def test_logprobs(ctx, dtype, vocab, top):
    r = np.random.default_rng(vocab)
    logits = rows_of(r, 5, vocab, dtype)
    tokens = r.integers(0, vocab, 5)
    tokens[1] = host(logits)[1].argmax()
    check_logprobs(ctx, logits, tokens, top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 300, 1100])
def test_logprobs_of_many_rows(ctx, dtype, rows):
    r = np.random.default_rng(rows)
    check_logprobs(ctx, rows_of(r, rows, 1003, dtype), r.integers(-1, 1005, rows), 7)


def test_logprobs_of_more_rows_than_a_launch_takes(ctx):
    """The most rows that 2^32 - 1 threads hold, all of them answered, and one more."""
    rows = 2 ** 24 - 1
    logits = torch.tensor([[1.0, 2.0, -1.0]], device="cuda").expand(rows + 1, 3)
    want = host(ctx.pq_token_logprobs(logits[:1], top=1)[4])[0, 0]
    out = (None, None, None, torch.full((rows, 1), -7, device="cuda"), torch.zeros((rows, 1), device="cuda"))
    ctx.pq_token_logprobs(logits[:rows], top=1, out=out)
    assert bool((out[3] == 1).all()) and bool((out[4] == float(want)).all())
    with pytest.raises(binding.PqError, match="token_logprobs") as e:
        ctx.pq_token_logprobs(logits, top=1)
    assert e.value.code == -3
    with pytest.raises(binding.PqError, match="sample_tokens") as e:
        ctx.pq_sample_tokens(logits, None)
    assert e.value.code == -3


def test_logprobs_of_the_largest_vocabulary(ctx):
    r = np.random.default_rng(1)
    for dtype in (F32, BF16):
        check_logprobs(ctx, rows_of(r, 2, 2 ** 20 - 1, dtype), [2 ** 20 - 2, 0], 20)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [300, 30011])
@pytest.mark.parametrize("top", [1, 20, 128])
def test_logprobs_of_equal_and_ordered_logits(ctx, dtype, vocab, top):
    """Equal logits, few values, rising and falling rows, and the likeliest tokens all at places that one thread reads."""
    r = np.random.default_rng(vocab)
    rows = [np.full(vocab, -2.5), np.full(vocab, -2.5), np.arange(vocab) * 2.0 ** -6, -np.arange(vocab) * 2.0 ** -6, r.integers(0, 3, vocab) / 2,
            np.zeros(vocab), np.zeros(vocab), np.zeros(vocab)]
    rows[1][::2] = 1.0
    rows[5][::256] = 1 + np.arange(len(rows[5][::256])) * 2.0 ** -5
    rows[6][:200] = 5.0
    rows[7][np.arange(vocab) % 2048 < 8] = 2.0 + (np.arange(vocab)[np.arange(vocab) % 2048 < 8] % 64) / 32
    check_logprobs(ctx, dev(np.stack(rows), dtype), r.integers(0, vocab, len(rows)), top)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [3000, 70001])
@pytest.mark.parametrize("top", [1, 50, 128])
def test_logprobs_of_close_logits(ctx, dtype, vocab, top):
    """Logits that lie close together, and a few that stand out of thousands of equal ones, in runs, far apart, in pairs."""
    r = np.random.default_rng(vocab)
    l = np.stack([r.uniform(0.99, 1, vocab), 20 + r.standard_normal(vocab) * 0.01, -r.uniform(300, 301, vocab)] + [np.full(vocab, 0.25)] * 6)
    out = r.permutation(vocab)
    l[3, out[:60]] = 1 + np.arange(60) / 16
    l[4, out[:60]] = 1 + np.arange(60) // 2 / 16
    l[5, ::300] = 2.0
    l[6, vocab // 2:] = -1.0
    l[7, out[:40]], l[7, vocab // 3:vocab // 3 + 1500] = 3 + np.arange(40) / 16, 2.5
    l[8] = -3e4
    l[8, out[:30]] = -5 - np.arange(30) / 16
    check_logprobs(ctx, dev(l, dtype), r.integers(0, vocab, 9), top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [40, 20000])
def test_logprobs_of_special_rows(ctx, dtype, vocab):
    """Masks of -inf, of NaN and of the type's lowest value, +inf, single tokens, rows without any."""
    lowest, largest = torch.finfo(dtype).min, torch.finfo(dtype).max
    l = np.random.default_rng(2).standard_normal((14, vocab))
    l[0], l[1] = -np.inf, np.nan
    l[2], l[2, 7] = -np.inf, -1.0
    l[3], l[3, 9], l[3, 11] = lowest, 2.0, 1.0
    l[4] = lowest
    l[5], l[5, ::3] = lowest, -np.inf
    l[6, 5], l[6, 30] = np.inf, np.inf
    l[7, 3], l[7, 4] = np.nan, np.inf
    l[8, 20] = largest
    l[9, 20], l[9, 21] = largest, largest
    l[10], l[10, 3], l[10, 4] = lowest, lowest / 2, lowest / 4
    l[11, 0] = -0.0
    l[11, 1:] = 0.0
    l[12] *= 1e4
    l[13], l[13, 6] = -300.0, 300.0
    tokens = [3, 0, 7, 11, 5, 1, 30, 3, 20, 20, 4, 1, 5, 0]
    check_logprobs(ctx, dev(l, dtype), tokens, 20)
    check_logprobs(ctx, dev(l, dtype), [0, 39, 6, 12, 39, 3, 5, 4, 5, 21, 3, 0, vocab, -1], 3)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [7, 600, 40000])
@pytest.mark.parametrize("mask", [-3e4, -6e5, -1.1e6, -1e9, -1e30, -3e38])
def test_logprobs_of_masks_and_large_logits(ctx, dtype, vocab, mask):
    """Masks that are numbers: most of a row, whole stretches of it, all of it but next to nothing; rows that lie as low or as high."""
    if dtype == F16:
        mask = max(mask, -65504.0)
    l = np.random.default_rng(3).standard_normal((8, vocab))
    l[0, : vocab // 2] = mask
    l[1, vocab // 3:] = mask
    l[2], l[2, 3] = mask, 1.0
    l[3], l[3, 2], l[3, 5] = mask, -np.inf, mask / 2
    l[4] = mask
    l[5, : vocab // 2] = mask
    l[5, vocab // 2:] = -np.inf
    l[6, 1], l[6, 4] = -mask, -mask
    l[7] += mask / 4
    check_logprobs(ctx, dev(l, dtype), [0, vocab - 1, 3, 5, 1, 2, 4, 6], 5)


def test_logprobs_layouts(ctx):
    """Rows of any stride, that begin at any element; results that are not wanted."""
    r = np.random.default_rng(3)
    for dtype in (F32, F16, BF16):
        wide = rows_of(r, 6, 5003, dtype)
        for a, b in ((1, 5000), (3, 2050), (2, 11), (5, 5003), (7, 8)):
            check_logprobs(ctx, wide[:, a:b], r.integers(0, b - a, 6), 9)
        check_logprobs(ctx, wide[::2], r.integers(0, 5003, 3), 9)
        check_logprobs(ctx, wide[:1].expand(4, 5003), r.integers(0, 5003, 4), 2)
    logits, tokens = rows_of(r, 6, 5003, F32), whole(r.integers(0, 5003, 6), np.int64)
    every = ctx.pq_token_logprobs(logits, tokens, 5)
    lp, ranks, *rest = ctx.pq_token_logprobs(logits, None, 5)
    assert lp is None and ranks is None and all(torch.equal(a, b) for a, b in zip(rest, every[2:]))
    for k in range(5):
        out = [None] * 5
        out[k] = torch.full_like(every[k], 7)
        assert ctx.pq_token_logprobs(logits, tokens, 5, out=tuple(out))[k] is out[k] and torch.equal(out[k], every[k])
    assert all(x.shape[0] == 0 for x in ctx.pq_token_logprobs(logits[:0], tokens[:0], 5))


def test_logprobs_are_those_of_the_draw(ctx):
    """The draw without filters at temperature 1 and the score of its token are one number."""
    r = np.random.default_rng(4)
    logits = rows_of(r, 40, 32000, BF16)
    tokens, drawn = ctx.pq_sample_tokens(logits, dev(r.random((40, 32000)).astype(np.float32).clip(1e-7, 1 - 1e-7)))
    scored, ranks, _, first, _ = ctx.pq_token_logprobs(logits, tokens, 1)
    assert (np.abs(host(scored) - host(drawn)) <= 4e-6 * (1 + np.abs(host(drawn)))).all()
    greedy, _ = ctx.pq_sample_tokens(logits, None)
    assert torch.equal(first[:, 0], greedy)


def test_logprobs_repeat_themselves_exactly(ctx):
    r = np.random.default_rng(5)
    for rows, vocab in ((3, 131072), (700, 5003)):
        logits, tokens = rows_of(r, rows, vocab, BF16), whole(r.integers(0, vocab, rows), np.int64)
        first = ctx.pq_token_logprobs(logits, tokens, 20)
        for _ in range(20):
            assert all(torch.equal(a, b) for a, b in zip(first, ctx.pq_token_logprobs(logits, tokens, 20)))


def test_logprobs_refusals(ctx):
    l, t = torch.zeros((2, 50), device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    for bad in (dict(logits=l.double()), dict(tokens=t.int()), dict(logits=l.cpu())):
        with pytest.raises(TypeError):
            ctx.pq_token_logprobs(**{**dict(logits=l, tokens=t, top=3), **bad})
    for bad in (dict(logits=l[0]), dict(tokens=t[:1]), dict(logits=l.T), dict(top=2 ** 40)):
        with pytest.raises((ValueError, RuntimeError)):
            ctx.pq_token_logprobs(**{**dict(logits=l, tokens=t, top=3), **bad})
    for bad, code in ((dict(top=-1), -1), (dict(top=129), -3), (dict(logits=torch.zeros((2, 0), device="cuda")), -1),
                      (dict(logits=torch.zeros((2, 2 ** 20), device="cuda")), -3)):
        with pytest.raises(binding.PqError, match="token_logprobs") as e:
            ctx.pq_token_logprobs(**{**dict(logits=l, tokens=t, top=3), **bad})
        assert e.value.code == code
    out = (torch.zeros(2, device="cuda"), None, None, None, None)
    with pytest.raises(binding.PqError):
        ctx.pq_token_logprobs(l, None, 0, out=out)


def test_calls_of_a_closed_context_are_refused():
    c = binding.Context(0)
    c.close()
    one, x = whole([1]), torch.zeros((1, 1, 64), device="cuda")
    cache, scales = torch.zeros((1, 16, 1, 64), device="cuda").to(E4M3), torch.ones((1, 1), device="cuda")
    for call in (lambda: c.pq_kv_append8(x, x, x, one, one.long(), cache, cache, scales, scales),
                 lambda: c.pq_kv_attention8(x, cache, cache, scales, scales, one.view(1, 1), whole([0, 1]), one, 1),
                 lambda: c.pq_token_logprobs(x[0], one.long())):
        with pytest.raises(binding.PqError, match="null context"):
            call()


# ---- together ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_steps_over_a_cache_of_8_bits(ctx, dtype):
    """Prompts and then single tokens through plan, append, attention and log-probabilities, each step against the oracles on a cache that
    they keep themselves; one request is refused half way."""
    r = np.random.default_rng(6)
    heads, q_heads, dim, size, blocks = 2, 4, 64, 16, 40
    codes = [torch.full((blocks, size, heads, dim), 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
    scales = [torch.full((blocks, heads), float("nan"), device="cuda") for _ in range(2)]
    held, held_scales = [host(c) for c in codes], [np.ones((blocks, heads)) for _ in range(2)]
    angle = r.uniform(-3, 3, (400, 32))
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    head = r.standard_normal((q_heads * dim, 777)).astype(np.float32)
    cached, tables, free = whole([0, 0, 0]), whole(np.full((3, 12), -1)), whole(r.permutation(blocks))
    for step, new in enumerate([[37, 5, 90], [1, 1, 1], [1, 1, 1], [20, 1, 3], [1, 1, 2000], [1, 1, 1]]):
        if step == 4:
            new = [1, 1, 190]           # more than the table's row holds: refused, now and from then on
        t = sum(new)
        cu, kv, positions, slots, taken = ctx.pq_kv_plan(whole(new), cached, tables, free, size, t)
        x = dev(r.standard_normal((t, q_heads + 2 * heads, dim)) * 2, dtype)
        q = ctx.pq_kv_append8(x[:, :q_heads], x[:, q_heads:q_heads + heads], x[:, q_heads + heads:], positions, slots, *codes, *scales, dev(cos), dev(sin))
        out, lse = ctx.pq_kv_attention8(q, *codes, *scales, tables, cu, kv, max(new))
        p, s = host(positions), host(slots)
        keys = read_oracle.turn(host(x[:, q_heads:q_heads + heads]), np.maximum(p, 0), cos, sin, None, float(np.float32(1e-6)), True, False).astype(np.float32)
        for i, rows in enumerate((keys, host(x[:, q_heads + heads:]))):
            orc.store(held[i], held_scales[i], rows, s, s >= 0)
            assert np.array_equal(host(codes[i]), held[i], equal_nan=True)
        full = [h * w[:, None, :, None] for h, w in zip(held, held_scales)]
        want, want_lse, spread = read_oracle.attention(host(q), *full, host(tables), host(cu), host(kv), dim ** -0.5, 0)
        seen = ~np.isneginf(want_lse)
        bound, fp32 = attention_bound(dtype, host(q), np.where(np.isnan(full[0]), 0, full[0]), spread, want, dim ** -0.5, 300, dim)
        assert (np.abs(host(out) - want) <= bound).all() and np.array_equal(seen, np.isfinite(host(lse)))
        logits = (out.reshape(t, -1).float() @ dev(head)).to(dtype)
        check_logprobs(ctx, logits, r.integers(0, 777, t), 5)
        free, cached = free[int(taken):], kv
    assert host(cached).tolist()[2] == -1 and host(cached)[0] > 60


def test_a_captured_step_replays(ctx):
    """Append, attention and log-probabilities in one HIP graph, replayed on new inputs with eager work in between."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = binding.Context(0, side)
        new, cached = whole([1, 1, 1]), whole([5, 16, 40])
        tables, free = whole(np.arange(12).reshape(3, 4)), whole(np.arange(12, 20))
        start = [torch.randn((20, 16, 2, 64), device="cuda").to(E4M3) for _ in range(2)] + [torch.full((20, 2), 2.0 ** -9, device="cuda") for _ in range(2)]
        cache = [x.clone() for x in start]
        qkv = torch.zeros((3, 8, 64), dtype=BF16, device="cuda")

        def step():
            cu, kv, positions, slots, _ = c.pq_kv_plan(new, cached, tables, free, 16, 3)
            q = c.pq_kv_append8(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], positions, slots, *cache)
            out, lse = c.pq_kv_attention8(q, *cache, tables, cu, kv, 1)
            return (out, lse) + tuple(c.pq_token_logprobs(out.view(3, 256), positions.long(), 4))

        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            captured = step()
        for k in range(4):
            qkv.copy_((torch.randn((3, 8, 64), device="cuda") * 4 ** k).to(BF16))
            found = []
            for run in (step, lambda: graph.replay() or captured):
                for x, s in zip(cache, start):
                    x.copy_(s)
                found.append([x.clone() for x in run()] + [x.clone().view(torch.uint8) for x in cache])
                side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(*found)), k
        c.close()
