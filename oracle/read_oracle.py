"""Plain 64-bit implementations of the reading step (numpy, loops where the definition has them): the plan of a paged
cache, the append, the attention and the draw.  Slow, for small inputs."""
import numpy as np


def plan(new_lens, cached_lens, tables, free_blocks, block_size, ntokens):
    """Returns (tables, cu, kv_lens, positions, slots, taken)."""
    tables = tables.copy()
    width = tables.shape[1]
    cu, kv = [0], []
    positions, slots = np.full(ntokens, -1, np.int32), np.full(ntokens, -1, np.int64)
    counted = taken = 0
    for r, (n, c) in enumerate(zip(new_lens.tolist(), cached_lens.tolist())):
        n, refused, c = max(n, 0), c < 0, max(c, 0)
        have, full = -(-c // block_size), -(-(c + n) // block_size)
        fits = not refused and full <= width
        need = full - have if fits else 0
        counted += need
        served = fits and counted <= len(free_blocks) and cu[-1] + n <= ntokens
        if served:
            taken += need
            tables[r, have:full] = free_blocks[counted - need:counted]
            for i in range(n):
                positions[cu[-1] + i] = c + i
                slots[cu[-1] + i] = int(tables[r, (c + i) // block_size]) * block_size + (c + i) % block_size
        kv.append(c + n if served else -1)
        cu.append(cu[-1] + n)
    return tables, np.minimum(np.array(cu), 2 ** 31 - 1).astype(np.int32), np.array(kv, np.int32), positions, slots, taken


def turn(x, positions, cos, sin, weight, eps, norm, pairs):
    """Norm and rotation of heads [tokens][heads][dim] in double."""
    x = x.astype(np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
        if weight is not None:
            x = x * weight.astype(np.float64)
    y = x.copy()
    half = 0 if cos is None else cos.shape[1]
    for t, p in enumerate(positions.tolist()):
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
            c, s = float(cos[p, i]), float(sin[p, i])
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, a] * s + x[t, :, b] * c
    return y


def attention(q, keys, values, tables, cu, kv_lens, scale, window):
    """q [tokens][q heads][dim], caches [blocks][block size][heads][dim]; returns (out, lse, spread) in double, spread = the
    sum of weight * |value|, which rounding errors are in proportion to.  Rows behind cu[-1] are NaN."""
    ntokens, q_heads, dim = q.shape
    block_size, heads = keys.shape[1:3]
    out, spread = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse = np.full((ntokens, q_heads), np.nan)
    for r, kv in enumerate(kv_lens.tolist()):
        for t in range(int(cu[r]), int(cu[r + 1])):
            at = kv - (int(cu[r + 1]) - t)
            seen = np.arange(max(0, at - window + 1) if window > 0 else 0, at + 1)
            out[t], spread[t], lse[t] = 0.0, 0.0, -np.inf
            if len(seen) == 0:
                continue
            block, place = tables[r, seen // block_size], seen % block_size
            for h in range(q_heads):
                g = h // (q_heads // heads)
                score = keys[block, place, g].astype(np.float64) @ q[t, h].astype(np.float64) * scale
                top = score.max()
                weight = np.exp(score - top)
                lse[t, h] = top + np.log(weight.sum())
                v = values[block, place, g].astype(np.float64)
                out[t, h] = weight @ v / weight.sum()
                spread[t, h] = weight @ np.abs(v) / weight.sum()
    return out, lse, spread


def kept(logits, temperature, top_k, top_p, min_p):
    """The tokens of one row that stay, in order, their x, and how near the limit of top_p was passed, as a share of all weight."""
    logits = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    order = np.argsort(-logits, kind="stable")
    top = logits[order[0]]
    x = np.where(logits == top, 0.0, (logits - top) / temperature if np.isfinite(top) else -np.inf)[order]
    weight = np.where(x >= -87, np.exp(x), 0.0)
    n, margin = int((weight > 0).sum()), 1.0
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        before = np.cumsum(weight[:n]) - weight[:n]
        limit = top_p * weight[:n].sum()
        margin = float(np.abs(before - limit).min() / weight[:n].sum())
        n = max(1, int((before < limit).sum()))
    if min_p > 0:
        n = max(1, min(n, int((weight[:n] >= min_p).sum())))
    return order[:n], x[:n], margin


def sample(logits, noise, temperature, top_k, top_p, min_p):
    """Draw of one row: (token, logprob, scores of the tokens that stay by token, margin)."""
    logits = logits.astype(np.float64)
    usable = logits[~np.isnan(logits)]
    if len(usable) == 0 or usable.max() == -np.inf:
        return -1, -np.inf, {}, 1.0
    if not temperature > 0:
        return int(np.argmax(np.where(np.isnan(logits), -np.inf, logits))), 0.0, {}, 1.0
    tokens, x, margin = kept(logits, temperature, top_k, top_p, min_p)
    with np.errstate(divide="ignore"):
        score = x if noise is None else x - np.log(-np.log(noise.astype(np.float64)[tokens]))
    best = min((-s, int(i)) for s, i in zip(score, tokens))[1]
    at = int(np.flatnonzero(tokens == best)[0])
    return best, float(x[at] - np.log(np.exp(x).sum())), dict(zip(tokens.tolist(), score.tolist())), margin
