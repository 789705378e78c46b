"""Plain 64-bit implementations (numpy, loops where the definition has them) of the append to a cache of 8 bits and of the
log-probabilities of tokens.  The attention over such a cache is that of read_oracle over what its elements stand for."""
import numpy as np


def numbers():
    """What the 256 codes of e4m3 stand for."""
    code = np.arange(256)
    exponent, fraction = code >> 3 & 15, code & 7
    size = np.where(exponent > 0, (1 + fraction / 8) * 2.0 ** (exponent - 7), fraction / 8 * 2.0 ** -6)
    size[[127, 255]] = np.nan
    return np.where(code < 128, size, -size)


def rounded(x):
    """The e4m3 numbers nearest to x, of two as near the one with an even fraction; what is larger than 448 becomes it."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        size = np.minimum(np.abs(x), 448.0)
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.where(np.isnan(size), 1.0, size), 2.0 ** -6))) - 3)
        return np.where(np.isnan(x), np.nan, np.copysign(np.round(size / step) * step, x))


def scale_for(amax):
    """The smallest power of two from 2^-126 on of which amax is at most 448 times."""
    k = -126
    while amax > 448.0 * 2.0 ** k:
        k += 1
    return 2.0 ** k


def runs(slots, block_size, written):
    """(first token, count) of the tokens that follow each other within a block; written: whether a token counts."""
    found = []
    for t, slot in enumerate(slots.tolist()):
        if not written[t]:
            continue
        if slot % block_size and t > 0 and written[t - 1] and slots[t - 1] == slot - 1:
            found[-1][1] += 1
        else:
            found.append([t, 1])
    return found


def store(values, scales, rows, slots, written):
    """Writes rows [tokens][heads][dim] (fp32 values) into a cache: values [blocks][block size][heads][dim] in units of the scales
    [blocks][heads], both in place."""
    block_size = values.shape[1]
    for t, count in runs(slots, block_size, written):
        block, place = slots[t] // block_size, slots[t] % block_size
        for h in range(values.shape[2]):
            x = rows[t:t + count, h].astype(np.float64)
            scale = scale_for(np.abs(x[np.isfinite(x)]).max(initial=0.0))
            if place > 0 and scales[block, h] >= scale:
                scale = scales[block, h]
            elif place > 0:
                values[block, :place, h] = rounded(values[block, :place, h] * (scales[block, h] / scale))
            values[block, place:place + count, h] = rounded(x / scale)
            scales[block, h] = scale


def logprobs(logits, token, top):
    """One row: (log p of token, its rank, entropy, first tokens, their log p)."""
    l = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    order = np.argsort(-l, kind="stable")
    high = l[order[0]]
    first, lp = np.full(top, -1), np.full(top, -np.inf)
    there = 0 <= token < len(l)
    rank = int(np.flatnonzero(order == token)[0]) if there else -1
    if high == -np.inf:
        return -np.inf, rank, 0.0, first, lp
    with np.errstate(invalid="ignore"):
        below = np.where(l == high, 0.0, l - high)
    weight = np.exp(below)
    log_p = below - np.log(weight.sum())
    n = min(top, int((l > -np.inf).sum()))
    first[:n], lp[:n] = order[:n], log_p[order[:n]]
    some = weight > 0
    entropy = -(np.exp(log_p[some]) * log_p[some]).sum()
    return log_p[token] if there else -np.inf, rank, entropy, first, lp
