"""The reading step over a cache of 8 bits and the log-probabilities of tokens at the ends of their ranges: bounds that know what of a row
counts, scales and sizes next to the limits, against the oracles in 64 bits."""
import gc

import numpy as np
import pytest
import torch

from oracle import read8_oracle as orc
from paper_1712_02912_amd import binding
from test_gpu_read8 import BF16, F16, F32, dev, host, whole

pytestmark = pytest.mark.gpu

HALF_UNIT = 2.0 ** -24   # of fp32, relative


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()
    gc.collect()


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
