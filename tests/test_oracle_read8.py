"""The oracle of the cache of 8 bits and of the log-probabilities against brute force and identities, on the CPU."""
import numpy as np
import pytest
import torch

from oracle import read8_oracle as orc


def test_numbers_are_those_of_the_type():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.numbers(), want, equal_nan=True)


def test_rounding_takes_the_nearest_number():
    r = np.random.default_rng(1)
    x = np.concatenate([r.uniform(-448, 448, 3000), r.standard_normal(3000) * 2.0 ** r.integers(-12, 8, 3000)])
    all_numbers = np.unique(orc.numbers()[~np.isnan(orc.numbers())])
    assert (np.abs(orc.rounded(x) - x) == np.abs(all_numbers[:, None] - x).min(axis=0)).all()
    # ties: the even fraction, which is the even code
    middle = (all_numbers[1:] + all_numbers[:-1]) / 2
    codes = torch.from_numpy(orc.rounded(middle)).float().to(torch.float8_e4m3fn).view(torch.uint8)
    assert (codes % 2 == 0).all()
    assert orc.rounded([448.0, 460.0, 1e30, -np.inf]).tolist() == [448, 448, 448, -448] and np.isnan(orc.rounded(np.nan))


def test_rounding_is_that_of_torch():
    x = torch.from_numpy(np.random.default_rng(2).standard_normal(20000)).float() * 30
    assert np.array_equal(orc.rounded(x.numpy()), x.to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("amax", [0.0, 1e-45, 448.0, np.nextafter(448.0, 449.0), 1.75, 3.4e38, 0.1])
def test_scales_are_the_smallest_that_hold(amax):
    s = orc.scale_for(amax)
    assert amax <= 448 * s and (s == 2.0 ** -126 or amax > 448 * (s / 2)) and np.log2(s) == int(np.log2(s))


def test_runs_end_with_blocks_gaps_and_tokens_that_are_not_written():
    slots = np.array([3, 4, 5, 6, 9, 10, -1, 11, 12, 12, 7])
    written = slots >= 0
    assert orc.runs(slots, 4, written) == [[0, 1], [1, 3], [4, 2], [7, 1], [8, 1], [9, 1], [10, 1]]


def test_store_keeps_the_rest_of_the_block_and_grows_its_scale():
    r = np.random.default_rng(3)
    values, scales = orc.rounded(r.standard_normal((3, 4, 2, 8)) * 100), np.full((3, 2), 0.5)
    before, old = values.copy(), scales.copy()
    rows = r.standard_normal((3, 2, 8)) * np.array([[[1.0], [5000.0]]])
    orc.store(values, scales, rows, np.array([6, 7, 8]), np.ones(3, bool))
    assert scales[1, 0] == 0.5 and scales[1, 1] > 0.5 and np.array_equal(scales[0], old[0])
    assert np.array_equal(values[0], before[0]) and np.array_equal(values[1, :2, 0], before[1, :2, 0]) and np.array_equal(values[2, 1:], before[2, 1:])
    held = (values * scales[:, None, :, None])
    # (half a step of the smallest numbers, in units of the scale)
    assert (np.abs(held[1, 2:] - rows[:2]) <= 2.0 ** -4 * np.abs(rows[:2]) + 2.0 ** -10 * scales[1][None, :, None]).all()
    assert (np.abs(held[1, :2, 1] - before[1, :2, 1] * 0.5) <= 2.0 ** -4 * np.abs(before[1, :2, 1] * 0.5) + 2.0 ** -10 * scales[1, 1]).all()
    assert scales[2, 0] == orc.scale_for(np.abs(rows[2, 0]).max())


def test_logprobs_against_torch():
    l = np.random.default_rng(4).standard_normal((5, 40)) * 3
    l[1, 7] = l[1, 20] = l[1].max() + 1
    for i in range(5):
        lp, rank, entropy, first, top = orc.logprobs(l[i], 20, 4)
        want = torch.log_softmax(torch.from_numpy(l[i]), 0)
        np.testing.assert_allclose(lp, float(want[20]), rtol=1e-12)
        np.testing.assert_allclose(entropy, float(torch.distributions.Categorical(logits=want).entropy()), rtol=1e-12)
        np.testing.assert_allclose(top, want[first].numpy(), rtol=1e-12)
        assert rank == int((l[i] > l[i, 20]).sum()) + int((l[i, :20] == l[i, 20]).sum())
    assert orc.logprobs(l[1], 20, 2)[1] == 1 and orc.logprobs(l[1], 7, 2)[3].tolist() == [7, 20]


def test_logprobs_of_special_rows():
    nan, inf = np.nan, np.inf
    lp, rank, entropy, first, top = orc.logprobs(np.array([nan, -inf, 2.0, -inf]), 0, 3)
    assert lp == -inf and rank == 1 and entropy == 0 and first.tolist() == [2, -1, -1] and top.tolist() == [0, -inf, -inf]
    lp, rank, entropy, first, top = orc.logprobs(np.array([1.0, inf, 2.0, inf]), 3, 4)
    assert lp == -np.log(2) and rank == 1 and entropy == np.log(2) and first.tolist() == [1, 3, 2, 0] and top[2] == -inf
    assert orc.logprobs(np.array([nan, -inf]), 1, 1)[:3] == (-inf, 1, 0.0) and orc.logprobs(np.zeros(3), 3, 0)[:2] == (-inf, -1)
