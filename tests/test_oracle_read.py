"""The oracle of the reading step against brute force and identities, on the CPU."""
import numpy as np
import pytest

from oracle import read_oracle as orc


def test_plan_gives_every_place_to_one_token():
    r = np.random.default_rng(1)
    new, cached = r.integers(0, 9, 40), r.integers(0, 30, 40)
    tables = np.full((40, 12), -1, np.int32)
    pool = r.permutation(600).astype(np.int32)
    at = 0
    for i, c in enumerate(cached):
        n = -(-int(c) // 4)
        tables[i, :n] = pool[at:at + n]
        at += n
    t, cu, kv, positions, slots, taken = orc.plan(new.astype(np.int32), cached.astype(np.int32), tables, pool[at:], 4, int(new.sum()))
    assert np.array_equal(kv, new + cached) and cu[-1] == new.sum()
    held = np.concatenate([t[i, :-(-int(k) // 4)] for i, k in enumerate(kv)])
    assert len(set(held.tolist())) == len(held) == at + taken
    assert len(set(slots.tolist())) == len(slots)
    for i in range(40):
        for j in range(cu[i], cu[i + 1]):
            p = cached[i] + j - cu[i]
            assert positions[j] == p and slots[j] == t[i, p // 4] * 4 + p % 4


def test_plan_refuses_in_order():
    new, cached = np.array([5, 5, 100, 1, 5]), np.array([0, 0, 0, 3, 0])
    t, cu, kv, positions, slots, taken = orc.plan(new, cached, np.zeros((5, 3), np.int32), np.arange(10, 13), 4, 200)
    # two blocks for the first; the second's two are one too many, so is every later need; the third does not fit its row
    assert kv.tolist() == [5, -1, -1, -1, -1] and taken == 2 and (positions[5:] == -1).all()


def test_plan_refuses_again_what_it_refused():
    tables = np.arange(15, dtype=np.int32).reshape(5, 3)
    t, cu, kv, positions, slots, taken = orc.plan(np.array([1, 3, 0, 1, 2]), np.array([4, -1, -7, -2 ** 31, 4]), tables, np.arange(20, 30), 4, 9)
    assert kv.tolist() == [5, -1, -1, -1, 6] and taken == 2 and cu.tolist() == [0, 1, 4, 4, 5, 7]
    assert positions.tolist() == [4, -1, -1, -1, -1, 4, 5, -1, -1] and np.array_equal(t[1:4], tables[1:4])
    assert slots.tolist() == [80, -1, -1, -1, -1, 84, 85, -1, -1]


@pytest.mark.parametrize("pairs", [False, True])
def test_turn_keeps_lengths_and_relative_angles(pairs):
    r = np.random.default_rng(2)
    x = r.standard_normal((2, 3, 8))
    angle = np.arange(20)[:, None] * np.array([1.0, 0.3, 0.1])
    cos, sin = np.cos(angle), np.sin(angle)

    def at(p, q):
        y = orc.turn(x, np.array([p, q]), cos, sin, None, 0.0, False, pairs)
        return y, np.einsum("hd,hd->h", y[0], y[1])
    y, dot = at(3, 11)
    np.testing.assert_allclose((y ** 2).sum(2), (x ** 2).sum(2), rtol=1e-12)
    np.testing.assert_allclose(dot, at(8, 16)[1], rtol=1e-12)
    n = orc.turn(x, np.array([0, 0]), None, None, 2 * np.ones(8), 0.0, True, pairs)
    np.testing.assert_allclose((n ** 2).mean(2), 4.0, rtol=1e-12)


def test_attention_of_equal_keys_is_the_mean_and_windows_cut():
    keys = np.ones((4, 2, 1, 4))
    values = np.arange(4 * 2 * 4, dtype=np.float64).reshape(4, 2, 1, 4)
    tables = np.array([[2, 0, 3]])
    rows = values.reshape(-1, 4)[[4, 5, 0, 1, 6]]
    out, lse, _ = orc.attention(np.ones((2, 2, 4)), keys, values, tables, np.array([0, 2]), np.array([5]), 0.5, 0)
    np.testing.assert_allclose(out[1, 0], rows.mean(0))
    np.testing.assert_allclose(out[0, 1], rows[:4].mean(0))
    np.testing.assert_allclose(lse[1], 2 + np.log(5))
    out, lse, _ = orc.attention(np.ones((2, 2, 4)), keys, values, tables, np.array([0, 2]), np.array([5]), 0.5, 2)
    np.testing.assert_allclose(out[1, 0], rows[3:].mean(0))
    out, lse, _ = orc.attention(np.ones((2, 2, 4)), keys, values, tables, np.array([0, 2]), np.array([-1]), 0.5, 0)
    assert (out == 0).all() and np.isneginf(lse).all()


def test_sample_filters():
    l = np.log(np.array([0.1, 0.4, 0.1, 0.25, 0.15]))
    assert orc.kept(l, 1.0, 0, 1.0, 0.0)[0].tolist() == [1, 3, 4, 0, 2]
    assert orc.kept(l, 1.0, 4, 1.0, 0.0)[0].tolist() == [1, 3, 4, 0]       # equal logits: the smaller index first
    assert orc.kept(l, 1.0, 0, 0.5, 0.0)[0].tolist() == [1, 3]
    assert orc.kept(l, 1.0, 2, 0.6, 0.0)[0].tolist() == [1]                # 0.4 of 0.65
    assert orc.kept(l, 1.0, 0, 1.0, 0.3)[0].tolist() == [1, 3, 4]
    assert orc.kept(l, 0.5, 0, 1.0, 0.3)[0].tolist() == [1, 3]             # squared shares
    assert orc.sample(np.array([-np.inf, np.nan]), None, 1.0, 0, 1.0, 0.0)[:2] == (-1, -np.inf)


def test_sample_is_a_draw_from_the_softmax():
    r = np.random.default_rng(3)
    p = np.array([0.05, 0.6, 0.2, 0.15])
    drawn = np.bincount([orc.sample(np.log(p), r.random(4), 1.0, 0, 1.0, 0.0)[0] for _ in range(20000)], minlength=4) / 20000
    # five standard deviations of a share
    assert (np.abs(drawn - p) < 5 * np.sqrt(p * (1 - p) / 20000)).all()
