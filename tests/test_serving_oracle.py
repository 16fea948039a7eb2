"""Pins of the serving oracle: closed forms, invariances and the oracle of the dense operators."""
import math

import numpy as np

from oracle import rf_oracle as O
from oracle import serving_oracle as S


def batch(seed, n, k, Hq, Hkv, d, page):
    r = np.random.default_rng(seed)
    per = [-(-x // page) for x in k]
    ids, table, at = r.permutation(sum(per)), np.full((len(k), max(per)), -1), 0
    for b, c in enumerate(per):
        table[b, :c] = ids[at:at + c]
        at += c
    starts = np.concatenate(([0], np.cumsum(n)))
    return (r.standard_normal((sum(n), Hq, d)), r.standard_normal((sum(per), page, Hkv, d)),
            r.standard_normal((sum(per), page, Hkv, d)), starts, np.array(k), table)


def test_paged_attention_is_dense_attention_of_the_gathered_keys():
    n, k = [3, 1, 4], [10, 5, 4]
    q, K, V, starts, lens, table = batch(1, n, k, 4, 2, 8, 3)
    for causal in (False, True):
        o, spread, _ = S.attention(q, K, V, starts, lens, table, 0.3, causal)
        for b in range(3):
            at = [(table[b, j // 3], j % 3) for j in range(k[b])]
            kk, vv = (np.stack([c[x] for x in at]).transpose(1, 0, 2)[None] for c in (K, V))
            qq = q[starts[b]:starts[b + 1]].transpose(1, 0, 2)[None]
            want = O.attention(qq, kk, vv, 0.3, causal)[0].transpose(1, 0, 2)
            assert np.allclose(o[starts[b]:starts[b + 1]], want, rtol=1e-12, atol=1e-14)
        assert (spread >= np.abs(o) - 1e-12).all()


def test_rows_that_see_nothing_are_zero_and_unseen_nan_does_not_show():
    q, K, V, starts, lens, table = batch(2, [4], [2], 2, 1, 4, 2)
    o, _, _ = S.attention(q, K, V, starts, lens, table, 1.0, True)
    assert (o[:2] == 0).all() and np.isfinite(o).all()
    V[table[0, 0], 1] = np.nan                    # key 1: seen by the last token alone
    o, _, _ = S.attention(q, K, V, starts, lens, table, 1.0, True)
    assert np.isfinite(o[:3]).all() and np.isnan(o[3]).all()


def test_rotation_turns_planes_and_scores_depend_on_distances():
    r = np.random.default_rng(3)
    d, rot = 12, 8
    freq = 10.0 ** (-np.arange(4) / 3)
    x, y = r.standard_normal((2, 1, d))
    for inter in (False, True):
        turn = lambda v, p: S.rotated(v, np.cos(p * freq), np.sin(p * freq), inter)  # noqa: E731
        assert np.allclose((turn(x, 7) ** 2).sum(), (x ** 2).sum()) and np.allclose(turn(x, 7)[:, rot:], x[:, rot:])
        assert np.allclose((turn(x, 9) * turn(y, 4)).sum(), (turn(x, 25) * turn(y, 20)).sum())
        assert np.allclose(turn(x, 0), x)
        e = np.zeros((1, d)); e[0, 0] = 1.0       # a quarter turn of plane 0 takes its first axis to its second
        quarter = S.rotated(e, np.array([0.0, 1, 1, 1]), np.array([1.0, 0, 0, 0]), inter)
        assert quarter[0, 1 if inter else 4] == 1.0 and quarter[0, 0] == 0.0


def test_norm_and_slots():
    r = np.random.default_rng(4)
    q, k, v = r.standard_normal((5, 2, 8)), r.standard_normal((5, 1, 8)), r.standard_normal((5, 1, 8))
    g = 1 + 0.1 * r.standard_normal(8)
    out, slots = S.append(q, k, v, g, None, 0.0, None, None, False, np.array([0, 2, 4]), np.array([3, 1]), np.array([[5, 9], [2, 0]]), 2)
    assert np.allclose((out[:2] / g) ** 2 @ np.ones(8), 8)                       # unit mean square
    assert sorted(slots) == [(2, 0), (5, 1), (9, 0)]                             # keys 1, 2 of the first, 0 of the second
    assert np.array_equal(slots[9, 0][0], k[1]) and np.array_equal(slots[2, 0][1], v[3])
    assert (out[2] == 0).all() and np.isnan(out[4]).all()                        # no position; no sequence


def test_verified_tokens_have_the_targets_distribution():
    """Over a fine grid of both random numbers, the first token out is distributed as p whatever q is."""
    V, N = 4, 400
    p, q = np.array([0.1, 0.2, 0.3, 0.4]), np.array([0.4, 0.3, 0.2, 0.1])
    grid = (np.arange(N) + 0.5) / N
    count = np.zeros(V)
    for x in range(V):
        for u in grid[::8]:
            for s in grid[::8]:
                out, acc, _ = S.verify(np.stack([p, p]), np.stack([q, q]), np.array([x, 0]), np.array([u, 0]), np.array([s]), np.array([0, 2]))
                assert (out[0] == x) if acc[0] else out[1] == -1
                count[out[0]] += q[x]
    assert np.allclose(count / count.sum(), p, atol=2.5 / (N / 8))


def test_verify_by_hand():
    p = np.array([[0.5, 0.5, 0.0], [0.0, 0.25, 0.75], [0.2, 0.3, 0.5]])
    q = np.array([[1.0, 0.0, 0.0], [0.5, 0.5, 0.0], [0.0, 0.0, 0.0]])
    run = lambda x, ua, us, q=q: tuple(a.tolist() for a in S.verify(p, q, np.array(x), np.array(ua), np.array([us]), np.array([0, 3]))[:2])  # noqa: E731
    assert run([0, 1, 9], [0.4, 0.4, 0], 0.6) == ([0, 1, 2], [2])               # 0.4 < 0.5; 0.2 < 0.25; then p_2: 0.5 < 0.6
    assert run([0, 1, 9], [0.5, 0.4, 0], 0.6) == ([1, -1, -1], [0])             # 0.5 is not below 0.5; rest (0, 0.5, 0)
    assert run([0, 1, 9], [0.1, 0.9, 0], 0.0) == ([0, 2, -1], [1])              # rest (0, 0, 0.75)
    assert run([1, 2, 9], [0.1, 0.9, 0], 0.9, None) == ([1, 1, -1], [1])        # without q: the draft leaves, (0, 0.25, -)
    assert run([0, 1, 9], [0.4, 0.4, 0], math.nan)[1] == [2]


def test_no_draft_is_probability_one_at_the_drafted_token():
    """Also where the target is not normalised, or not a number there."""
    r = np.random.default_rng(6)
    for at_x in (0.1, 0.0, 3.0, math.inf, math.nan):
        for u in (0.5, math.nan):
            p, x = r.random((2, 6)), np.array([4, 0])
            p[0, 4] = at_x
            args = x, np.array([u, 0]), np.array([0.9]), np.array([0, 2])
            alone, given = S.verify(p, None, *args), S.verify(p, np.eye(6)[x], *args)
            assert all(np.array_equal(a, b) for a, b in zip(alone, given))
            if not math.isfinite(at_x) and alone[1][0] == 0:
                assert alone[0][0] == -1
