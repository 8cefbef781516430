"""The 64-bit forms of the serving operators against closed forms, brute force and invariants."""
import itertools
import math
import random

import numpy as np
import pytest

from oracle import serving as ref


def angles(n, rot):
    a = np.arange(n)[:, None] * 10.0 ** (-np.arange(rot // 2))
    return np.cos(a), np.sin(a)


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_keeps_lengths_and_depends_on_the_distance(pairs):
    """|R x| = |x|, and (R_i q) . (R_j k) is a function of i - j."""
    rng = np.random.default_rng(0)
    cos, sin = angles(40, 8)
    q, k = rng.normal(size=(2, 1, 1, 12))
    r = lambda x, i: ref.norm_rope(x, None, 0, cos[i:i + 1], sin[i:i + 1], pairs)[0, 0]  # noqa: E731
    assert np.allclose(np.linalg.norm(r(q, 17)), np.linalg.norm(q))
    assert np.array_equal(r(q, 0), q[0, 0]) and np.array_equal(r(q, 5)[8:], q[0, 0, 8:])
    for i, j in ((3, 1), (30, 28), (39, 37)):
        assert np.allclose(r(q, i) @ r(k, j), r(q, 2) @ r(k, 0))


def test_the_norm_has_mean_square_one():
    x = np.random.default_rng(1).normal(size=(3, 2, 16)) * 50
    y = ref.norm_rope(x, np.ones(16), 0.0, np.zeros((3, 0)), np.zeros((3, 0)), False)
    assert np.allclose((y * y).mean(-1), 1) and np.allclose(y / x, (y / x)[..., :1])


def test_attention_closed_forms():
    v = np.arange(12.0).reshape(6, 2)
    seen = ref.visible(4, 6, 0, 0)
    out, lse, _, _ = ref.attend_row(np.zeros(3), np.ones((6, 3)), v, seen, 1.0)
    assert np.allclose(out, v[:5].mean(0)) and math.isclose(lse, math.log(5))   # equal scores: the mean
    k = np.zeros((6, 3))
    k[2] = 1e4
    out, _, _, _ = ref.attend_row(np.ones(3), k, v, seen, 1.0)
    assert np.allclose(out, v[2])                                               # one large score: its value
    out, lse, _, _ = ref.attend_row(np.ones(3), k, v, np.zeros(6, bool), 1.0)
    assert np.array_equal(out, np.zeros(2)) and lse == -math.inf


def test_visible_keys():
    assert ref.visible(5, 8, 0, 0).tolist() == [1, 1, 1, 1, 1, 1, 0, 0]
    assert ref.visible(5, 8, 2, 0).tolist() == [0, 0, 0, 0, 1, 1, 0, 0]
    assert ref.visible(5, 8, 2, 1).tolist() == [1, 0, 0, 0, 1, 1, 0, 0]
    assert ref.visible(1, 8, 2, 4).tolist() == [1, 1, 0, 0, 0, 0, 0, 0]         # a sink in the future is not seen
    assert not ref.visible(-1, 3, 0, 0).any()


@pytest.mark.parametrize("seed", range(20))
def test_pages_invariants_over_random_calls(seed):
    """refs counts the table's entries, every token of a sequence keeps its contents through
    copies and moves, and a call without enough pages changes nothing."""
    r = random.Random(seed)
    p = ref.Pages(r.randint(4, 60), r.choice((1, 2, 4)), 6, 8)
    text = [[] for _ in range(6)]  # what each sequence has written
    mark = itertools.count(1)
    for _ in range(120):
        s, d = r.randrange(6), r.randrange(6)
        what = r.choice(("extend", "extend", "fork", "cut", "compact"))
        before = (list(p.refs), [list(x) for x in p.table], list(p.len))
        if what == "extend":
            a = r.randint(0, 6)
            missing, left_out = p.extend([s], [a])
            if missing or left_out:
                assert before == (p.refs, p.table, p.len)
            else:
                for j in range(len(text[s]), len(text[s]) + a):
                    text[s].append(next(mark))
                    p.data[p.table[s][j // p.page]][j % p.page] = text[s][-1]
        elif what == "fork":
            missing, left_out = p.fork([s], [d])
            if missing or left_out:
                assert before == (p.refs, p.table, p.len)
            else:
                text[d] = list(text[s])
        elif what == "cut":
            n = r.randint(0, 40)
            p.free([s], [n])
            text[s] = text[s][:n]
        else:
            n = p.compact()
            assert all(p.refs[:n]) and not any(p.refs[n:])
        assert p.len == [len(t) for t in text]
        for q in range(len(p.refs)):
            assert p.refs[q] == sum(row.count(q) for row in p.table)
        for t, row in zip(text, p.table):
            assert [p.data[row[j // p.page]][j % p.page] for j in range(len(t))] == t


def test_sampling_without_limits_is_the_inverse_of_the_distribution():
    x = np.log(np.array([0.1, 0.2, 0.3, 0.4]))
    shares = np.exp(x - x.max()).astype(np.float32)
    for u, want in ((0.0, 0), (0.09, 0), (0.11, 1), (0.29, 1), (0.31, 2), (0.59, 2), (0.61, 3), (0.999, 3), (1.0, 3)):
        assert ref.sample(x, shares, u)[0] == want
    assert math.isclose(ref.sample(x, shares, 0.61)[1], 0.4, rel_tol=1e-6)


def test_sampling_limits_by_hand():
    x = np.log(np.array([0.1, 0.2, 0.3, 0.4]))
    s = np.exp(x - x.max()).astype(np.float32)
    assert ref.sample(x, s, 0.0, top_k=2) == (2, pytest.approx(3 / 7), 2)
    assert ref.sample(x, s, 0.0, top_p=0.39)[::2] == (3, 1)
    assert ref.sample(x, s, 0.0, top_p=0.41)[::2] == (2, 2)
    assert ref.sample(x, s, 0.0, top_k=3, top_p=0.8)[::2] == (1, 3)   # of the top 3's 0.9: 0.4 + 0.3 are below 0.72
    assert ref.sample(x, s, 0.0, min_p=0.6)[::2] == (2, 2)
    assert ref.sample(x, s, 0.99, temperature=0.0) == (3, 1.0, 1)
    ties = np.zeros(5)
    assert ref.sample(ties, np.ones(5, np.float32), 0.99, top_k=2)[::2] == (1, 2)
    assert ref.sample(np.full(3, -np.inf), np.ones(3), 0.5) == (-1, 0.0, 0)


def test_extension_of_a_sequence_that_ends_in_pages_it_gave_back():
    """12 tokens in pages of 4; the first 8 are given back, and the sequence is cut to 6: tokens 6 and 7
    need a page again."""
    p = ref.Pages(8, 4, 2, 5)
    assert p.extend([0, 1], [12, 3]) == (0, 0)
    p.free([0], [0], [8])
    p.free([0], [6])
    assert p.table[0] == [-1] * 5 and p.len[0] == 6 and p.refs == [0, 0, 0, 1, 0, 0, 0, 0]
    assert p.extend([0], [0]) == (0, 0) and p.table[0] == [-1] * 5
    assert p.extend([0, 1], [3, 1]) == (0, 0)
    assert p.table[0] == [-1, 0, 1, -1, -1] and p.len[0] == 9 and p.refs[:4] == [1, 1, 0, 1]
