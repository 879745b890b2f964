"""Pins of the sequence operators' oracle (oracle/seq.py): closed forms,
differences and symmetries. CPU only."""
import numpy as np
import pytest

from oracle import seq


def _rng(s):
    return np.random.Generator(np.random.PCG64(s))


@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
def test_rope_is_a_rotation_of_relative_positions(pairing):
    """Lengths stay, inverse undoes it, and q.k depends on the positions' difference only."""
    r = _rng(1)
    sections, freqs = (3, 2), r.uniform(0.1, 1.0, 5)
    q, k = r.standard_normal((2, 7, 12))
    pos = r.integers(-50, 50, (2, 7))
    a = seq.rope(q, pos, sections, freqs, pairing)
    assert np.allclose((a ** 2).sum(1), (q ** 2).sum(1), atol=1e-12)
    assert np.array_equal(a[:, 10:], q[:, 10:])
    assert np.allclose(seq.rope(a, pos, sections, freqs, pairing, inverse=True), q, atol=1e-12)
    b = seq.rope(k, pos, sections, freqs, pairing)
    c, d = (seq.rope(x, pos + np.array([[5], [-9]]), sections, freqs, pairing) for x in (q, k))
    assert np.allclose((a * b).sum(1), (q * k).sum(1), atol=1e-11)
    assert np.allclose(a @ b.T, c @ d.T, atol=1e-11)


def test_rope_pair_by_hand():
    y = seq.rope(np.array([[1.0, 0.0, 0.0, 2.0]]), np.array([[1], [1]]), (1, 1), (np.pi / 2, np.pi))
    assert np.allclose(y, [[0.0, 1.0, 0.0, -2.0]], atol=1e-15)
    y = seq.rope(np.array([[1.0, 0.0, 0.0, 2.0]]), np.array([[1], [1]]), (1, 1), (np.pi / 2, np.pi), "halves")
    assert np.allclose(y, [[0.0, 0.0, 1.0, -2.0]], atol=1e-15)


def test_grid_positions():
    p = seq.grid_positions(7, (2, 3, 2), (10, 0, -1))
    assert p[:, 0].tolist() == [10, 0, -1] and p[:, 6].tolist() == [11, 0, -1]
    assert p[:, 5].tolist() == [10, 2, 0]


def test_visible_by_hand():
    see = seq.visible(4, 6, left=1, sinks=1, causal=True)  # queries at 2, 3, 4, 5
    want = [[1, 1, 1, 0, 0, 0], [1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    assert np.array_equal(see, np.array(want, bool))
    assert not seq.visible(5, 2, causal=True)[:3].any()  # positions -3, -2, -1
    assert seq.visible(3, 3, left=0, right=0, sinks=0).tolist() == np.eye(3, dtype=bool).tolist()


@pytest.mark.parametrize("kw", [dict(left=2, sinks=1, causal=True), dict(left=1, right=2), dict(causal=True)])
def test_gradients_against_differences(kw):
    r = _rng(3)
    q, k, v, do = r.standard_normal((5, 4)), r.standard_normal((7, 4)), r.standard_normal((7, 4)), r.standard_normal((5, 4))
    see, h = seq.visible(5, 7, **kw), 1e-6
    g = seq.attend_backward(q, k, v, do, see, 0.5)
    f = lambda *x: (seq.attend(*x, see, 0.5)[0] * do).sum()  # noqa: E731
    for n, x in enumerate((q, k, v)):
        for i in np.ndindex(x.shape):
            d = np.zeros_like(x)
            d[i] = h
            up, dn = [q, k, v], [q, k, v]
            up[n], dn[n] = x + d, x - d
            assert abs((f(*up) - f(*dn)) / (2 * h) - g[n][i]) < 1e-8


def test_hidden_rows_are_zero():
    r = _rng(4)
    q, k, v = r.standard_normal((3, 4)), r.standard_normal((1, 4)), r.standard_normal((1, 4))
    see = seq.visible(3, 1, causal=True)
    o, lse, P = seq.attend(q, k, v, see, 1.0)
    assert not o[:2].any() and np.all(lse[:2] == -np.inf) and np.allclose(o[2], v[0])
    assert not seq.attend_backward(q, k, v, np.ones((3, 4)), see, 1.0)[0].any()
