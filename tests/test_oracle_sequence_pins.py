"""CPU-only pins of oracle/sequence_ops.py: closed forms, sums row against row, and differences of a scalar loss."""
import numpy as np
import pytest

from oracle import sequence_ops as so

OFFSETS = np.array([0, 5, 5, 6, 13])
LOG_DECAY = np.array([0.0, -0.3, -np.inf])


def _inputs(seed=0, H=3, D=4):
    rng = np.random.default_rng(seed)
    n, B = OFFSETS[-1], len(OFFSETS) - 1
    return [rng.standard_normal((n, H, D)) for _ in range(4)] + [rng.standard_normal((B, H, D, D)) for _ in range(2)]


def test_linear_attention_is_the_decayed_sum_over_earlier_rows():
    q, k, v, _, S0, _ = _inputs()
    out, final = so.linear_attention(q, k, v, LOG_DECAY, OFFSETS, 0.7, S0)
    for b in range(4):
        lo, hi = OFFSETS[b], OFFSETS[b + 1]
        for h, g in enumerate(np.exp(LOG_DECAY)):
            for i in range(hi - lo):
                want = g ** (i + 1) * q[lo + i, h] @ S0[b, h] + sum(g ** (i - j) * (q[lo + i, h] @ k[lo + j, h]) * v[lo + j, h] for j in range(i + 1))
                np.testing.assert_allclose(out[lo + i, h], 0.7 * want, rtol=1e-12, atol=1e-12)
            want = g ** (hi - lo) * S0[b, h] + sum((g ** (hi - lo - 1 - j) * np.outer(k[lo + j, h], v[lo + j, h]) for j in range(hi - lo)), np.zeros((4, 4)))
            np.testing.assert_allclose(final[b, h], want, rtol=1e-12, atol=1e-12)


def test_states_hand_a_sample_over():
    q, k, v, _, S0, _ = _inputs()
    whole, final = so.linear_attention(q, k, v, LOG_DECAY, OFFSETS, 0.7, S0)
    cut = np.array([0, 2, 2, 2, 2])
    rows = slice(OFFSETS[0], OFFSETS[1])
    first, state = so.linear_attention(q[rows], k[rows], v[rows], LOG_DECAY, cut, 0.7, S0)
    rest, last = so.linear_attention(q[rows][2:], k[rows][2:], v[rows][2:], LOG_DECAY, np.array([0, 3, 3, 3, 3]), 0.7, state)
    np.testing.assert_allclose(np.concatenate([first[:2], rest[:3]]), whole[rows], rtol=1e-12)
    np.testing.assert_allclose(last[0], final[0], rtol=1e-12)


def _difference(loss, x, at, step=1e-6):
    up, down = x.copy(), x.copy()
    up[at] += step
    down[at] -= step
    return (loss(up) - loss(down)) / (2 * step)


def test_linear_attention_gradients_are_differences():
    q, k, v, dout, S0, dS = _inputs(1)
    grads = so.linear_attention_backward(q, k, v, dout, LOG_DECAY, OFFSETS, 0.7, S0, dS)

    def loss(**changed):
        a = dict(q=q, k=k, v=v, S0=S0, **{})
        a.update(changed)
        out, final = so.linear_attention(a["q"], a["k"], a["v"], LOG_DECAY, OFFSETS, 0.7, a["S0"])
        return (out * dout).sum() + (final * dS).sum()

    rng = np.random.default_rng(2)
    for name, x, grad in zip(("q", "k", "v", "S0"), (q, k, v, S0), grads):
        for _ in range(20):
            at = tuple(rng.integers(0, s) for s in x.shape)
            assert abs(_difference(lambda y: loss(**{name: y}), x, at) - grad[at]) < 1e-7, (name, at)


def test_layer_norm_and_its_gradients():
    rng = np.random.default_rng(3)
    x, w, b, dy = rng.standard_normal((6, 5)) * 3 + 1, rng.standard_normal(5), rng.standard_normal(5), rng.standard_normal((6, 5))
    y, mean, rstd = so.layer_norm(x, None, None, 0.0)
    np.testing.assert_allclose(y.mean(-1), 0, atol=1e-14)
    np.testing.assert_allclose(y.var(-1), 1, rtol=1e-12)
    np.testing.assert_allclose(so.layer_norm(x, w, b, 0.0)[0], y * w + b, rtol=1e-12)
    np.testing.assert_allclose(so.layer_norm(np.full((1, 5), 7.0), None, b, 1e-5)[0], b[None])   # no variance: eps decides
    dx, dw, db = so.layer_norm_backward(x, w, dy, 1e-3)
    loss = lambda x, w, b: (so.layer_norm(x, w, b, 1e-3)[0] * dy).sum()
    for at in np.ndindex(x.shape):
        assert abs(_difference(lambda z: loss(z, w, b), x, at) - dx[at]) < 1e-7
    for i in range(5):
        assert abs(_difference(lambda z: loss(x, z, b), w, (i,)) - dw[i]) < 1e-7
        assert abs(_difference(lambda z: loss(x, w, z), b, (i,)) - db[i]) < 1e-7


@pytest.mark.parametrize("ids", [[3, 0, 3, 3, -1, 5, 6, 2], []])
def test_embedding_and_its_gradient(ids):
    rng = np.random.default_rng(4)
    table, dout = rng.standard_normal((6, 3)), rng.standard_normal((len(ids), 3))
    ids = np.array(ids, dtype=np.int64)
    out = so.embedding(table, ids, 2.0)
    for i, v in enumerate(ids):
        np.testing.assert_array_equal(out[i], 2.0 * table[v] if 0 <= v < 6 else np.zeros(3))
    grad = so.embedding_backward(dout, ids, 6, 2.0)
    for at in np.ndindex(table.shape):
        assert abs(_difference(lambda t: (so.embedding(t, ids, 2.0) * dout).sum(), table, at) - grad[at]) < 1e-7
