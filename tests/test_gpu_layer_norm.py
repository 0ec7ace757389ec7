"""Layer norm of jagged rows against oracle/sequence_ops.py (fp64).

Bounds: an output of bf16 is off by at most 2^-8 of itself for its rounding.  In fp32, with u = 2^-24 and M the largest |x| of a row: the mean is off by at
most (log2 of the additions + ITEMS) u M, less than 32 u M here, x - mean by that much too, the statistics' relative error is as small: hat is off by
64 u (M rstd + |hat|) at most and what is made of it by that times its factors.  Sums over rows: their additions u each, (rows / 64 + 64) u of the
sum of absolute values at most, the terms' own errors added.
"""
import numpy as np
import pytest
import torch

from oracle import sequence_ops as so
from helpers import f64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float32]


def make(rows, reps, N, dtype, seed=0, mean=1.0, guard=0):
    rng = np.random.default_rng(seed)
    t = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32)).to(dtype).cuda()
    x, dy = t(rng.standard_normal((rows + guard, reps, N)) * 2 + mean), t(rng.standard_normal((rows + guard, reps, N)))
    return x, t(1 + 0.2 * rng.standard_normal(N)), t(rng.standard_normal(N)), dy


def check(x, w, b, dy, got, eps=1e-5):
    """got: y, mean, rstd, dx, dweight, dbias (any of them None)"""
    half = 2.0 ** -8 if x.dtype == torch.bfloat16 else U
    xs, dys = f64(x), f64(dy)
    ws, bs = (None if t is None else f64(t) for t in (w, b))
    y, mean, rstd = so.layer_norm(xs, ws, bs, eps)
    hat = so.layer_norm(xs, None, None, eps)[0]
    dx, dw, db = so.layer_norm_backward(xs, ws, dys, eps)
    M = np.abs(xs).max(-1, keepdims=True)
    d_hat = 64 * U * (M * rstd[..., None] + np.abs(hat)) + 1e-30
    aw = 1.0 if ws is None else np.abs(ws)
    bounds = {"y": half * np.abs(y) + d_hat * aw + 2 * U * (np.abs(hat) * aw + np.abs(y)), "mean": 32 * U * M[..., 0] + 1e-30, "rstd": 64 * U * rstd * (1 + M[..., 0] * rstd)}
    dhat = np.abs(dys) * aw
    reach = rstd[..., None] * (dhat + dhat.mean(-1, keepdims=True) + np.abs(hat) * (dhat * np.abs(hat)).mean(-1, keepdims=True))
    spread = rstd[..., None] * (d_hat * (dhat * np.abs(hat)).mean(-1, keepdims=True) + np.abs(hat) * (dhat * d_hat).mean(-1, keepdims=True))
    rel = (64 + M * rstd[..., None]) * U * 2
    bounds["dx"] = half * np.abs(dx) + rel * reach + 2 * spread + 1e-30
    lead = (0, 1)
    additions = (xs.shape[0] * xs.shape[1] / 64 + 64) * U
    bounds["dweight"] = half * np.abs(dw) + additions * (np.abs(dys) * np.abs(hat)).sum(lead) + (np.abs(dys) * d_hat).sum(lead) + 1e-30
    bounds["dbias"] = half * np.abs(db) + additions * np.abs(dys).sum(lead) + 1e-30
    for (name, bound), g, r in zip(((k, bounds[k]) for k in ("y", "mean", "rstd", "dx", "dweight", "dbias")), got, (y, mean, rstd, dx, dw, db)):
        if g is None:
            continue
        err = np.abs(f64(g) - r)
        assert np.isfinite(err).all(), f"{name}: not finite"
        assert (err <= bound).all(), f"{name}: {err.max()}, {(err / bound).max()} of the bound"


def both(x, w, b, dy, offsets=None, eps=1e-5):
    from paper_2409_15373_amd import binding
    y, mean, rstd = binding.jfa_layer_norm(x, w, b, offsets, eps)
    dx, dw, db = binding.jfa_layer_norm_backward(x, w, dy, mean, rstd, offsets, normalized_shape=x.shape[-1:])
    torch.cuda.synchronize()
    return y, mean, rstd, dx, dw, db


# every spread of a row: 16-byte vectors over part of a wave, a wave, several vectors each, long rows; single elements likewise
@pytest.mark.parametrize("N", [1, 2, 7, 8, 32, 33, 63, 64, 100, 128, 129, 256, 257, 511, 512, 513, 520, 1000, 1024, 2048, 2056, 4096, 4104, 5001, 8200])
@pytest.mark.parametrize("dtype", TYPES)
def test_row_lengths(dtype, N):
    x, w, b, dy = make(37, 1, N, dtype, seed=N)
    check(x, w, b, dy, both(x, w, b, dy))


@pytest.mark.parametrize("rows", [1, 2, 3, 63, 64, 65, 1000, 9000])
@pytest.mark.parametrize("N", [48, 65, 8200])
@pytest.mark.parametrize("dtype", TYPES)
def test_row_counts(dtype, N, rows):
    if rows * N > 10 ** 7:
        rows = 1100
    x, w, b, dy = make(rows, 1, N, dtype, seed=rows)
    check(x, w, b, dy, both(x, w, b, dy))


@pytest.mark.parametrize("dtype", TYPES)
def test_heads_of_a_row_each_for_itself(dtype):
    from paper_2409_15373_amd import binding
    x, w, b, dy = make(300, 3, 64, dtype, seed=2)
    check(x, w, b, dy, both(x, w, b, dy))
    flat = x.reshape(300, 192)
    wide = binding.jfa_layer_norm(x, w.repeat(3).view(3, 64), b.repeat(3).view(3, 64))[0]   # and all of a row together
    assert torch.equal(wide.view(300, 192), binding.jfa_layer_norm(flat, w.repeat(3), b.repeat(3))[0])


@pytest.mark.parametrize("N", [64, 65, 5001])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_are_not_there(dtype, N):
    """Rows from offsets[B] on are neither read nor written, and add nothing to the sums."""
    from paper_2409_15373_amd import binding
    x, w, b, dy = make(200, 2, N, dtype, seed=N, guard=5)
    off = torch.tensor([0, 150, 150, 200], device="cuda")
    x[200:], dy[200:] = float("nan"), float("nan")
    y, dx = torch.full_like(x, 777.0), torch.full_like(x, 777.0)
    _, mean, rstd = binding.jfa_layer_norm(x, w, b, off, y=y)
    _, dw, db = binding.jfa_layer_norm_backward(x, w, dy, mean, rstd, off, dx=dx)
    torch.cuda.synchronize()
    assert (y[200:] == 777.0).all() and (dx[200:] == 777.0).all()
    check(x[:200], w, b, dy[:200], (y[:200], mean[:200], rstd[:200], dx[:200], dw, db))


@pytest.mark.parametrize("N", [64, 65, 5001])
def test_nothing_to_normalise(N):
    """No rows at all, and offsets that end at zero: sums of nothing are zeros."""
    from paper_2409_15373_amd import binding
    x, w, b, dy = make(4, 1, N, torch.float32)
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    y = torch.full_like(x, 777.0)
    _, mean, rstd = binding.jfa_layer_norm(x, w, b, off, y=y)
    _, dw, db = binding.jfa_layer_norm_backward(x, w, dy, mean, rstd, off)
    assert (y == 777.0).all() and not dw.any() and not db.any()
    y, mean, rstd = binding.jfa_layer_norm(x[:0], w, b)
    dx, dw, db = binding.jfa_layer_norm_backward(x[:0], w, dy[:0], mean, rstd)
    assert y.shape == dx.shape == (0, 1, N) and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [96, 77, 8200])
def test_without_weight_or_bias(dtype, N):
    x, w, b, dy = make(70, 1, N, dtype, seed=1)
    check(x, None, None, dy, both(x, None, None, dy))
    check(x, w, None, dy, both(x, w, None, dy))
    check(x, None, b, dy, both(x, None, b, dy))


@pytest.mark.parametrize("N", [128, 129, 5001])
def test_rows_with_a_mean_far_from_zero_and_without_variance(N):
    x, w, b, dy = make(50, 1, N, torch.float32, seed=3, mean=1000.0)
    x[7] = 3.25    # no variance: eps decides
    x[8] = 0.0
    check(x, w, b, dy, both(x, w, b, dy))
    check(x, w, b, dy, both(x, w, b, dy, eps=0.1), eps=0.1)


def test_a_row_that_is_not_finite_reaches_no_other():
    x, w, b, dy = make(50, 1, 96, torch.bfloat16, seed=3)
    clean = both(x, w, b, dy)
    x[9, 0, 4], x[20] = float("nan"), float("inf")
    got = both(x, w, b, dy)
    rest = torch.ones(50, dtype=torch.bool, device="cuda")
    rest[[9, 20]] = False
    for i in (0, 3):
        assert torch.equal(got[i][rest], clean[i][rest]) and torch.isnan(got[i][~rest]).all()
    assert torch.equal(got[5], clean[5])


@pytest.mark.parametrize("N", [64, 512])
def test_tensors_that_start_anywhere(N):
    """Views whose first element is not on 16 bytes give what aligned copies give, to the last place of a sum in another order."""
    from paper_2409_15373_amd import binding
    x, w, b, dy = make(33, 1, N, torch.float32, seed=4)
    shifted = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)
    xs, ws, bs, dys = (shifted(t) for t in (x, w, b, dy))
    assert xs.data_ptr() % 16 == 4
    check(x, w, b, dy, both(xs, ws, bs, dys))
    check(x, w, b, dy, both(x, ws, b, dy))


@pytest.mark.parametrize("dtype", TYPES)
def test_through_autograd(dtype):
    from paper_2409_15373_amd import binding
    from paper_2409_15373_amd.autograd import jagged_layer_norm
    x, w, b, dy = make(90, 2, 64, dtype, seed=5)
    off = torch.tensor([0, 40, 90], device="cuda")
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    y = jagged_layer_norm(*leaves, off)
    strided = dy.transpose(1, 2).contiguous().transpose(1, 2)
    got = (y,) + torch.autograd.grad(y, leaves, strided)
    ref = both(x, w, b, dy, off)
    assert all(torch.equal(a, b) for a, b in zip(got, (ref[0], ref[3], ref[4], ref[5])))
    # gradients of some only
    y = jagged_layer_norm(x, leaves[1], b, off)
    assert torch.equal(torch.autograd.grad(y, leaves[1], dy)[0], ref[4])
    y = jagged_layer_norm(leaves[0])   # neither weight nor bias
    (dx,) = torch.autograd.grad(y, leaves[0], dy)
    check(x, None, None, dy, (y, None, None, dx, None, None))


def test_gradients_are_differences():
    from paper_2409_15373_amd.autograd import jagged_layer_norm
    x, w, b, dy = make(20, 1, 40, torch.float32, seed=6)
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    loss = lambda: (jagged_layer_norm(*leaves).double() * dy.double()).sum()
    grads = torch.autograd.grad(loss(), leaves)
    gen = torch.Generator(device="cuda").manual_seed(0)
    for leaf, grad in zip(leaves, grads):
        step = torch.randn(leaf.shape, device="cuda", generator=gen) * 1e-2
        with torch.no_grad():
            leaf += step
            up = loss()
            leaf -= 2 * step
            down = loss()
            leaf += step
        want = 2 * (grad.double() * step.double()).sum()
        assert abs((up - down - want).item()) <= 2e-3 * max(1.0, abs(want.item()))   # third order: 1e-6 of the terms; rounding: 800 times 2^-23


def test_a_captured_step_replays_to_the_eager_results():
    x, w, b, dy = make(700, 1, 256, torch.bfloat16, seed=7)
    eager = [t.clone() for t in both(x, w, b, dy)]
    g = torch.cuda.CUDAGraph()
    from paper_2409_15373_amd import binding
    with torch.cuda.graph(g):
        y, mean, rstd = binding.jfa_layer_norm(x, w, b)
        results = (y, mean, rstd) + binding.jfa_layer_norm_backward(x, w, dy, mean, rstd)
    for _ in range(3):
        for t in results:
            t.fill_(float("nan"))
        g.replay()
        both(x, w, b, dy)
        assert all(torch.equal(a, c) for a, c in zip(results, eager))


def test_what_is_refused():
    from paper_2409_15373_amd import binding
    from paper_2409_15373_amd.autograd import jagged_layer_norm
    x, w, b, dy = make(8, 1, 32, torch.float32)
    for bad in ((x, w[:16], b), (x, w, b[:16]), (x, w.bfloat16(), b), (x, w.cpu(), b), (x.transpose(1, 2).contiguous().transpose(1, 2).expand(8, 2, 32), w, b),
                (x, w, b, torch.tensor([0, 8], device="cuda", dtype=torch.int32)), (x, w, b, torch.tensor([0, 8]))):
        with pytest.raises(AssertionError):
            jagged_layer_norm(*bad)
    with pytest.raises(TypeError):
        jagged_layer_norm(x.half(), w.half(), b.half())
    _, mean, rstd = binding.jfa_layer_norm(x, w, b)
    for bad in ((x, w, dy[:4], mean, rstd), (x, w, dy.bfloat16(), mean, rstd), (x, w, dy, mean[:4], rstd), (x, w, dy, mean, rstd.double())):
        with pytest.raises(AssertionError):
            binding.jfa_layer_norm_backward(*bad)
