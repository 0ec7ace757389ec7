"""Embedding lookup into jagged rows against oracle/sequence_ops.py (fp64).

The lookup is one product in fp32, rounded once: it is compared for equality.  The gradient is a sum in fp32, rounded once: off by half a step of
its type (2^-8 of itself in bf16, 2^-24 in fp32) and 2^-24 of the absolute sum per addition, of which a row has at most as many as it has ids.
"""
import numpy as np
import pytest
import torch

from oracle import sequence_ops as so
from helpers import f64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float32]


def make(ids, V, N, dtype, seed=0):
    rng = np.random.default_rng(seed)
    t = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype).cuda()
    return t(V, N), torch.as_tensor(np.asarray(ids), dtype=torch.int64).cuda(), t(len(ids), N)


def check(table, ids, dout, scale, out, dtable):
    V = table.shape[0]
    inside = (ids >= 0) & (ids < V)
    want = torch.where(inside[:, None], table.float()[ids.long().clamp(0, V - 1)] * torch.tensor(scale, dtype=torch.float32, device="cuda"), 0.0).to(table.dtype)
    assert torch.equal(out, want)
    i, d = ids.cpu().numpy(), f64(dout)
    ref, absolute = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1]))
    keep = (i >= 0) & (i < V)
    np.add.at(ref, i[keep], d[keep] * scale)
    np.add.at(absolute, i[keep], np.abs(d[keep] * scale))
    count = np.bincount(i[keep], minlength=V)[:, None]
    half = 2.0 ** -8 if table.dtype == torch.bfloat16 else U
    err = np.abs(f64(dtable) - ref)
    bound = half * np.abs(ref) + (count + 1) * U * absolute
    assert np.isfinite(err).all() and (err <= bound).all(), f"dtable: {err.max()}"


def both(table, ids, dout, scale=1.5, offsets=None):
    from paper_2409_15373_amd import binding
    out = binding.jfa_embedding(table, ids, offsets, scale)
    dtable = binding.jfa_embedding_backward(dout, ids, table.shape[0], offsets, scale)
    torch.cuda.synchronize()
    return out, dtable


def test_the_oracle_adds_as_this_test_does():
    table, ids, dout = make([3, 1, 3, -1, 9, 0], 5, 4, torch.float32)
    check(table, ids, dout, 1.5, torch.from_numpy(so.embedding(f64(table), ids.cpu().numpy(), 1.5)).float().cuda(),
          torch.from_numpy(so.embedding_backward(f64(dout), ids.cpu().numpy(), 5, 1.5)).float().cuda())


@pytest.mark.parametrize("N", [1, 3, 8, 16, 31, 32, 64, 100, 128, 130, 256, 257, 512, 1000, 1024, 3000])
@pytest.mark.parametrize("dtype", TYPES)
def test_row_lengths(dtype, N):
    rng = np.random.default_rng(N)
    table, ids, dout = make(rng.integers(-2, 60, size=333), 57, N, dtype, seed=N)
    check(table, ids, dout, 1.5, *both(table, ids, dout))


@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 255, 4095, 4096, 4097, 20000])
@pytest.mark.parametrize("V", [1, 2, 1023, 1024, 70001])
def test_row_and_table_sizes(V, rows):
    """Table sizes on either side of a digit of the sort; positions on either side of its tiles."""
    rng = np.random.default_rng(rows + V)
    table, ids, dout = make(rng.integers(0, V, size=rows), V, 16, torch.float32, seed=rows)
    check(table, ids, dout, 1.5, *both(table, ids, dout))


@pytest.mark.parametrize("rows", [1023, 1024, 1025, 2047, 2048, 2049, 65535, 65536, 65537, 131073, 524288, 524289])
@pytest.mark.parametrize("V", [900, 5000])
def test_where_the_sort_changes_its_tiles(V, rows):
    from paper_2409_15373_amd import binding
    gen = torch.Generator(device="cuda").manual_seed(rows)
    ids = torch.randint(-1, V + 1, (rows,), device="cuda", generator=gen)
    ids[::7] = V // 2
    dout = torch.randint(-8, 9, (rows, 8), device="cuda", generator=gen).float()   # whole numbers: sums are exact
    inside = (ids >= 0) & (ids < V)
    want = torch.zeros(V, 8, device="cuda", dtype=torch.float64).index_add_(0, ids[inside], dout[inside].double())
    assert torch.equal(binding.jfa_embedding_backward(dout, ids, V).double(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [3, 1100000])
def test_frequent_ids(dtype, V):
    """One id for all positions but a few, runs of it that start and end anywhere in a block, and two that share the positions."""
    rng = np.random.default_rng(V)
    for rows, hot in ((12345, 1.0), (9000, 0.97), (200, 0.5), (64, 1.0), (4096, 1.0), (70000, 0.999)):
        ids = rng.integers(0, V, size=rows)
        ids[rng.random(rows) < hot] = V - 1
        table, ids, dout = make(ids, V, 24, dtype, seed=rows)
        check(table, ids, dout, 1.5, *both(table, ids, dout))
    ids = np.where(rng.random(20000) < 0.5, 0, 2)
    table, ids, dout = make(ids, V, 24, dtype, seed=1)
    check(table, ids, dout, 1.5, *both(table, ids, dout))


def test_ids_outside_the_table():
    big = [2 ** 40, -2 ** 40, 2 ** 32 + 1, 2 ** 32, -1, 7, 8, 2 ** 31, 0]   # also such as are inside in their lower 32 bits
    table, ids, dout = make(big, 8, 16, torch.float32)
    check(table, ids, dout, 1.5, *both(table, ids, dout))
    table, ids, dout = make([-1, 99, -1], 8, 16, torch.float32)
    out, dtable = both(table, ids, dout)
    assert not out.any() and not dtable.any()
    table[0] = float("nan")   # a row that nobody asks for
    assert not both(table, ids, dout)[0].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_ids_of_32_bits(dtype):
    rng = np.random.default_rng(1)
    table, ids, dout = make(rng.integers(-1, 5001, size=5000), 5000, 33, dtype)
    a, b = both(table, ids, dout), both(table, ids.int(), dout)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    odd = torch.cat([ids.new_zeros(1), ids])[1:]   # ids that start on 8 bytes
    assert torch.equal(both(table, odd, dout)[1], a[1])


def test_rows_that_are_not_there():
    from paper_2409_15373_amd import binding
    rng = np.random.default_rng(2)
    table, ids, dout = make(rng.integers(0, 50, size=505), 50, 40, torch.float32)
    off = torch.tensor([0, 100, 100, 500], device="cuda")
    dout[500:] = float("nan")
    out = torch.full_like(dout, 777.0)
    binding.jfa_embedding(table, ids, off, 1.5, out=out)
    dtable = binding.jfa_embedding_backward(dout, ids, 50, off, 1.5)
    assert (out[500:] == 777.0).all()
    check(table, ids[:500], dout[:500], 1.5, out[:500], dtable)
    nothing = torch.zeros(2, dtype=torch.int64, device="cuda")
    assert not binding.jfa_embedding_backward(dout, ids, 50, nothing, 1.5).any()
    assert not binding.jfa_embedding_backward(dout[:0], ids[:0], 50, None, 1.5).any()
    assert binding.jfa_embedding(table, ids[:0]).shape == (0, 40)


def test_the_same_every_time():
    rng = np.random.default_rng(3)
    ids = rng.integers(0, 300, size=30000)
    ids[::3] = 7
    table, ids, dout = make(ids, 300, 64, torch.float32)
    first = both(table, ids, dout)[1]
    assert all(torch.equal(both(table, ids, dout)[1], first) for _ in range(5))


def test_rows_of_several_dimensions_and_unaligned_tables():
    from paper_2409_15373_amd import binding
    rng = np.random.default_rng(4)
    table, ids, dout = make(rng.integers(0, 30, size=400), 30, 64, torch.float32)
    out, dtable = both(table, ids, dout)
    shaped = binding.jfa_embedding(table.view(30, 2, 32), ids, scale=1.5)
    assert shaped.shape == (400, 2, 32) and torch.equal(shaped.view(400, 64), out)
    assert torch.equal(binding.jfa_embedding_backward(dout.view(400, 2, 32), ids, 30, scale=1.5).view(30, 64), dtable)
    shifted = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)
    assert torch.equal(binding.jfa_embedding(shifted(table), ids, scale=1.5), out)
    check(table, ids, dout, 1.5, out, binding.jfa_embedding_backward(shifted(dout), ids, 30, scale=1.5))


@pytest.mark.parametrize("dtype", TYPES)
def test_through_autograd(dtype):
    from paper_2409_15373_amd.autograd import jagged_embedding
    rng = np.random.default_rng(5)
    table, ids, dout = make(rng.integers(-1, 100, size=700), 100, 64, dtype)
    leaf = table.clone().requires_grad_()
    off = torch.tensor([0, 600, 700], device="cuda")
    out = jagged_embedding(leaf, ids, off, 1.5)
    grad, = torch.autograd.grad(out, leaf, dout.t().contiguous().t())
    ref = both(table, ids, dout, 1.5)
    assert torch.equal(out, ref[0]) and torch.equal(grad, ref[1])
    step = torch.randn_like(table)   # the loss is linear in the table
    if dtype == torch.float32:
        loss = lambda t: (jagged_embedding(t, ids, off, 1.5).double() * dout.double()).sum()
        assert abs((loss(table + step) - loss(table) - (grad.double() * step.double()).sum()).item()) <= 1e-2   # 45000 terms off by 2^-23 of about 5 each


def test_a_captured_step_replays_to_the_eager_results():
    from paper_2409_15373_amd import binding
    rng = np.random.default_rng(6)
    tables = [make(rng.integers(0, V, size=9000), V, 64, torch.bfloat16) for V in (1200, 50000)]
    eager = [[t.clone() for t in both(*x)] for x in tables]
    graphs = []
    for table, ids, dout in tables:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results = binding.jfa_embedding(table, ids, None, 1.5), binding.jfa_embedding_backward(dout, ids, table.shape[0], None, 1.5)
        graphs.append((g, results))
    for _ in range(3):
        for _, results in graphs:
            for t in results:
                t.fill_(float("nan"))
        for g, _ in graphs:
            g.replay()
        both(*tables[0])
        assert all(torch.equal(a, b) for (_, results), want in zip(graphs, eager) for a, b in zip(results, want))


def test_what_is_refused():
    from paper_2409_15373_amd import binding
    from paper_2409_15373_amd.autograd import jagged_embedding
    table, ids, dout = make([1, 2, 3], 8, 16, torch.float32)
    for bad in ((table, ids.float()), (table, ids.view(3, 1)), (table.t(), ids), (table, ids.cpu()), (table.cpu(), ids), (table, ids, torch.tensor([0, 3]))):
        with pytest.raises(AssertionError):
            jagged_embedding(*bad)
    with pytest.raises(TypeError):
        jagged_embedding(table.half(), ids)
    with pytest.raises(AssertionError):
        binding.jfa_embedding_backward(dout[:2], ids, 8)
    with pytest.raises(binding.JfaError):
        binding.jfa_embedding(table[:0], ids)
