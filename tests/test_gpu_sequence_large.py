"""Linear attention, layer norm and embedding lookup where offsets pass 32 bits (tensors of more than 2^31 elements) and where the sort has many tiles: the rows at
the far end against the same rows in tensors of their own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_linear_attention_at_the_end_of_a_large_tensor():
    from paper_2409_15373_amd import binding
    H, D, n, tail = 64, 128, 262400, 133
    assert (n - tail) * H * D > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(0)
    q, k, v, dout = (torch.randn(n, H, D, device="cuda", dtype=torch.bfloat16, generator=gen) for _ in range(4))
    decay = torch.full((H,), -0.05, device="cuda")
    cut = list(range(0, n - tail, 4000)) + [n - tail, n]
    off, own = torch.tensor(cut, device="cuda"), torch.tensor([0, tail], device="cuda")
    ends = [x[n - tail:].clone() for x in (q, k, v, dout)]
    out = binding.jfa_linear_attention(q, k, v, decay, off, 4000)[0][n - tail:]
    assert torch.equal(out, binding.jfa_linear_attention(*ends[:3], decay, own, 4000)[0])
    grads = binding.jfa_linear_attention_backward(q, k, v, dout, decay, off, 4000)[:3]
    want = binding.jfa_linear_attention_backward(*ends, decay, own, 4000)[:3]
    assert all(torch.equal(a[n - tail:], b) for a, b in zip(grads, want))


def test_layer_norm_at_the_end_of_a_large_tensor():
    from paper_2409_15373_amd import binding
    rows, N = 2200000, 1000
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, N, device="cuda", dtype=torch.bfloat16, generator=gen)
    w, b = (torch.randn(N, device="cuda", generator=gen).bfloat16() for _ in range(2))
    y, mean, rstd = binding.jfa_layer_norm(x, w, b)
    end = binding.jfa_layer_norm(x[-50:].clone(), w, b)
    assert torch.equal(y[-50:], end[0]) and torch.equal(mean[-50:], end[1]) and torch.equal(rstd[-50:], end[2])
    dy = y
    dx, _, db = binding.jfa_layer_norm_backward(x, w, dy, mean, rstd)
    assert torch.equal(dx[-50:], binding.jfa_layer_norm_backward(x[-50:].clone(), w, dy[-50:].clone(), mean[-50:].clone(), rstd[-50:].clone())[0])
    want = sum(part.double().sum(0) for part in dy.split(200000))
    # 2200000 terms in at most 2200000 / 64 + 64 additions of 2^-24 of the absolute sum (3 times the rows), and the result's rounding
    assert ((db.double() - want).abs() <= 2.0 ** -8 * want.abs() + (rows / 64 + 64) * 2.0 ** -24 * 3 * rows).all()


def test_embedding_at_the_end_of_a_large_table():
    from paper_2409_15373_amd import binding
    V, N, rows = 17000000, 128, 17000001
    assert (V - 10) * N > 2 ** 31 and (rows - 10) * N > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(2)
    table = torch.randn(V, N, device="cuda", dtype=torch.bfloat16, generator=gen)
    ids = torch.randperm(V, device="cuda", generator=gen)
    ids = torch.cat([ids, ids[:1]])
    ids[-10:-1] = torch.arange(V - 9, V, device="cuda")
    out = binding.jfa_embedding(table, ids, scale=2.0)
    assert torch.equal(out[-10:], 2.0 * table[ids[-10:]]) and torch.equal(out[:10], 2.0 * table[ids[:10]])
    del table
    dtable = binding.jfa_embedding_backward(out, ids, V, scale=0.5)
    for v in (V - 1, V - 9, 12345, int(ids[0])):
        want = out[(ids == v).nonzero().flatten()].double().sum(0) * 0.5
        assert ((dtable[v].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20).all(), v
    some = torch.randint(0, rows, (100000,), device="cuda", generator=gen)
    counts = torch.bincount(ids, minlength=V)[ids[some]]
    alone = some[counts == 1]
    assert torch.equal(dtable[ids[alone]], (out[alone].float() * 0.5).bfloat16())


@pytest.mark.parametrize("V", [900, 70001])
def test_many_tiles_of_the_sort(V):
    from paper_2409_15373_amd import binding
    rows, N = 700001, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(0, V, (rows,), device="cuda", generator=gen)
    ids[::5] = V // 2
    dout = torch.randint(-8, 9, (rows, N), device="cuda", generator=gen).float()   # whole numbers: sums are exact
    want = torch.zeros(V, N, device="cuda", dtype=torch.float64).index_add_(0, ids, dout.double())
    assert torch.equal(binding.jfa_embedding_backward(dout, ids, V).double(), want)
