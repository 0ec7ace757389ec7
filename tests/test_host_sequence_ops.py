"""CPU-only: what the entry points of linear attention, layer norm and embedding lookup refuse before anything reaches the GPU."""
import pytest
import torch

from paper_2409_15373_amd import binding


@pytest.fixture(scope="module")
def lib():
    return binding.load()


OK, BAD, UNSUPPORTED = binding.JFA_OK, binding.JFA_ERR_INVALID_ARG, binding.JFA_ERR_UNSUPPORTED


def refused(status, expected, word):
    assert status == expected
    assert word in binding.jfa_last_error()


@pytest.mark.parametrize("suffix", ["", "_f32"])
def test_linear_attention(lib, suffix):
    forward, backward, step = (getattr(lib, f"jfa_linear_attention{x}{suffix}") for x in ("", "_backward", "_step"))

    def call(B=2, rows=16, max_len=8, H=2, D=64, q=16, state=None, offsets=16, workspace=None, n=0):
        return forward(q, 16, 16, 16, offsets, B, rows, max_len, H, D, 1.0, state, 16, None, workspace, n, None)

    refused(call(B=-1), BAD, "negative")
    refused(call(max_len=-1), BAD, "max_len")
    refused(call(max_len=1 << 31), BAD, "max_len")
    refused(call(rows=-1), BAD, "rows")
    refused(call(H=0), BAD, "H = 0")
    refused(call(H=1 << 15), UNSUPPORTED, "H * D")
    refused(call(D=48), UNSUPPORTED, "D = 48")
    refused(call(B=(1 << 22) + 1, H=1), UNSUPPORTED, "exceeds")
    refused(call(B=1 << 62, H=8), UNSUPPORTED, "exceeds")
    refused(call(q=None), BAD, "null")
    refused(call(q=8), BAD, "aligned")
    refused(call(state=8), BAD, "state")
    refused(call(offsets=None), BAD, "null")
    assert call(B=0, q=None, offsets=None) == OK
    # a long sample needs a workspace
    need = binding.load().jfa_linear_attention_workspace_bytes(1, 100000, 100000, 1, 64, 0)
    assert need > 0
    refused(call(B=1, rows=100000, max_len=100000, H=1), BAD, "workspace")
    refused(call(B=1, rows=100000, max_len=100000, H=1, workspace=16, n=need - 1), BAD, "workspace")
    refused(call(B=1, rows=100000, max_len=100000, H=1, workspace=8, n=need), BAD, "aligned")
    refused(backward(16, 16, 16, 16, 16, 16, 2, 16, 8, 2, 64, 1.0, None, None, 16, None, 16, None, None, 0, None), BAD, "null")
    refused(backward(16, 16, 16, 16, 16, 16, 2, 16, 8, 2, 96, 1.0, None, None, 16, 16, 16, None, None, 0, None), UNSUPPORTED, "D = 96")
    refused(backward(16, 16, 16, 16, 16, 16, 2, 16, 8, 2, 64, 1.0, None, None, 16, 16, 16, 24, None, 0, None), BAD, "state")
    refused(backward(16, 16, 16, 16, 16, 16, 1, 100000, 100000, 1, 64, 1.0, None, None, 16, 16, 16, None, 16, 16, None), BAD, "workspace")
    refused(step(16, 16, 16, 16, 2, 2, 64, 1.0, None, 16, 16, None), BAD, "null")
    refused(step(16, 16, 16, 16, 2, 2, 64, 1.0, 16, 16, 24, None), BAD, "aligned")
    refused(step(16, 16, 16, 16, 2, 2, 65, 1.0, 16, 16, 16, None), UNSUPPORTED, "D = 65")
    assert step(None, None, None, None, 0, 2, 64, 1.0, None, None, None, None) == OK


def test_the_workspace_of_linear_attention_is_bounded():
    """Samples of like lengths need none; of others, an order of them, or states between segments: as many bytes as a bf16 tensor of that many rows at
    most, whatever bound on the lengths is given."""
    size = binding.load().jfa_linear_attention_workspace_bytes
    assert size(4096, 4096 << 10, 1 << 10, 8, 128, 1) == 0
    assert 0 < size(512, 200000, 1024, 4, 128, 0) == size(512, 200000, 1024, 4, 128, 1) < 10000   # an order
    for B, H in [(1, 1), (3, 7), (64, 8)]:
        for D in (32, 64, 128):
            for rows in (2000, 1 << 20):
                assert size(B, rows, 1 << 30, H, D, 0) <= rows * H * D * 2 * D // 128
                assert size(B, rows, 1 << 30, H, D, 1) <= rows * H * D * 4 * D // 128
            assert size(1, 1, 1 << 30, H, D, 0) == 0 < size(1, 1 << 20, 1 << 30, 1, D, 0)
    assert size(4, 256, 64, 2, 64, 0) == 0 and size(0, 0, 64, 2, 64, 0) == 0 and size(4, 256, 64, 2, 63, 0) == 0


@pytest.mark.parametrize("suffix", ["", "_f32"])
def test_layer_norm(lib, suffix):
    forward, backward = getattr(lib, "jfa_layer_norm" + suffix), getattr(lib, "jfa_layer_norm_backward" + suffix)

    def call(x=16, weight=16, offsets=None, B=0, rows=4, reps=1, N=8, y=16, mean=None):
        return forward(x, weight, 16, offsets, B, rows, reps, N, 1e-5, y, mean, None, None)

    refused(call(rows=-1), BAD, "rows")
    refused(call(rows=(1 << 30) + 1), UNSUPPORTED, "rows")
    refused(call(N=0), BAD, "N = 0")
    refused(call(N=(1 << 20) + 1), UNSUPPORTED, "N = ")
    refused(call(reps=0), BAD, "reps")
    refused(call(reps=1 << 29), BAD, "reps")
    refused(call(offsets=16, B=-1), BAD, "B = -1")
    refused(call(offsets=12, B=1), BAD, "offsets")
    refused(call(x=None), BAD, "x is null")
    refused(call(y=None), BAD, "y is null")
    refused(call(weight=17), BAD, "weight")
    refused(call(mean=18), BAD, "mean")
    assert call(rows=0, x=None, y=None) == OK
    refused(backward(16, 16, 16, 16, 16, None, 0, 4, 1, 8, 16, 16, 16, None, 0, None), BAD, "workspace")
    refused(backward(16, 16, 16, 16, 16, None, 0, 4, 1, 8, 16, 16, 16, 16, 4 * 2 * 8 * 4 - 1, None), BAD, "workspace")
    refused(backward(16, 16, 16, 16, 16, None, 0, 4, 1, 8, 16, 16, 16, 8, 1 << 20, None), BAD, "aligned")
    refused(backward(16, 16, 16, None, 16, None, 0, 4, 1, 8, 16, None, None, None, 0, None), BAD, "mean")
    refused(backward(16, 16, 16, 16, 16, None, 0, 4, 1, 8, None, None, None, None, 0, None), BAD, "dx")
    assert backward(None, None, None, None, None, None, 0, 0, 1, 8, None, None, None, None, 0, None) == OK
    assert lib.jfa_layer_norm_workspace_bytes(1 << 20, 1, 100) == 1024 * 2 * 100 * 4
    assert lib.jfa_layer_norm_workspace_bytes(-1, 1, 100) == 0


@pytest.mark.parametrize("suffix", ["", "_f32"])
def test_embedding(lib, suffix):
    forward, backward = getattr(lib, "jfa_embedding" + suffix), getattr(lib, "jfa_embedding_backward" + suffix)

    def call(table=16, ids=16, id_bytes=8, offsets=None, B=0, rows=4, V=10, N=8, out=16):
        return forward(table, ids, id_bytes, offsets, B, rows, V, N, 1.0, out, None)

    refused(call(rows=-1), BAD, "rows")
    refused(call(V=0), BAD, "V = 0")
    refused(call(V=(1 << 30) + 1), UNSUPPORTED, "V = ")
    refused(call(N=-3), BAD, "N = -3")
    refused(call(id_bytes=2), BAD, "id_bytes")
    refused(call(ids=12), BAD, "ids")
    refused(call(table=17), BAD, "table")
    refused(call(out=None), BAD, "out is null")
    assert call(rows=0, table=None, ids=None, out=None) == OK
    need = lib.jfa_embedding_workspace_bytes(4, 10, 8)
    assert need > 0 and lib.jfa_embedding_workspace_bytes(4, 0, 8) == 0
    refused(backward(16, 16, 8, None, 0, 4, 10, 8, 1.0, 16, None, 0, None), BAD, "workspace")
    refused(backward(16, 16, 8, None, 0, 4, 10, 8, 1.0, 16, 16, need - 1, None), BAD, "workspace")
    refused(backward(16, 16, 8, None, 0, 4, 10, 8, 1.0, 16, 24, need, None), BAD, "aligned")
    refused(backward(16, 16, 8, None, 0, 4, 10, 8, 1.0, None, 16, need, None), BAD, "dtable")


def test_tensors_that_are_not_on_a_gpu_are_refused():
    from paper_2409_15373_amd import autograd
    x = torch.randn(8, 2, 32)
    offsets, decay = torch.tensor([0, 8]), torch.zeros(2)
    with pytest.raises(AssertionError):
        autograd.jagged_linear_attention(x, x, x, decay, offsets, 8)
    with pytest.raises(AssertionError):
        binding.jfa_linear_attention_step(x, x, x, decay, torch.zeros(8, 2, 32, 32))
    with pytest.raises(AssertionError):
        autograd.jagged_layer_norm(x, torch.ones(32), torch.zeros(32))
    with pytest.raises(AssertionError):
        autograd.jagged_embedding(x, torch.arange(8))
    with pytest.raises(ValueError):
        autograd.jagged_linear_attention(x, x, x, decay.requires_grad_(), offsets, 8)


def test_linear_attention_of_more_rows_than_there_can_be(lib):
    assert lib.jfa_linear_attention_workspace_bytes(1, 1 << 38, 5, 1, 32, 0) == 0   # none needed
    refused(lib.jfa_linear_attention(16, 16, 16, 16, 16, 1, (1 << 38) + 1, 5, 1, 32, 1.0, None, 16, None, None, 0, None), BAD, "rows")
    assert lib.jfa_linear_attention_workspace_bytes(1, (1 << 38) + 1, 5, 1, 32, 0) == 0
    assert "rows" in binding.jfa_last_error()
