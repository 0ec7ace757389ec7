"""Linear attention, layer norm and embedding lookup through the C++ functions against the same through the Python functions, bit for bit; what hooks on saved
tensors give back; and that what is not an ordinary call reaches the Python function."""
import pytest
import torch

pytestmark = pytest.mark.gpu
OPS = ["linear", "linear_state", "norm", "norm_plain", "embedding"]


def setup(op, dtype, seed=0):
    """(call of the public function, call of the Python function, leaves, gradients of the results)"""
    from paper_2409_15373_amd import autograd as a
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, kind=dtype: torch.randn(*s, device="cuda", generator=g).to(kind)
    off = torch.tensor([0, 70, 70, 103], device="cuda")
    if op.startswith("linear"):
        q, k, v = (r(103, 2, 64).requires_grad_() for _ in range(3))
        S0, decay = r(3, 2, 64, 64, kind=torch.float32).requires_grad_(), torch.tensor([-0.1, -0.01], device="cuda")
        state = op == "linear_state"
        args = (q, k, v, decay, off, 70, 0.25, S0, state)
        douts = (r(103, 2, 64),) + ((r(3, 2, 64, 64, kind=torch.float32),) if state else ())
        return (lambda: a.jagged_linear_attention(*args[:6], scale=0.25, initial_state=S0, return_state=state)), (lambda: a._LinearAttention.apply(*args)), (q, k, v, S0), douts
    if op.startswith("norm"):
        x = r(103, 3, 40).requires_grad_()
        w, b = (None, None) if op == "norm_plain" else (torch.nn.Parameter(r(3, 40)), torch.nn.Parameter(r(3, 40)))
        return (lambda: a.jagged_layer_norm(x, w, b, off, 1e-3)), (lambda: a._LayerNorm.apply(x, w, b, off, 1e-3)), tuple(t for t in (x, w, b) if t is not None), (r(103, 3, 40),)
    table, ids = torch.nn.Parameter(r(50, 40)), torch.randint(-1, 50, (103,), device="cuda", generator=g)
    return (lambda: a.jagged_embedding(table, ids, off, 0.5)), (lambda: a._Embedding.apply(table, ids, off, 0.5)), (table,), (r(103, 40),)


def results(call, leaves, douts):
    out = call()
    outs = out if isinstance(out, tuple) else (out,)
    return tuple(o.detach() for o in outs) + torch.autograd.grad(outs, leaves, douts)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("op", OPS)
def test_nodes_equal_the_python_functions(op, dtype):
    from paper_2409_15373_amd import autograd
    public, python, leaves, douts = setup(op, dtype)
    out = public()
    name = type((out[0] if isinstance(out, tuple) else out).grad_fn).__name__
    assert autograd._native and "Backward" not in name, name   # the Python functions' are named after them
    for a, b in zip(results(public, leaves, douts), results(python, leaves, douts)):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)
    with torch.no_grad():
        a, b = public(), python()
        for x, y in zip(a if isinstance(a, tuple) else (a,), b if isinstance(b, tuple) else (b,)):
            assert torch.equal(x, y) and not x.requires_grad and not y.requires_grad


@pytest.mark.parametrize("op", OPS)
def test_hooks_on_saved_tensors(op):
    public, _, leaves, douts = setup(op, torch.float32)
    want = results(public, leaves, douts)

    def step(unpack, pack=lambda t: t):
        with torch.autograd.graph.saved_tensors_hooks(pack, unpack):
            out = public()
        return torch.autograd.grad(out, leaves, douts)
    assert all(torch.equal(a, b) for a, b in zip(step(lambda t: t.cuda(), lambda t: t.cpu()), want[-len(leaves):]))
    with pytest.raises(AssertionError):
        step(lambda t: t.cpu())
    for unpack in (lambda t: t[1:].contiguous(), lambda t: t.half() if t.is_floating_point() else t.short()):
        with pytest.raises(RuntimeError, match="was saved"):
            step(unpack)


@pytest.mark.parametrize("op", OPS)
def test_calls_that_others_listen_to(op):
    """Under a function mode, a tracer or a function transform the Python function has the call."""
    from torch.overrides import TorchFunctionMode
    public, _, leaves, _ = setup(op, torch.float32)

    class Mode(TorchFunctionMode):
        seen = 0

        def __torch_function__(self, func, types, args=(), kwargs=None):
            Mode.seen += 1
            return func(*args, **(kwargs or {}))
    with Mode():
        public()
    assert Mode.seen > 0
    with pytest.raises((RuntimeError, NotImplementedError)):   # the Python functions have no rule for it, and say so
        torch.func.vmap(lambda t: _with(op, t))(leaves[0].detach().expand(2, *leaves[0].shape).contiguous())


def _with(op, t):
    from paper_2409_15373_amd import autograd as a
    off = torch.tensor([0, 70, 70, 103], device="cuda")
    if op.startswith("linear"):
        return a.jagged_linear_attention(t, t, t, torch.zeros(2, device="cuda"), off, 70)
    if op.startswith("norm"):
        return a.jagged_layer_norm(t)
    return a.jagged_embedding(t, torch.zeros(103, dtype=torch.int64, device="cuda"))


def test_a_single_token_through_cpp_and_ctypes(monkeypatch):
    from paper_2409_15373_amd import binding
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k, v = (torch.randn(7, 2, 64, device="cuda", generator=g).bfloat16() for _ in range(3))
    S, decay = torch.randn(7, 2, 64, 64, device="cuda", generator=g), torch.tensor([-0.1, -0.5], device="cuda")
    answers, ask = [], binding._native
    with monkeypatch.context() as m:
        m.setattr(binding, "_native", lambda *args: answers.append(ask(*args)) or answers[-1])
        a = binding.jfa_linear_attention_step(q, k, v, decay, S, new_state=torch.empty_like(S))
    assert len(answers) == 1 and answers[0] is not None
    with monkeypatch.context() as m:
        m.setattr(binding, "_calls", False)
        b = binding.jfa_linear_attention_step(q, k, v, decay, S, new_state=torch.empty_like(S))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tensors_without_rows(dtype):
    """No rows in any sample: results without rows, states handed through, gradients of nothing."""
    from paper_2409_15373_amd import autograd as a
    off, decay = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.tensor([-0.1, -0.5], device="cuda")
    q = torch.empty(0, 2, 32, device="cuda", dtype=dtype, requires_grad=True)
    S0 = torch.randn(3, 2, 32, 32, device="cuda", requires_grad=True)
    out, final = a.jagged_linear_attention(q, q, q, decay, off, 0, initial_state=S0, return_state=True)
    assert out.shape == (0, 2, 32) and torch.equal(final, S0)
    dq, dS0 = torch.autograd.grad(final, (q, S0), torch.ones_like(final))
    assert dq.shape == (0, 2, 32) and torch.equal(dS0, torch.ones_like(S0))
    x, w = torch.empty(0, 32, device="cuda", dtype=dtype, requires_grad=True), torch.ones(32, device="cuda", dtype=dtype, requires_grad=True)
    y = a.jagged_layer_norm(x, w, None, off)
    dx, dw = torch.autograd.grad(y, (x, w), torch.empty_like(y))
    assert y.shape == dx.shape == (0, 32) and not dw.any()
    table = torch.randn(9, 32, device="cuda", dtype=dtype).requires_grad_()
    out = a.jagged_embedding(table, torch.empty(0, dtype=torch.int64, device="cuda"), off)
    dtable, = torch.autograd.grad(out, table, torch.empty_like(out))
    assert out.shape == (0, 32) and not dtable.any()


@pytest.mark.parametrize("which", ["public", "python"])
@pytest.mark.parametrize("op", OPS)
def test_gradients_are_not_differentiated(op, which):
    """A graph of a backward may be made (and equals the gradients without one); what goes through it raises instead of leaving these terms out."""
    public, python, leaves, douts = setup(op, torch.float32)
    call = public if which == "public" else python
    want = results(call, leaves, douts)
    out = call()
    outs = out if isinstance(out, tuple) else (out,)
    douts = tuple(d.clone().requires_grad_() for d in douts)
    grads = torch.autograd.grad(outs, leaves, douts, create_graph=True)
    for a, b in zip(grads, want[len(outs):]):
        assert torch.equal(a, b)
    loss = sum((g * g).sum() for g in grads) + sum((t * t).sum() for t in leaves)
    for inputs in (douts,) if op == "embedding" else (leaves, douts):   # (the table's gradient does not depend on the table)
        with pytest.raises(RuntimeError, match="differentia"):
            torch.autograd.grad(loss, inputs, retain_graph=True)
    with pytest.raises(RuntimeError, match="differentia"):
        loss.backward()


def test_decays_that_want_gradients():
    from paper_2409_15373_amd.autograd import jagged_linear_attention
    q, k, v = (torch.randn(10, 2, 32, device="cuda") for _ in range(3))
    decay, off = torch.nn.Parameter(torch.tensor([-0.1, -0.01], device="cuda")), torch.tensor([0, 10], device="cuda")
    with pytest.raises(ValueError, match="log_decay"):
        jagged_linear_attention(q, k, v, decay, off, 10)
    with torch.no_grad():
        assert torch.equal(jagged_linear_attention(q, k, v, decay, off, 10), jagged_linear_attention(q, k, v, decay.detach(), off, 10))
