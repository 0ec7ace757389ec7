"""The sequence operators as a model has them: ids to rows, layer norm, attention over each history (linear or causal softmax), layer norm, and the gradients
back to the table; against the same model in fp64 with torch's own operators.
"""
import gc

import numpy as np
import pytest
import torch

from paper_2409_15373_amd.synthetic import offsets_from_lengths

pytestmark = pytest.mark.gpu


class Block:
    def __init__(self, lengths, V, H, D, dtype, seed=0):
        gen = torch.Generator().manual_seed(seed)
        N = H * D
        self.H, self.D, self.max_len = H, D, max(lengths)
        self.offsets = torch.from_numpy(offsets_from_lengths(np.array(lengths)))
        n = int(self.offsets[-1])
        self.ids = torch.randint(-1, V, (n,), generator=gen)
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(3.0, 7.0, H)))
        normal = lambda *s, scale=1.0: (torch.randn(*s, generator=gen) * scale).to(dtype)
        self.leaves = [normal(V, N), 1 + normal(N, scale=0.1), normal(N, scale=0.1), normal(N, N, scale=N ** -0.5), normal(N, N, scale=N ** -0.5), normal(N, N, scale=N ** -0.5),
                       1 + normal(N, scale=0.1), normal(N, scale=0.1)]
        self.dout = normal(n, N, scale=0.1)

    def ours(self, softmax):
        from paper_2409_15373_amd.autograd import jagged_embedding, jagged_flash_attention, jagged_layer_norm, jagged_linear_attention
        leaves = [t.cuda().requires_grad_() for t in self.leaves]
        table, w1, b1, wq, wk, wv, w2, b2 = leaves
        offsets, log_decay = self.offsets.cuda(), self.log_decay.cuda()
        x = jagged_embedding(table, self.ids.cuda(), offsets, scale=0.5)
        h = jagged_layer_norm(x, w1, b1, offsets)
        q, k, v = ((h @ w).view(-1, self.H, self.D) for w in (wq, wk, wv))
        mixed = jagged_flash_attention(q, k, v, offsets, self.max_len, causal=True) if softmax else jagged_linear_attention(q, k, v, log_decay, offsets, self.max_len)
        y = jagged_layer_norm(x + mixed.reshape(x.shape), w2, b2, offsets)
        return [y.detach()] + list(torch.autograd.grad(y, leaves, self.dout.cuda()))

    def plain(self, softmax):
        leaves = [t.double().requires_grad_() for t in self.leaves]
        table, w1, b1, wq, wk, wv, w2, b2 = leaves
        x = torch.cat([table, torch.zeros_like(table[:1])])[self.ids] * 0.5   # id -1: the row of zeros
        h = torch.nn.functional.layer_norm(x, w1.shape, w1, b1)
        mixed = []
        for lo, hi in zip(self.offsets[:-1].tolist(), self.offsets[1:].tolist()):
            q, k, v = ((h[lo:hi] @ w).view(-1, self.H, self.D).transpose(0, 1) for w in (wq, wk, wv))
            i = torch.arange(hi - lo)
            apart = i[:, None] - i[None, :]
            scores = q @ k.transpose(1, 2) * self.D ** -0.5
            if softmax:
                weights = torch.softmax(scores.masked_fill(apart < 0, float("-inf")), -1)
            else:
                weights = scores * torch.exp(self.log_decay.double()[:, None, None] * apart.clamp(min=0)) * (apart >= 0)
            mixed.append((weights @ v).transpose(0, 1).reshape(hi - lo, self.H * self.D))
        y = torch.nn.functional.layer_norm(x + torch.cat(mixed), w2.shape, w2, b2)
        return [y.detach()] + list(torch.autograd.grad(y, leaves, self.dout.double()))


@pytest.mark.parametrize("softmax", [False, True])
@pytest.mark.parametrize("dtype,tolerance", [(torch.float32, 2e-4), (torch.bfloat16, 6e-2)])
def test_a_model_and_its_gradients(dtype, tolerance, softmax):
    """Root mean square errors against each result's own.  A bf16 number is off by up to 2^-8; every result has passed through about twelve
    roundings of intermediate tensors (x, h, q, k, v, the attention's two, the sum, and the same on the way back), which add up to at most
    12 * 2^-8 = 4.7e-2 where all have the same sign and size.  fp32: products of 128 terms, a few dozen of them in a row, 2^-24 each."""
    block = Block([70, 1, 0, 133, 20], 50, 2, 64, dtype)
    for name, a, b in zip(("y", "table", "w1", "b1", "wq", "wk", "wv", "w2", "b2"), block.ours(softmax), block.plain(softmax)):
        err = (a.double().cpu() - b).square().mean().sqrt() / b.square().mean().sqrt()
        assert torch.isfinite(a).all() and err <= tolerance, (name, float(err))


def test_on_a_stream_of_its_own():
    """All on a stream that is not the default one, behind a long wait, with inputs that are only written after it."""
    block = Block([300, 40], 50, 2, 64, torch.float32)
    want = block.ours(False)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        got = block.ours(False)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_captured_training_step():
    """A step captured, with gradients, and replayed with eager work in between.  While an eager graph of the same leaves is alive the captured backward is
    refused: the leaves' gradients belong to the eager graph's stream, and drawing that into the capture ends the process."""
    from paper_2409_15373_amd.autograd import jagged_embedding, jagged_layer_norm, jagged_linear_attention
    block = Block([300, 0, 41], 50, 2, 64, torch.bfloat16)
    leaves = [block.leaves[i].cuda().requires_grad_() for i in (0, 1, 2)]
    offsets, log_decay, ids, dout = block.offsets.cuda(), block.log_decay.cuda(), block.ids.cuda(), block.dout.cuda()

    def step():
        x = jagged_layer_norm(jagged_embedding(leaves[0], ids, offsets, 0.5), leaves[1], leaves[2], offsets).view(-1, 2, 64)
        out = jagged_linear_attention(x, x, x, log_decay, offsets, block.max_len).view(-1, 128)
        return out, torch.autograd.grad(out, leaves, dout, retain_graph=True)
    alive, eager = step()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            step()
    torch.cuda.synchronize()
    alive = alive.detach()
    gc.collect()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, grads = step()
    for _ in range(3):
        for t in grads:
            t.fill_(float("nan"))
        g.replay()
        again = step()
        torch.cuda.synchronize()
        assert torch.equal(again[0], alive) and all(torch.equal(a, b) for a, b in zip(again[1], eager))
        assert torch.equal(out, alive) and all(torch.equal(a, b) for a, b in zip(grads, eager))


def test_two_streams_at_once():
    """Two batches' steps on a stream each, with no wait between them; the first call waits so that the others overlap."""
    blocks = [Block([300, 40, 0, 200], 50, 2, 64, torch.float32, seed) for seed in (1, 2)]
    want = [block.ours(False) for block in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for stream in streams:
        with torch.cuda.stream(stream):
            torch.cuda._sleep(20_000_000)
    got = [[], []]
    for _ in range(3):
        for i, (block, stream) in enumerate(zip(blocks, streams)):
            with torch.cuda.stream(stream):
                got[i].append(block.ours(False))
    torch.cuda.synchronize()
    for results, expected in zip(got, want):
        for result in results:
            assert all(torch.equal(a, b) for a, b in zip(result, expected))


def test_two_graphs_replayed_at_once():
    """The gradients' calls, captured into two graphs with workspaces of their own, replayed on two streams at a time."""
    from paper_2409_15373_amd import binding
    gen = torch.Generator(device="cuda").manual_seed(4)
    offsets = torch.tensor([0, 1500, 1500, 1503], device="cuda")
    decay, ids = torch.tensor([-0.01], device="cuda"), torch.randint(0, 5000, (1503,), device="cuda", generator=gen)
    w = torch.ones(64, device="cuda")

    def calls(t):
        norm = binding.jfa_layer_norm(t[0].view(-1, 64), w, w, offsets)
        return (*binding.jfa_linear_attention_backward(*t, decay, offsets, 1500)[:3], *binding.jfa_layer_norm_backward(t[0].view(-1, 64), w, t[1].view(-1, 64), norm[1], norm[2], offsets),
                binding.jfa_embedding_backward(t[0].view(-1, 64), ids, 5000, offsets))
    tensors = [[torch.randn(1503, 1, 64, device="cuda", generator=gen) for _ in range(4)] for _ in range(2)]
    want = [calls(t) for t in tensors]
    graphs, results = [], []
    for t in tensors:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(calls(t))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        for result in results:
            for x in result:
                x.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for result, expected in zip(results, want):
            assert all(torch.equal(a, b) for a, b in zip(result, expected))
