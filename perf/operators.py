"""Sizes, inputs and plain forms of the sequence operators around jagged attention: linear attention with a decay for each head
(whole samples, their gradient, single tokens), layer norm of jagged rows, embedding lookup into jagged rows.

``own`` chooses what ``run`` computes: the plain form out of elementary torch operations, or the framework's operators.
"""
import functools
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- cases -----------------------------------------------------------------------------------------------------------

def _linear(mode, B, max_len, H, D, dtype, lengths, lengths_seed, states=False):
    return {"op": "linear", "mode": mode, "B": B, "max_len": max_len, "H": H, "D": D, "dtype": dtype, "lengths": lengths,
            "lengths_seed": lengths_seed, "states": states}


def _step(B, H, D, dtype):
    return {"op": "step", "B": B, "H": H, "D": D, "dtype": dtype}


def _norm(mode, rows, N, dtype):
    return {"op": "norm", "mode": mode, "rows": rows, "N": N, "dtype": dtype}


def _embedding(mode, rows, V, N, dtype, ids):
    return {"op": "embedding", "mode": mode, "rows": rows, "V": V, "N": N, "dtype": dtype, "ids": ids}


def listed():
    cases = [
        # four short histories answered one batch at a time: the smallest call, all latency
        ("linear_short_prompts", _linear("prompt", 4, 64, 1, 32, "fp32", "uniform", 0, states=True)),
        # a training step's attention over histories of every length up to 1024
        ("linear_train", _linear("train", 512, 1024, 4, 128, "bf16", "uniform", 4)),
        # two long histories taken in at once, continued from and into a state
        ("linear_long_prompts", _linear("prompt", 2, 16000, 8, 128, "bf16", "uniform", 11, states=True)),
        # a training step of a small model in full precision, most histories short
        ("linear_train_fp32", _linear("train", 200, 300, 2, 64, "fp32", "geometric", 1)),
        # one event for each of 1024 users being served
        ("linear_step", _step(1024, 8, 128, "bf16")),
        # one event for five users
        ("linear_step_few", _step(5, 2, 64, "fp32")),
        # the rows of a training batch with 51 samples in 512 long, all heads of a row at once
        ("norm_train", _norm("train", 213593, 1024, "bf16")),
        # a small batch with a row length that no vector divides
        ("norm_train_odd", _norm("train", 1501, 257, "fp32")),
        # a served batch of histories
        ("norm_forward", _norm("forward", 14848, 512, "bf16")),
        # a training batch's items out of a catalogue of a million
        ("embedding_train", _embedding("train", 322248, 1000003, 128, "bf16", "zipf")),
        # the items of four short histories
        ("embedding_forward_short", _embedding("forward", 147, 5000, 32, "fp32", "zipf")),
        # ids of a small catalogue, one in three the id that stands for anything unknown
        ("embedding_train_hot", _embedding("train", 131072, 30011, 512, "bf16", "hot")),
    ]
    return [dict(case, name=name) for name, case in cases]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "step", "norm", "embedding"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "linear":
        mode = rng.choice(["prompt", "train"])
        H, D = rng.randint(1, 8), rng.choice([32, 64, 128])
        max_len = _log_uniform(rng, 1, 16000 if mode == "prompt" else 4096)
        most = max(1, min(1024, 512 * 1024 * 4 * 128 // (2 * max_len * H * D)))
        return _linear(mode, _log_uniform(rng, 1, most), max_len, H, D, dtype, rng.choice(["uniform", "geometric", "bimodal"]),
                       rng.randrange(1 << 30), states=mode == "prompt" and rng.random() < 0.7)
    if op == "step":
        H, D = rng.randint(1, 8), rng.choice([32, 64, 128])
        return _step(_log_uniform(rng, 1, 1024), H, D, dtype)
    mode = rng.choice(["forward", "train"])
    if op == "norm":
        N = _log_uniform(rng, 8, 8192)
        return _norm(mode, _log_uniform(rng, 1, max(1, min(262144, 213593 * 512 // N))), N, dtype)
    N = _log_uniform(rng, 8, 1024)
    return _embedding(mode, _log_uniform(rng, 1, max(1, min(322248, 322248 * 64 // N))), _log_uniform(rng, 2, max(2, min(1000003, 1000003 * 64 // N))), N,
                      dtype, rng.choice(["uniform", "zipf", "hot"]))


def _lengths(case):
    """The samples' lengths: part of the case, whatever the inputs' seed."""
    rng = np.random.default_rng(case["lengths_seed"])
    B, most = case["B"], case["max_len"]
    if case["lengths"] == "uniform":
        lengths = rng.integers(1, most + 1, size=B)
    elif case["lengths"] == "geometric":
        lengths = np.minimum(rng.geometric(min(1.0, 4.0 / most), size=B), most)
    else:   # one in ten long
        lengths = np.where(rng.random(B) < 0.1, rng.integers(max(1, most // 2), most + 1, size=B), rng.integers(0, max(1, most // 16) + 1, size=B))
    lengths[rng.integers(0, B)] = most   # max_len is a bound that some sample reaches
    return lengths


@functools.lru_cache(maxsize=4)
def _id_weights(V, ids):
    """How often each id comes up."""
    if ids == "uniform":
        return np.full(V, 1.0 / V)
    weights = 1.0 / np.arange(1, V + 1) ** 1.05
    weights /= weights.sum()
    if ids == "hot":
        weights *= 2.0 / 3.0
        weights[0] += 1.0 / 3.0
    return weights


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "linear":
        H, D, B, n = case["H"], case["D"], case["B"], int(_lengths(case).sum())
        rows = n * H * D
        moved, flops = 4 * rows * size, 4 * rows * D
        if case["mode"] == "train":
            moved, flops = (4 + 5) * rows * size, (4 + 10) * rows * D   # dout is read and three gradients written; q, k and v are there already
        if case["states"]:
            moved += 2 * B * H * D * D * 4
        return {"bytes": moved + 8 * (B + 1) + 4 * H, "flops": flops}
    if case["op"] == "step":
        B, H, D = case["B"], case["H"], case["D"]
        return {"bytes": B * H * (8 * D * D + 4 * D * size) + 4 * H, "flops": 5 * B * H * D * D}
    rows, N = case["rows"], case["N"]
    if case["op"] == "norm":
        if case["mode"] == "train":
            return {"bytes": 4 * rows * N * size + 4 * N * size, "flops": 20 * rows * N}
        return {"bytes": 2 * rows * N * size + 2 * N * size, "flops": 8 * rows * N}
    V = case["V"]
    distinct = float((1.0 - np.exp(rows * np.log1p(-np.minimum(_id_weights(V, case["ids"]), 1.0 - 1e-12)))).sum())
    moved, flops = 8 * rows + (distinct + rows) * N * size, rows * N
    if case["mode"] == "train":
        moved, flops = moved + (rows + V) * N * size, flops + rows * N + V * N
    return {"bytes": int(moved), "flops": int(flops)}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = _TYPES[case["dtype"]]

    def normal(*shape, sigma=1.0, kind=dtype):
        return (torch.randn(*shape, device="cuda", generator=gen) * sigma).to(kind)

    state = {"case": case}
    if case["op"] in ("linear", "step"):
        H, D, B = case["H"], case["D"], case["B"]
        # from a few dozen events' memory to several thousand, head by head, as models with fixed decays have it
        state["log_decay"] = torch.log1p(-torch.exp2(-torch.linspace(4.0, 11.0, H, dtype=torch.float64))).float().cuda()
        state["scale"] = D ** -0.5
    if case["op"] == "linear":
        lengths = _lengths(case)
        n = int(lengths.sum())
        state["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)).cuda()
        for name in ("q", "k", "v"):
            state[name] = normal(n, H, D).requires_grad_(case["mode"] == "train")
        if case["mode"] == "train":
            state["dout"] = normal(n, H, D, sigma=0.1)
        if case["states"]:
            state["initial"] = normal(B, H, D, D, kind=torch.float32)
    elif case["op"] == "step":
        for name in ("q", "k", "v"):
            state[name] = normal(B, H, D)
        state["state"], state["out_state"] = normal(B, H, D, D, sigma=4.0, kind=torch.float32), torch.empty(B, H, D, D, device="cuda")
    elif case["op"] == "norm":
        rows, N = case["rows"], case["N"]
        grad = case["mode"] == "train"
        state["x"] = (normal(rows, N, kind=torch.float32) * 2.0 + normal(rows, 1, kind=torch.float32)).to(dtype).requires_grad_(grad)
        state["weight"] = (1.0 + normal(N, sigma=0.2, kind=torch.float32)).to(dtype).requires_grad_(grad)
        state["bias"] = normal(N, sigma=0.2).requires_grad_(grad)
        if grad:
            state["dout"] = normal(rows, N, sigma=0.1)
    else:
        rows, V, N = case["rows"], case["V"], case["N"]
        grad = case["mode"] == "train"
        cumulated = torch.from_numpy(np.cumsum(_id_weights(V, case["ids"]))).cuda()
        rank = torch.searchsorted(cumulated, torch.rand(rows, device="cuda", generator=gen, dtype=torch.float64)).clamp_(max=V - 1)
        state["ids"] = (rank * 7919 + 17) % V if math.gcd(7919, V) == 1 else rank   # the frequent ids lie all over the table
        state["table"] = normal(V, N).requires_grad_(grad)
        state["scale"] = float(N) ** 0.5
        if grad:
            state["dout"] = normal(rows, N, sigma=0.1)
    return state


# ---- the plain form --------------------------------------------------------------------------------------------------

def _powers(log_decay, exponents):
    """exp(log_decay * exponents) for whole exponents from zero on, [H, ...]."""
    return torch.exp(log_decay.view(-1, *([1] * exponents.dim())) * exponents)


def _plain_linear(q, k, v, log_decay, offsets, max_len, scale, initial):
    """Padded samples, 64 rows at a time: inside a chunk by products of rows, from chunk to chunk through the state."""
    n, H, D = q.shape
    B = offsets.numel() - 1
    C = min(64, max_len)
    chunks = (max_len + C - 1) // C
    lengths = offsets[1:] - offsets[:-1]
    sample = torch.repeat_interleave(torch.arange(B, device=q.device), lengths, output_size=n)
    place = sample * (chunks * C) + torch.arange(n, device=q.device) - offsets[sample]

    def pad(x):   # [chunks, B, H, C, D]
        dense = torch.zeros(B * chunks * C, H, D, device=x.device).index_copy(0, place, x.float())
        return dense.view(B, chunks, C, H, D).permute(1, 0, 3, 2, 4).contiguous()

    qd, kd, vd = pad(q), pad(k), pad(v)
    at = torch.arange(C, device=q.device, dtype=torch.float32)
    apart = at[:, None] - at[None, :]
    inside = torch.where(apart >= 0, _powers(log_decay, apart.clamp(min=0)), 0.0)   # [H, C, C]
    before = _powers(log_decay, at + 1)[..., None]                                     # [H, C, 1]
    after = _powers(log_decay, C - 1 - at)[..., None]
    whole = _powers(log_decay, torch.tensor(float(C), device=q.device))[:, None, None]
    S = torch.zeros(B, H, D, D, device=q.device) if initial is None else initial
    out = []
    for c in range(chunks):
        out.append((qd[c] @ kd[c].transpose(-1, -2) * inside) @ vd[c] + (qd[c] * before) @ S)
        if c + 1 < chunks:
            S = S * whole + (kd[c] * after).transpose(-1, -2) @ vd[c]
    out = torch.stack(out).permute(1, 0, 3, 2, 4).reshape(B * chunks * C, H, D)
    return (out.index_select(0, place) * scale).to(q.dtype)


def _plain_final_state(k, v, log_decay, offsets, max_len, initial):
    n, H, D = k.shape
    B = offsets.numel() - 1
    lengths = offsets[1:] - offsets[:-1]
    sample = torch.repeat_interleave(torch.arange(B, device=k.device), lengths, output_size=n)
    row = torch.arange(n, device=k.device) - offsets[sample]
    weight = torch.exp(log_decay * (lengths[sample] - 1 - row)[:, None].float())   # [n, H]

    def pad(x):
        dense = torch.zeros(B * max_len, H, D, device=x.device).index_copy(0, sample * max_len + row, x)
        return dense.view(B, max_len, H, D).transpose(1, 2).contiguous()

    return torch.exp(log_decay * lengths[:, None].float())[..., None, None] * initial + pad(k.float() * weight[..., None]).transpose(-1, -2) @ pad(v.float())


def _plain_norm(x, weight, bias, eps):
    x32 = x.float()
    centred = x32 - x32.mean(-1, keepdim=True)
    return (centred * torch.rsqrt(centred.square().mean(-1, keepdim=True) + eps) * weight.float() + bias.float()).to(x.dtype)


class _PlainLookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale):
        V = table.shape[0]
        inside = (ids >= 0) & (ids < V)
        ctx.save_for_backward(ids, inside)
        ctx.like, ctx.scale = table, scale
        return torch.where(inside[:, None], table[ids.clamp(0, V - 1)].float() * scale, 0.0).to(table.dtype)

    @staticmethod
    def backward(ctx, dout):
        ids, inside = ctx.saved_tensors
        V, N = ctx.like.shape
        kind = torch.float64 if dout.dtype == torch.float32 else torch.float32   # a frequent id's sum is a long one
        rows = torch.where(inside[:, None], dout.to(kind), 0.0)
        return (torch.zeros(V, N, device=dout.device, dtype=kind).index_add_(0, ids.clamp(0, V - 1), rows) * ctx.scale).to(dout.dtype), None, None


def run(state):
    case = state["case"]
    if own:
        from paper_2409_15373_amd import autograd, binding
    if case["op"] == "linear":
        q, k, v, log_decay, offsets = (state[x] for x in ("q", "k", "v", "log_decay", "offsets"))
        max_len, scale, initial = case["max_len"], state["scale"], state.get("initial")
        if case["states"]:
            if own:
                out, final = autograd.jagged_linear_attention(q, k, v, log_decay, offsets, max_len, scale=scale, initial_state=initial, return_state=True)
            else:
                out, final = (_plain_linear(q, k, v, log_decay, offsets, max_len, scale, initial),
                              _plain_final_state(k, v, log_decay, offsets, max_len, initial))
            return {"out": out, "final_state": final}
        if own:
            out = autograd.jagged_linear_attention(q, k, v, log_decay, offsets, max_len, scale=scale)
        else:
            out = _plain_linear(q, k, v, log_decay, offsets, max_len, scale, None)
        if case["mode"] == "prompt":
            return {"out": out}
        dq, dk, dv = torch.autograd.grad(out, (q, k, v), state["dout"])
        return {"out": out.detach(), "dq": dq, "dk": dk, "dv": dv}
    if case["op"] == "step":
        q, k, v, log_decay, S = (state[x] for x in ("q", "k", "v", "log_decay", "state"))
        if own:
            out, new = binding.jfa_linear_attention_step(q, k, v, log_decay, S, state["scale"], new_state=state["out_state"])
            return {"out": out, "state": new}
        new = S * torch.exp(log_decay)[:, None, None] + k.float()[..., :, None] * v.float()[..., None, :]
        return {"out": ((q.float()[..., None, :] @ new)[..., 0, :] * state["scale"]).to(q.dtype), "state": new}
    if case["op"] == "norm":
        x, weight, bias = state["x"], state["weight"], state["bias"]
        y = autograd.jagged_layer_norm(x, weight, bias, eps=1e-5) if own else _plain_norm(x, weight, bias, 1e-5)
        if case["mode"] == "forward":
            return {"y": y}
        dx, dweight, dbias = torch.autograd.grad(y, (x, weight, bias), state["dout"])
        return {"y": y.detach(), "dx": dx, "dweight": dweight, "dbias": dbias}
    table, ids, scale = state["table"], state["ids"], state["scale"]
    out = autograd.jagged_embedding(table, ids, scale=scale) if own else _PlainLookup.apply(table, ids, scale)
    if case["mode"] == "forward":
        return {"out": out}
    return {"out": out.detach(), "dtable": torch.autograd.grad(out, table, state["dout"])[0]}


# ---- in 64 bits, from the definitions --------------------------------------------------------------------------------

def _exact_linear(case, state):
    """Row against row, a sample and a block of rows at a time."""
    lam, scale, train = state["log_decay"].double(), state["scale"], case["mode"] == "train"
    bounds = state["offsets"].tolist()
    outputs = {"out": torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")}
    if train:
        outputs.update({name: torch.zeros_like(outputs["out"]) for name in ("dq", "dk", "dv")})
    if case["states"]:
        outputs["final_state"] = torch.empty(state["initial"].shape, dtype=torch.float64, device="cuda")

    def rows(name, lo, hi):
        return state[name].detach()[lo:hi].double().transpose(0, 1).contiguous()   # [H, rows, D]

    for b, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        L = hi - lo
        k, v = rows("k", lo, hi), rows("v", lo, hi)
        i = torch.arange(L, dtype=torch.float64, device="cuda")
        for r0 in range(0, L, 1024):
            r1 = min(L, r0 + 1024)
            q = rows("q", lo + r0, lo + r1)
            apart = i[r0:r1, None] - i[None, :r1]
            weight = torch.exp(lam[:, None, None] * apart) * (apart >= 0) * scale   # [H, rows, r1]
            probs = weight * torch.matmul(q, k[:, :r1].transpose(1, 2).contiguous())
            out = torch.matmul(probs, v[:, :r1])
            if case["states"]:
                out += scale * torch.exp(lam[:, None] * (i[r0:r1] + 1))[..., None] * torch.matmul(q, state["initial"][b].double())
            outputs["out"][lo + r0:lo + r1] = out.transpose(0, 1)
            if train:
                dout = rows("dout", lo + r0, lo + r1)
                dprobs = weight * torch.matmul(dout, v[:, :r1].transpose(1, 2).contiguous())
                outputs["dq"][lo + r0:lo + r1] = torch.matmul(dprobs, k[:, :r1]).transpose(0, 1)
                outputs["dk"][lo:lo + r1] += torch.matmul(dprobs.transpose(1, 2).contiguous(), q).transpose(0, 1)
                outputs["dv"][lo:lo + r1] += torch.matmul(probs.transpose(1, 2).contiguous(), dout).transpose(0, 1)
        if case["states"]:
            left = torch.exp(lam[:, None] * (L - 1 - i))[..., None]
            outputs["final_state"][b] = torch.exp(lam * L)[:, None, None] * state["initial"][b].double() + torch.matmul((k * left).transpose(1, 2).contiguous(), v)
    return outputs


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(case, state)
    if case["op"] == "step":
        q, k, v, S = (state[x].double() for x in ("q", "k", "v", "state"))
        S = torch.exp(state["log_decay"].double()).view(-1, 1, 1) * S + k.unsqueeze(-1) * v.unsqueeze(-2)
        return {"out": state["scale"] * (q.unsqueeze(-1) * S).sum(-2), "state": S}
    if case["op"] == "norm":
        x, w, b = (state[name].detach().double() for name in ("x", "weight", "bias"))
        N = x.shape[1]
        deviation = x - x.sum(1, keepdim=True) / N
        rstd = 1.0 / torch.sqrt((deviation * deviation).sum(1, keepdim=True) / N + 1e-5)
        hat = deviation * rstd
        outputs = {"y": hat * w + b}
        if case["mode"] == "train":
            dy = state["dout"].double()
            outputs["dweight"], outputs["dbias"] = (dy * hat).sum(0), dy.sum(0)
            dhat = dy * w
            outputs["dx"] = rstd * (dhat - dhat.sum(1, keepdim=True) / N - hat * ((dhat * hat).sum(1, keepdim=True) / N))
            outputs = {name: outputs[name] for name in ("y", "dx", "dweight", "dbias")}
        return outputs
    table, ids = state["table"].detach(), state["ids"]
    outputs = {"out": table[ids].double() * state["scale"]}
    if case["mode"] == "train":
        order = torch.argsort(ids, stable=True)
        sums = torch.cat([torch.zeros(1, table.shape[1], dtype=torch.float64, device="cuda"), torch.cumsum(state["dout"].double()[order], 0)])
        ends = torch.searchsorted(ids[order], torch.arange(table.shape[0], device="cuda"), right=True)
        starts = torch.searchsorted(ids[order], torch.arange(table.shape[0], device="cuda"))
        outputs["dtable"] = (sums[ends] - sums[starts]) * state["scale"]
    return outputs
