#!/usr/bin/env python3
"""Timing of the operators around attention in a sequence model -- linear attention with a decay for each head, layer norm,
embedding lookup -- and of their gradients, against the HBM roofline.

    python -m paper_2409_15373_amd.bench.sequence_ops_bench [--B 1024] [--max-len 1024] [--H 4] [--D 128] [--V 1000003] [--dtype bf16|fp32] [--reps 10]

Lengths are uniform on [1, max_len], values random normals drawn on the device, ids Zipf-distributed.  For every operator it
reports microseconds per call (HIP events inside the library) and the rate at which it moves its algorithmic bytes: each input
and output tensor once (of the table the rows that are asked for), the state of a single token's step read and written once.
Prints one JSON line.
"""
import argparse
import json

import numpy as np


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--B", type=int, default=1024)
    ap.add_argument("--max-len", type=int, default=1024)
    ap.add_argument("--H", type=int, default=4)
    ap.add_argument("--D", type=int, default=128)
    ap.add_argument("--V", type=int, default=1000003)
    ap.add_argument("--dtype", choices=["bf16", "fp32"], default="bf16")
    ap.add_argument("--reps", type=int, default=10)
    args = ap.parse_args()
    import torch
    from .. import binding
    from ..synthetic import lengths_for, offsets_from_lengths
    binding.load()
    assert torch.cuda.is_available(), "needs the GPU"
    B, L, H, D, V = args.B, args.max_len, args.H, args.D, args.V
    dtype, size = (torch.bfloat16, 2) if args.dtype == "bf16" else (torch.float32, 4)
    lengths = lengths_for("uniform", B, L, np.random.Generator(np.random.PCG64(0)))
    n, N = int(lengths.sum()), H * D
    off = torch.from_numpy(offsets_from_lengths(lengths)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(0)
    mk = lambda *shape: torch.randn(*shape, device="cuda", generator=gen).to(dtype)
    q, k, v, dout = (mk(n, H, D) for _ in range(4))
    out, dq, dk, dv = (torch.empty_like(q) for _ in range(4))
    log_decay = torch.log1p(-torch.exp2(-torch.linspace(4.0, 11.0, H, dtype=torch.float64))).float().cuda()
    tokens, state, new_state = [mk(B, H, D) for _ in range(4)], torch.zeros(B, H, D, D, device="cuda"), torch.empty(B, H, D, D, device="cuda")
    x, dy, y, dx = q.view(n, N), dout.view(n, N), out.view(n, N), dq.view(n, N)
    w, b = mk(N), mk(N)
    _, mean, rstd = binding.jfa_layer_norm(x, w, b, off)
    weights = 1.0 / torch.arange(1, V + 1, device="cuda", dtype=torch.float64) ** 1.05
    ids = torch.searchsorted((weights / weights.sum()).cumsum(0), torch.rand(n, device="cuda", generator=gen, dtype=torch.float64)).clamp_(max=V - 1)
    distinct, table = int(torch.unique(ids).numel()), mk(V, N)
    dtable, rows = torch.empty_like(table), n * N * size
    calls = {   # name of the library's timer: (call, algorithmic bytes)
        "linear_attention": (lambda: binding.jfa_linear_attention(q, k, v, log_decay, off, L, out=out), 4 * rows),
        "linear_attention_bwd": (lambda: binding.jfa_linear_attention_backward(q, k, v, dout, log_decay, off, L, dq=dq, dk=dk, dv=dv), 7 * rows),
        "linear_attention_step": (lambda: binding.jfa_linear_attention_step(*tokens[:3], log_decay, state, out=tokens[3], new_state=new_state), 8 * B * H * D * D + 4 * B * N * size),
        "layer_norm": (lambda: binding.jfa_layer_norm(x, w, b, off, y=y), 2 * rows),
        "layer_norm_bwd": (lambda: binding.jfa_layer_norm_backward(x, w, dy, mean, rstd, off, dx=dx), 3 * rows),
        "embedding": (lambda: binding.jfa_embedding(table, ids, off, out=x), 8 * n + rows + distinct * N * size),
        "embedding_bwd": (lambda: binding.jfa_embedding_backward(dy, ids, V, off, dtable=dtable), 8 * n + rows + V * N * size),
    }
    for fn, _ in calls.values():
        fn()
    torch.cuda.synchronize()
    binding.jfa_timing_enable(True)
    binding.jfa_timing_read()
    for _ in range(args.reps):
        for fn, _ in calls.values():
            fn()
    torch.cuda.synchronize()
    timers = binding.jfa_timing_read()
    binding.jfa_timing_enable(False)
    ops = {}
    for name, (_, nbytes) in calls.items():
        ms, cnt = timers[name]
        us = ms * 1e3 / cnt
        ops[name] = {"us": round(us, 1), "algorithmic_MB": round(nbytes / 1e6, 1), "GB_per_s": round(nbytes / us / 1e3, 1), "frac_of_8TBps": round(nbytes / us / 1e3 / 8000.0, 3)}
    print(json.dumps({"workload": {"B": B, "max_len": L, "H": H, "D": D, "V": V, "rows": n, "distinct_ids": distinct, "lengths": "uniform[1, max_len]"},
                      "dtype": args.dtype, "data": "synthetic", "bound": "hbm", "operators": ops}))


if __name__ == "__main__":
    main()
