"""Linear attention with a decay for each head, layer norm and embedding lookup in fp64 (numpy), written from their formulas.

Linear attention goes row by row through the recurrence, its gradient row by row back through it; `magnitude` is the same sums over
absolute values, which error bounds are stated in.
"""
import numpy as np


def linear_attention(q, k, v, log_decay, offsets, scale, initial_state=None):
    """(out [n, H, D], final states [B, H, D, D])."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, H, D = q.shape
    B = len(offsets) - 1
    decay = np.exp(np.asarray(log_decay, dtype=np.float64))[:, None, None]
    out, final = np.zeros((n, H, D)), np.zeros((B, H, D, D))
    for b in range(B):
        S = np.zeros((H, D, D)) if initial_state is None else np.asarray(initial_state[b], dtype=np.float64)
        for i in range(offsets[b], offsets[b + 1]):
            S = decay * S + k[i][:, :, None] * v[i][:, None, :]
            out[i] = scale * np.einsum("hd,hde->he", q[i], S)
        final[b] = S
    return out, final


def linear_attention_backward(q, k, v, dout, log_decay, offsets, scale, initial_state=None, dfinal_state=None):
    """(dq, dk, dv [n, H, D], gradient of the initial states [B, H, D, D])."""
    q, k, v, dout = (np.asarray(x, dtype=np.float64) for x in (q, k, v, dout))
    n, H, D = q.shape
    B = len(offsets) - 1
    decay = np.exp(np.asarray(log_decay, dtype=np.float64))[:, None, None]
    dq, dk, dv, dinitial = np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((B, H, D, D))
    for b in range(B):
        S = np.zeros((H, D, D)) if initial_state is None else np.asarray(initial_state[b], dtype=np.float64)
        for i in range(offsets[b], offsets[b + 1]):
            S = decay * S + k[i][:, :, None] * v[i][:, None, :]
            dq[i] = scale * np.einsum("hde,he->hd", S, dout[i])
        dS = np.zeros((H, D, D)) if dfinal_state is None else np.asarray(dfinal_state[b], dtype=np.float64)
        for i in range(offsets[b + 1] - 1, offsets[b] - 1, -1):
            dS = dS + scale * q[i][:, :, None] * dout[i][:, None, :]
            dk[i] = np.einsum("hde,he->hd", dS, v[i])
            dv[i] = np.einsum("hde,hd->he", dS, k[i])
            dS = decay * dS
        dinitial[b] = dS
    return dq, dk, dv, dinitial


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd) over the last dimension."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(-1)
    rstd = 1.0 / np.sqrt(((x - mean[..., None]) ** 2).mean(-1) + eps)
    y = (x - mean[..., None]) * rstd[..., None]
    return y * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64)), mean, rstd


def layer_norm_backward(x, weight, dy, eps):
    """(dx, dweight, dbias); dweight and dbias are sums over all but the last dimension."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    hat, _, rstd = layer_norm(x, None, None, eps)
    dhat = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = rstd[..., None] * (dhat - dhat.mean(-1, keepdims=True) - hat * (dhat * hat).mean(-1, keepdims=True))
    lead = tuple(range(x.ndim - 1))
    return dx, (dy * hat).sum(lead), dy.sum(lead)


def embedding(table, ids, scale):
    table, ids = np.asarray(table, dtype=np.float64), np.asarray(ids)
    inside = (ids >= 0) & (ids < len(table))
    return np.where(inside[:, None], scale * table[np.where(inside, ids, 0)], 0.0)


def embedding_backward(dout, ids, V, scale):
    dout, ids = np.asarray(dout, dtype=np.float64), np.asarray(ids)
    dtable = np.zeros((V, dout.shape[1]))
    for i, v in enumerate(ids):
        if 0 <= v < V:
            dtable[v] += scale * dout[i]
    return dtable
