"""Plain forms, in 64 bits, of dense layers with bias, activation and residual, of gated feed-forward blocks of routed experts
and of embeddings, and of their gradients.  Written from the formulas; shares no code with the library."""
import math

import numpy as np


def _erf(v):
    return np.vectorize(math.erf, otypes=[np.float64])(v)


def activate(name, v):
    v = np.asarray(v, np.float64)
    if name == "none":
        return v.copy()
    if name == "relu":
        return np.where(v < 0, 0.0, v)
    if name == "silu":
        return v * (0.5 + 0.5 * np.tanh(0.5 * v))
    return v * (0.5 + 0.5 * _erf(v / math.sqrt(2)))


def slope(name, v):
    v = np.asarray(v, np.float64)
    if name == "none":
        return np.ones_like(v)
    if name == "relu":
        return np.where(v > 0, 1.0, 0.0)
    if name == "silu":
        p = 0.5 + 0.5 * np.tanh(0.5 * v)
        return p * (1 + v * (1 - p))
    return 0.5 + 0.5 * _erf(v / math.sqrt(2)) + v * np.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)


def linear(x, weight, bias, residual, act):
    """(out, what the activation is taken of)"""
    pre = x @ weight + (0.0 if bias is None else bias)
    return activate(act, pre) + (0.0 if residual is None else residual), pre


def linear_gradients(b, x, weight, pre, dout, act):
    """(dx, dweight of every worker, dbias of every worker)"""
    dz = dout * slope(act, pre) if act != "none" else dout
    ends = np.concatenate([[0], np.cumsum(b)]).astype(int)
    parts = [slice(i, j) for i, j in zip(ends, ends[1:])]
    return dz @ weight.T, np.stack([x[r].T @ dz[r] for r in parts]), np.stack([dz[r].sum(0) for r in parts])


def gated_block(offsets, x, w_gate, w_up, w_down, act):
    """(y, gate, up), zeros in rows that no expert has"""
    gate, up = np.zeros((x.shape[0], w_gate.shape[2])), np.zeros((x.shape[0], w_gate.shape[2]))
    y = np.zeros((x.shape[0], w_down.shape[2]))
    for e in range(len(offsets) - 1):
        r = slice(offsets[e], offsets[e + 1])
        gate[r], up[r] = x[r] @ w_gate[e], x[r] @ w_up[e]
        y[r] = (activate(act, gate[r]) * up[r]) @ w_down[e]
    return y, gate, up


def gated_block_gradients(segments, x, w_gate, w_up, w_down, gate, up, dy, act):
    """(dx, dw_gate, dw_up, dw_down), the last three of every worker"""
    E, K = segments.shape[0], segments.shape[1] - 1
    dx = np.zeros_like(x)
    dg, du, dd = (np.zeros((K,) + w.shape) for w in (w_gate, w_up, w_down))
    for e in range(E):
        r = slice(segments[e][0], segments[e][K])
        dhidden = dy[r] @ w_down[e].T
        dgate = np.zeros_like(gate)
        dup = np.zeros_like(up)
        hidden = activate(act, gate) * up
        dgate[r] = dhidden * up[r] * slope(act, gate[r])
        dup[r] = dhidden * activate(act, gate[r])
        dx[r] = dgate[r] @ w_gate[e].T + dup[r] @ w_up[e].T
        for k in range(K):
            q = slice(segments[e][k], segments[e][k + 1])
            dg[k, e], du[k, e], dd[k, e] = x[q].T @ dgate[q], x[q].T @ dup[q], hidden[q].T @ dy[q]
    return dx, dg, du, dd


def embedding(ids, table, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < table.shape[0]:
            out[t] = scale * table[i]
    return out


def embedding_gradient(b, ids, dout, vocabulary, scale):
    out = np.zeros((len(b), vocabulary, dout.shape[1]))
    worker = np.repeat(np.arange(len(b)), b)
    here = (ids >= 0) & (ids < vocabulary)
    np.add.at(out, (worker[here], ids[here]), dout[here])
    return scale * out
