"""Plain 64-bit forms of the operators around the products of a residual block with routed experts: the
root-mean-square norm and its 8-bit outputs, tokens sorted by expert and back, AdamW with the workers' average
and 8-bit states.  Written from the formulas, without the library's code.
"""
import numpy as np

FP8_TOP, INT8_TOP = 448.0, 127.0


def rms_norm(x, residual, gain, eps):
    """(s, rstd, y)."""
    s = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    with np.errstate(all="ignore"):
        rstd = 1.0 / np.sqrt(np.mean(s * s, axis=1) + eps)
        y = s * rstd[:, None] * (1.0 if gain is None else np.asarray(gain, np.float64))
    return s, rstd, y


def block_scales(y, top, block):
    """Scale of each block of `block` columns (0: the row): NaN where a value is not finite."""
    rows, cols = y.shape
    block = block or cols
    n = -(-cols // block)
    out = np.zeros((rows, n))
    for b in range(n):
        a = np.abs(y[:, b * block:(b + 1) * block])
        out[:, b] = np.where(np.isfinite(a).all(1), a.max(1, initial=0.0) / top, np.nan)
    return out


def rms_norm_grad(s, rstd, gain, dy, dsum, b):
    """(dx, dgain[K])."""
    s, dy = np.asarray(s, np.float64), np.asarray(dy, np.float64)
    shat = s * np.asarray(rstd, np.float64)[:, None]
    g = dy * (1.0 if gain is None else np.asarray(gain, np.float64))
    dx = np.asarray(rstd, np.float64)[:, None] * (g - shat * np.mean(g * shat, axis=1, keepdims=True))
    if dsum is not None:
        dx = dx + np.asarray(dsum, np.float64)
    dgain, at = [], 0
    for n in b:
        dgain.append((dy[at:at + n] * shat[at:at + n]).sum(0))
        at += n
    return dx, np.stack(dgain)


def route_plan(experts, n_experts):
    """(offsets, slot, source): choices in the order of their numbers, expert by expert."""
    ids = np.asarray(experts, np.int64)
    tokens, k = ids.shape
    flat = ids.reshape(-1)
    source = [i for e in range(n_experts) for i in np.flatnonzero(flat == e)]
    offsets = np.concatenate([[0], np.cumsum([(flat == e).sum() for e in range(n_experts)])])
    slot = np.full(tokens * k, -1, np.int64)
    slot[source] = np.arange(len(source))
    return offsets, slot.reshape(tokens, k), np.array(list(source) + [-1] * (tokens * k - len(source)), np.int64)


def route_segments(offsets, source, b, top_k):
    """segments[e][k] and, last, expert e's end."""
    first = np.concatenate([[0], np.cumsum(b)]) * top_k
    out = []
    for e in range(len(offsets) - 1):
        mine = source[offsets[e]:offsets[e + 1]]
        out.append([offsets[e] + int((mine < f).sum()) for f in first[:-1]] + [offsets[e + 1]])
    return np.array(out)


def route_gather(x, slot):
    tokens, k = slot.shape
    out = np.zeros((tokens * k, x.shape[1]))
    for t in range(tokens):
        for j in range(k):
            if slot[t, j] >= 0:
                out[slot[t, j]] = x[t]
    return out


def route_combine(sorted_rows, slot, weights, addend):
    tokens, k = slot.shape
    out = np.zeros((tokens, sorted_rows.shape[1])) if addend is None else np.array(addend, np.float64)
    for t in range(tokens):
        for j in range(k):
            if slot[t, j] >= 0:
                with np.errstate(all="ignore"):
                    out[t] = out[t] + (1.0 if weights is None else float(weights[t, j])) * sorted_rows[slot[t, j]]
    return out


def route_combine_grad(dout, sorted_rows, slot, weights):
    """(dsorted, dweights)."""
    tokens, k = slot.shape
    dsorted, dweights = np.zeros((tokens * k, dout.shape[1])), np.zeros((tokens, k))
    for t in range(tokens):
        for j in range(k):
            s = slot[t, j]
            if s >= 0:
                dsorted[s] = float(weights[t, j]) * dout[t]
                dweights[t, j] = np.dot(np.asarray(dout[t], np.float64), np.asarray(sorted_rows[s], np.float64))
    return dsorted, dweights


# ---- 8-bit states -----------------------------------------------------------------------------------------------

BLOCK = 256
TOPS = {7: 1.875, 8: 1.9375}
_M = (1 << 32) - 1


def random_bits(n, ordinal, seed):
    """The 32 bits of each element of a tensor."""
    out = []
    for i in range(n):
        x = (i * 0x9E3779B1 + ordinal * 0x7F4A7C15 + seed) & _M
        x = ((x ^ (x >> 16)) * 0x6A09E667) & _M
        x = ((x ^ (x >> 15)) * 0xBB67AE85) & _M
        out.append(x ^ (x >> 16))
    return np.array(out, np.int64)


def code_values(bits):
    """Magnitude of every code in units of the scale: 16 octaves of equal steps, less the lowest value."""
    per = 8 if bits == 7 else 16
    return np.array([2.0 ** (c // per - 15) * (1 + (c % per) / per) - 2.0 ** -15 for c in range(1 << bits)])


def encode(x, bits, u):
    """(codes, scales) of a vector; u in [0, 1): how much of a step is added before the rounding down."""
    table, x = code_values(bits), np.asarray(x, np.float64)
    codes, scales = np.zeros(len(x), np.int64), []
    for b in range(0, len(x), BLOCK):
        part = np.abs(x[b:b + BLOCK])
        if not np.isfinite(part).all():
            scales.append(np.nan)
            continue
        amax = part.max(initial=0.0)
        scale = amax / TOPS[bits] if amax >= 2.0 ** -100 else 0.0
        scales.append(scale)
        if scale == 0.0:
            continue
        t = part / scale
        low = np.clip(np.searchsorted(table, t, side="right") - 1, 0, len(table) - 2)
        frac = (t - table[low]) / (table[low + 1] - table[low])
        codes[b:b + BLOCK] = np.minimum(low + (frac + u[b:b + BLOCK] >= 1.0), len(table) - 1)
    if bits == 7:
        codes = codes | np.where(x < 0, 128, 0)
    return codes, np.array(scales)


def encode_root(root, u):
    """sqrt(v) as it is kept: 8 bits, and a positive value has code 1 at least (0 beside an m that is not 0 would make a
    step of m / eps)."""
    codes, scales = encode(root, 8, u)
    lowest = (np.asarray(root) > 0) & (np.repeat(scales, BLOCK)[:len(codes)] > 0)
    return np.maximum(codes, lowest), scales


def decode(codes, scales, bits):
    codes = np.asarray(codes, np.int64)
    table = code_values(bits)
    v = table[codes & (len(table) - 1)] * np.repeat(scales, BLOCK)[:len(codes)]
    return np.where(codes & 128, -v, v) if bits == 7 else v


def adamw(p, m, v, grads, b, decay, lr, beta1, beta2, eps, step):
    """(p, m, v) after a step; grads [K][n]."""
    total = float(sum(b))
    g = np.zeros(len(p))
    for k, n in enumerate(b):
        if n > 0:
            g = g + n / total * np.asarray(grads[k], np.float64)
    m = beta1 * np.asarray(m, np.float64) + (1 - beta1) * g
    v = beta2 * np.asarray(v, np.float64) + (1 - beta2) * g * g
    with np.errstate(all="ignore"):
        hat = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return np.asarray(p, np.float64) * (1 - lr * decay) - lr * hat, m, v
