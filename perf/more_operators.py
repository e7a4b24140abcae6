"""Timed operators around the experts of a block that is trained on ragged workers: what turns tokens into rows, the
experts' products, and dense products.

  op = "gated"      gated feed-forward of rows sorted by expert, y = (act(x Wg[e]) * (x Wu[e])) Wd[e]: direction "forward"
                    (with keep: the two pre-activations are outputs too) or "backward" (the gradient of the rows and every
                    worker's gradients of the three weights, from the kept pre-activations)
  op = "linear"     act(x W + bias) + residual: "forward" or "backward" (the gradient of the rows and every worker's
                    gradients of weight and bias)
  op = "embedding"  scale * table[id]: "forward" or "backward" (every worker's gradient of the table)

Sizes are plain values: `b` are the workers' batch sizes in tokens; a token has `top_k` sorted rows, some of which a
capacity has `dropped`.  `pad` elements stand between rows of activations.  With `own` false an operator is computed from
elementary torch operations in 32 bits; with `own` true by the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIXTEEN = "637,547,469,402,345,296,254,218,187,160,137,118,101,87,74,64"
SEVEN = "600,399,266,0,133,90,43"


# ---- the cases ------------------------------------------------------------------------------

def listed():
    return [
        # sixteen sequences that write their next token, 8 of 64 experts each: about two rows to an expert, and all that
        # counts is how fast the weights arrive
        dict(name="gated 16 tokens 8 of 64", op="gated", direction="forward", dtype="bf16", grads="bf16", b="16", top_k=8,
             experts=64, cols=2048, hidden=1024, act="silu", pad=0, keep=False, dropped=0.0),
        # a large training batch, 2 of 8 wide experts, pre-activations kept: the largest case
        dict(name="gated 16384x4096x4096 2 of 8", op="gated", direction="forward", dtype="bf16", grads="bf16",
             b="4096,4096,4096,4096", top_k=2, experts=8, cols=4096, hidden=4096, act="silu", pad=0, keep=True, dropped=0.0),
        # many narrow experts, some choices cut off by a capacity
        dict(name="gated 4096x2048x768 8 of 128", op="gated", direction="forward", dtype="bf16", grads="bf16",
             b="2048,1024,1024", top_k=8, experts=128, cols=2048, hidden=768, act="silu", pad=0, keep=True, dropped=0.02),
        # the gradients of a training batch of four workers
        dict(name="gated grad 8192x2048x2048 2 of 8", op="gated", direction="backward", dtype="bf16", grads="bf16",
             b="4096,2048,1024,1024", top_k=2, experts=8, cols=2048, hidden=2048, act="silu", pad=0, keep=True, dropped=0.0),
        # the gradients in fp32 at odd sizes, seven workers, one of them idle, many choices dropped
        dict(name="gated grad 1531x777x301 f32 3 of 11", op="gated", direction="backward", dtype="f32", grads="f32",
             b=SEVEN, top_k=3, experts=11, cols=777, hidden=301, act="gelu", pad=3, keep=True, dropped=0.2),
        # one token through a wide layer: the weight is read once
        dict(name="linear token 4096x14336", op="linear", direction="forward", dtype="bf16", grads="bf16", b="1", n_in=4096,
             n_out=14336, act="gelu", pad=0, bias=True, residual=False, keep=False),
        # a layer of the wide dense benchmark with everything that an epilogue does
        dict(name="linear 4096x4096x4096 residual", op="linear", direction="forward", dtype="bf16", grads="bf16", b="4096",
             n_in=4096, n_out=4096, act="gelu", pad=0, bias=True, residual=True, keep=True),
        # its gradients, sixteen ragged workers
        dict(name="linear grad 4096x4096x4096 K16", op="linear", direction="backward", dtype="bf16", grads="bf16", b=SIXTEEN,
             n_in=4096, n_out=4096, act="gelu", pad=0, bias=True, residual=False, keep=True),
        # fp32 at odd sizes
        dict(name="linear 1531x2050x777 f32", op="linear", direction="forward", dtype="f32", grads="f32", b=SEVEN,
             n_in=2050, n_out=777, act="relu", pad=5, bias=True, residual=True, keep=True),
        # sixteen sequences' next tokens become rows: latency
        dict(name="embedding 16 of 32000x4096", op="embedding", direction="forward", dtype="bf16", b="16", vocabulary=32000,
             cols=4096, pad=0, scale=64.0, foreign=0.0),
        # a training batch of four workers over a large vocabulary: most of the table gets no token
        dict(name="embedding grad 16384 of 32000x2048", op="embedding", direction="backward", dtype="bf16",
             b="8192,4096,2048,2048", vocabulary=32000, cols=2048, pad=0, scale=1.0, foreign=0.0),
        # a small odd vocabulary in fp32, padding tokens among the others
        dict(name="embedding grad 1531 of 1009x301 f32", op="embedding", direction="backward", dtype="f32", b=SEVEN,
             vocabulary=1009, cols=301, pad=3, scale=0.5, foreign=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _split(rng, total, K):
    cut = [0] + sorted(rng.randint(0, total) for _ in range(K - 1)) + [total]
    return ",".join(str(cut[k + 1] - cut[k]) for k in range(K))


def _width(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.6 else n


def draw(rng):
    most = {op: [max(work(c)[m] for c in listed() if c["op"] == op) for m in ("bytes", "flops")]
            for op in ("gated", "linear", "embedding")}
    while True:
        op = rng.choice(["gated", "gated", "linear", "linear", "embedding"])
        K = rng.choice([1, rng.randint(2, 8)])
        tokens = _log_int(rng, 1, 16384)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = dict(op=op, direction=rng.choice(["forward", "backward"]), dtype=dtype, grads=dtype, b=_split(rng, tokens, K),
                 pad=rng.choice([0, 0, 8, rng.randint(1, 31)]))
        room = 0
        if op == "embedding":
            del c["grads"]
            c.update(vocabulary=_log_int(rng, 100, 131072), cols=_width(rng, 64, 8192),
                     scale=rng.choice([1.0, 0.5, 64.0]), foreign=rng.choice([0.0, 0.1]))
        elif op == "linear":
            c.update(n_in=_width(rng, 64, 8192), n_out=_width(rng, 64, 16384), act=rng.choice(["none", "relu", "gelu", "silu"]),
                     bias=rng.random() < 0.7, residual=rng.random() < 0.5, keep=rng.random() < 0.5)
            room = tokens * K * max(c["n_in"], c["n_out"])
        else:
            c["top_k"] = rng.randint(1, 8)
            c["experts"] = max(c["top_k"], _log_int(rng, 1, 128))
            c.update(cols=_width(rng, 64, 4096), hidden=_width(rng, 64, 8192), act=rng.choice(["silu", "silu", "gelu", "relu"]),
                     keep=rng.random() < 0.5, dropped=rng.choice([0.0, 0.02, 0.2]))
            room = tokens * c["top_k"] * K * max(c["cols"], c["hidden"])
        w = work(c)
        # (room: what the plain form's groups take when they are filled up to the same length)
        if w["bytes"] <= most[op][0] and w["flops"] <= most[op][1] and room < 1 << 30:
            return c


# ---- what a program has in hand ---------------------------------------------------------------

def _workers(case):
    return [int(v) for v in case["b"].split(",")]


def _new(*shape, dtype=torch.float32):
    return torch.empty(*shape, device=DEV, dtype=dtype)


def _rows(g, rows, cols, pad, dtype, scale=1.0):
    """[rows][cols] inside rows of cols + pad elements."""
    t = _new(rows, cols + pad, dtype=dtype)
    t.copy_(torch.randn(rows, cols + pad, generator=g, device=DEV).mul_(scale))
    return t[:, :cols]


def _weights(g, *shape, dtype):
    t = _new(*shape, dtype=dtype)
    flat = t.view(-1, shape[-2], shape[-1])
    for w in flat:
        w.copy_(torch.randn(shape[-2], shape[-1], generator=g, device=DEV).mul_(shape[-2] ** -0.5))
    return t


def _groups(bounds):
    """For groups of rows [bounds[i], bounds[i + 1]): the rows of each, filled up to the longest, and which of them count."""
    first, last = bounds[..., :-1].reshape(-1, 1), bounds[..., 1:].reshape(-1, 1)
    longest = max(1, int((last - first).max()))
    at = first + torch.arange(longest, device=DEV)
    live = at < last
    return torch.where(live, at, 0), live


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s = dict(case=case, b=_workers(case))
    return {"gated": _prepare_gated, "linear": _prepare_linear, "embedding": _prepare_embedding}[case["op"]](case, s, g)


def _prepare_gated(case, s, g):
    E, H, F, k, dt, pad, K = (case["experts"], case["cols"], case["hidden"], case["top_k"], TYPES[case["dtype"]], case["pad"],
                              len(s["b"]))
    T = sum(s["b"])
    R = T * k
    # a token's experts are the best of random scores on top of how popular each expert is; the rows of an expert stand
    # in the order of the tokens, so that each worker's follow each other
    score = torch.rand(T, E, generator=g, device=DEV).log().neg_().log_().neg_()
    score += 0.7 * torch.randn(E, generator=g, device=DEV)
    ids = score.topk(k, dim=1).indices
    kept = torch.rand(T, k, generator=g, device=DEV) >= case["dropped"]
    worker = torch.repeat_interleave(torch.arange(K, device=DEV), torch.tensor(s["b"], device=DEV), output_size=T)
    counts = torch.bincount((ids * K + worker[:, None])[kept], minlength=E * K)
    ends = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    s["segments"] = torch.stack([ends[i:i + E * K:K] if i < K else ends[K::K] for i in range(K + 1)], 1).to(torch.int32).contiguous()
    s["offsets"] = ends[::K].to(torch.int32).contiguous()
    s["x"] = _rows(g, R, H, pad, dt)
    s["wg"], s["wu"] = _weights(g, E, H, F, dtype=dt), _weights(g, E, H, F, dtype=dt)
    s["wd"] = _weights(g, E, F, H, dtype=dt)
    s["of_expert"] = _groups(s["offsets"].long())
    if case["direction"] == "backward":
        s["of_worker"] = _groups(s["segments"].long())
        s["gate"], s["up"] = _rows(g, R, F, 0, dt), _rows(g, R, F, 0, dt)
        s["dy"] = _rows(g, R, H, pad, dt, 1e-2)
    if own:
        from paper_2305_12213_amd import binding
        s["desc"] = d = binding.gated_block_desc(case["dtype"], H, F, E, R, activation=case["act"], grad=case["grads"],
                                                 ld_x=H + pad, ld_y=H, ld_dy=H + pad, ld_dx=H)
        if case["direction"] == "forward":
            s["bytes"] = binding.gated_block_workspace_bytes(d)
            s["y"] = _new(R, H, dtype=dt).zero_()
            s["gate"], s["up"] = (_new(R, F, dtype=dt).zero_() if case["keep"] else None for _ in range(2))
        else:
            s["bytes"] = binding.gated_block_backward_workspace_bytes(d, K)
            s["dx"], gt = _new(R, H, dtype=dt).zero_(), TYPES[case["grads"]]
            s["grads"] = _new(K, 3, E * H * F, dtype=gt)
        s["workspace"] = _new(max(1, s["bytes"]), dtype=torch.uint8)
    return s


def _prepare_linear(case, s, g):
    n, m, dt, pad, T, K = case["n_in"], case["n_out"], TYPES[case["dtype"]], case["pad"], sum(s["b"]), len(s["b"])
    s["x"] = _rows(g, T, n, pad, dt)
    s["w"] = _weights(g, n, m, dtype=dt)
    s["bias"] = torch.randn(m, generator=g, device=DEV).mul_(0.1) if case["bias"] else None
    if case["direction"] == "forward":
        s["residual"] = _rows(g, T, m, pad, dt, 2.0) if case["residual"] else None
    else:
        ends = torch.tensor([sum(s["b"][:i]) for i in range(K + 1)], device=DEV)
        s["of_worker"] = _groups(ends)
        s["pre"] = _rows(g, T, m, 0, dt) if case["act"] != "none" else None
        s["dout"] = _rows(g, T, m, pad, dt, 1e-2)
    if own:
        from paper_2305_12213_amd import binding
        s["desc"] = d = binding.linear_desc(case["dtype"], n, m, activation=case["act"], grad=case["grads"], ld_x=n + pad,
                                            ld_residual=m + pad, ld_dout=m + pad)
        if case["direction"] == "forward":
            s["out"], s["kept"] = _new(T, m, dtype=dt), _new(T, m, dtype=dt) if case["keep"] else None
            s["bytes"] = binding.linear_workspace_bytes(d, T)
        else:
            s["dx"], gt = _new(T, n, dtype=dt), TYPES[case["grads"]]
            s["dw"], s["db"] = _new(K, n * m, dtype=gt), _new(K, m, dtype=gt) if case["bias"] else None
            s["bytes"] = binding.linear_backward_workspace_bytes(d, s["b"])
        s["workspace"] = _new(max(1, s["bytes"]), dtype=torch.uint8)
    return s


def _prepare_embedding(case, s, g):
    V, H, dt, pad, T, K = case["vocabulary"], case["cols"], TYPES[case["dtype"]], case["pad"], sum(s["b"]), len(s["b"])
    # a few tokens make up much of any text: the n-th of them appears about 1 / n times as often as the first
    u = torch.rand(T, generator=g, device=DEV, dtype=torch.float64)
    s["ids"] = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1).to(torch.int32)
    # some places hold no token of the vocabulary
    s["ids"][torch.rand(T, generator=g, device=DEV) < case["foreign"]] = -1
    if case["direction"] == "forward":
        s["table"] = _rows(g, V, H, pad, dt, H ** -0.5)
    else:
        s["dout"] = _rows(g, T, H, pad, dt, 1e-2)
        s["worker"] = torch.repeat_interleave(torch.arange(K, device=DEV), torch.tensor(s["b"], device=DEV), output_size=T)
    if own:
        from paper_2305_12213_amd import binding
        s["desc"] = d = binding.embedding_desc(case["dtype"], H, V, T, scale=case["scale"], ld_table=H + pad, ld_dout=H + pad)
        if case["direction"] == "forward":
            s["out"] = _new(T, H, dtype=dt)
        else:
            s["dtable"] = _new(K, V, H)
            s["bytes"] = binding.embedding_backward_workspace_bytes(d, K)
            s["workspace"] = _new(max(1, s["bytes"]), dtype=torch.uint8)
    return s


# ---- one pass -----------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return {"gated": _own_gated, "linear": _own_linear, "embedding": _own_embedding}[case["op"]](s, case)
    return {"gated": _plain_gated, "linear": _plain_linear, "embedding": _plain_embedding}[case["op"]](s, case)


def _own_gated(s, case):
    from paper_2305_12213_amd import binding
    d = s["desc"]
    if case["direction"] == "forward":
        binding.gated_block(d, s["offsets"], s["x"], s["wg"], s["wu"], s["wd"], s["gate"], s["up"], s["y"], s["workspace"],
                            s["bytes"])
        return dict(y=s["y"], gate=s["gate"], up=s["up"]) if case["keep"] else dict(y=s["y"])
    G = s["grads"]
    binding.gated_block_backward(d, len(s["b"]), s["offsets"], s["segments"], s["x"], s["wg"], s["wu"], s["wd"], s["gate"],
                                 s["up"], s["dy"], s["dx"], G[0, 0], G[0, 1], G[0, 2], G.stride(0), s["workspace"], s["bytes"])
    E, H, F, K = case["experts"], case["cols"], case["hidden"], len(s["b"])
    return dict(dx=s["dx"], dwg=G[:, 0].view(K, E, H, F), dwu=G[:, 1].view(K, E, H, F), dwd=G[:, 2].view(K, E, F, H))


def _own_linear(s, case):
    from paper_2305_12213_amd import binding
    if case["direction"] == "forward":
        binding.linear(s["desc"], s["x"].shape[0], s["x"], s["w"], s["bias"], s["residual"], s["kept"], s["out"], s["workspace"],
                       s["bytes"])
        return dict(out=s["out"], pre=s["kept"]) if case["keep"] else dict(out=s["out"])
    binding.linear_backward(s["desc"], s["b"], s["x"], s["w"], s["pre"], s["dout"], s["dx"], s["dw"], s["dw"].stride(0), s["db"],
                            case["n_out"], s["workspace"], s["bytes"])
    found = dict(dx=s["dx"], dw=s["dw"].view(-1, case["n_in"], case["n_out"]))
    if case["bias"]:
        found["db"] = s["db"]
    return found


def _own_embedding(s, case):
    from paper_2305_12213_amd import binding
    if case["direction"] == "forward":
        binding.embedding(s["desc"], s["ids"], s["table"], s["out"])
        return dict(out=s["out"])
    binding.embedding_backward(s["desc"], s["b"], s["ids"], s["dout"], s["dtable"], case["vocabulary"] * case["cols"],
                               s["workspace"], s["bytes"])
    return dict(dtable=s["dtable"])


# ---- the plain forms ------------------------------------------------------------------------------

def _act(name, v):
    """An activation and its derivative."""
    if name == "none":
        return v, torch.ones_like(v)
    if name == "relu":
        return v.clamp_min(0.0), (v > 0).to(v.dtype)
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-v))
        return v * p, p * (1.0 + v * (1.0 - p))
    p = 0.5 * (1.0 + torch.erf(v * 0.5 ** 0.5))
    return v * p, p + v * torch.exp(-0.5 * v * v) * (2.0 * math.pi) ** -0.5


def _grouped(x, groups):
    """The rows of each group in 32 bits, zeros where it has none."""
    at, live = groups
    return x[at].float().masked_fill_(~live[..., None], 0.0)


def _scattered(v, groups, rows):
    """The groups' rows back in their places."""
    at, live = groups
    out = torch.zeros(rows, v.shape[-1], device=DEV)
    out[at[live]] = v[live]
    return out


def _plain_gated(s, case):
    dt, R, by = TYPES[case["dtype"]], s["x"].shape[0], s["of_expert"]
    if case["direction"] == "forward":
        z = _grouped(s["x"], by)
        gate, up = torch.bmm(z, s["wg"].float()), torch.bmm(z, s["wu"].float())
        y = torch.bmm(_act(case["act"], gate)[0] * up, s["wd"].float())
        out = dict(y=_scattered(y, by, R).to(dt))
        if case["keep"]:
            out.update(gate=_scattered(gate, by, R).to(dt), up=_scattered(up, by, R).to(dt))
        return out
    dy, gate, up = _grouped(s["dy"], by), _grouped(s["gate"], by), _grouped(s["up"], by)
    a, slope = _act(case["act"], gate)
    dh = torch.bmm(dy, s["wd"].float().transpose(1, 2).contiguous())
    dgate, dup, hidden = dh * up * slope, dh * a, a * up
    dx = torch.bmm(dgate, s["wg"].float().transpose(1, 2).contiguous())
    dx += torch.bmm(dup, s["wu"].float().transpose(1, 2).contiguous())
    of, K, E, gt = s["of_worker"], len(s["b"]), case["experts"], TYPES[case["grads"]]
    turned = lambda t: t.transpose(1, 2).contiguous()  # noqa: E731
    by_worker = lambda t: t.view(E, K, *t.shape[1:]).transpose(0, 1).to(gt)  # noqa: E731
    z, dgate, dup = (_grouped(t, of) for t in (s["x"], _scattered(dgate, by, R), _scattered(dup, by, R)))
    hidden, dy = _grouped(_scattered(hidden, by, R), of), _grouped(s["dy"], of)
    z = turned(z)
    return dict(dx=_scattered(dx, by, R).to(dt), dwg=by_worker(torch.bmm(z, dgate)), dwu=by_worker(torch.bmm(z, dup)),
                dwd=by_worker(torch.bmm(turned(hidden), dy)))


def _plain_linear(s, case):
    dt = TYPES[case["dtype"]]
    if case["direction"] == "forward":
        pre = s["x"].float() @ s["w"].float()
        if s["bias"] is not None:
            pre = pre + s["bias"]
        out = _act(case["act"], pre)[0]
        if s["residual"] is not None:
            out = out + s["residual"].float()
        return dict(out=out.to(dt), pre=pre.to(dt)) if case["keep"] else dict(out=out.to(dt))
    dpre = s["dout"].float()
    if s["pre"] is not None:
        dpre = dpre * _act(case["act"], s["pre"].float())[1]
    gt, of = TYPES[case["grads"]], s["of_worker"]
    x, d = _grouped(s["x"], of), _grouped(dpre, of)
    found = dict(dx=(dpre @ s["w"].float().t()).to(dt), dw=torch.bmm(x.transpose(1, 2).contiguous(), d).to(gt))
    if case["bias"]:
        found["db"] = d.sum(1).to(gt)
    return found


def _plain_embedding(s, case):
    ids, V = s["ids"].long(), case["vocabulary"]
    here = (ids >= 0) & (ids < V)
    if case["direction"] == "forward":
        rows = s["table"][torch.where(here, ids, 0)].float() * case["scale"]
        return dict(out=rows.masked_fill_(~here[:, None], 0.0).to(TYPES[case["dtype"]]))
    K = len(s["b"])
    out = torch.zeros(K * V, case["cols"], device=DEV)
    out.index_add_(0, (s["worker"] * V + ids)[here], s["dout"][here].float())
    return dict(dtable=out.mul_(case["scale"]).view(K, V, -1))


# ---- from the definition in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"gated": _exact_gated, "linear": _exact_linear, "embedding": _exact_embedding}[case["op"]](s, case)


def _curve(name, v):
    """An activation and its derivative, in 64 bits."""
    if name == "none":
        return v, torch.ones_like(v)
    if name == "relu":
        return torch.where(v > 0, v, 0.0), torch.where(v > 0, 1.0, 0.0).double()
    if name == "silu":
        half = torch.tanh(v / 2)
        return v * (1 + half) / 2, (1 + half) / 2 + v * (1 - half * half) / 4
    return v * torch.special.ndtr(v), torch.special.ndtr(v) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)


def _exact_gated(s, case):
    R, H, F, E, K = s["x"].shape[0], case["cols"], case["hidden"], case["experts"], len(s["b"])
    cut = s["segments"].tolist()
    zeros = lambda *shape: torch.zeros(*shape, device=DEV, dtype=torch.float64)  # noqa: E731
    if case["direction"] == "forward":
        y, gate, up = zeros(R, H), zeros(R, F), zeros(R, F)
        for e in range(E):
            r = slice(cut[e][0], cut[e][K])
            x = s["x"][r].double()
            gate[r], up[r] = x @ s["wg"][e].double(), x @ s["wu"][e].double()
            y[r] = (_curve(case["act"], gate[r])[0] * up[r]) @ s["wd"][e].double()
        return dict(y=y, gate=gate, up=up) if case["keep"] else dict(y=y)
    dx, dwg, dwu, dwd = zeros(R, H), zeros(K, E, H, F), zeros(K, E, H, F), zeros(K, E, F, H)
    for e in range(E):
        r = slice(cut[e][0], cut[e][K])
        dh = s["dy"][r].double() @ s["wd"][e].double().t()
        a, slope = _curve(case["act"], s["gate"][r].double())
        dgate, dup, hidden = dh * s["up"][r].double() * slope, dh * a, a * s["up"][r].double()
        dx[r] = dgate @ s["wg"][e].double().t() + dup @ s["wu"][e].double().t()
        for k in range(K):
            q = slice(cut[e][k], cut[e][k + 1])
            p = slice(q.start - r.start, q.stop - r.start)
            dwg[k, e], dwu[k, e] = s["x"][q].double().t() @ dgate[p], s["x"][q].double().t() @ dup[p]
            dwd[k, e] = hidden[p].t() @ s["dy"][q].double()
    return dict(dx=dx, dwg=dwg, dwu=dwu, dwd=dwd)


def _exact_linear(s, case):
    w = s["w"].double()
    if case["direction"] == "forward":
        pre = s["x"].double() @ w
        if case["bias"]:
            pre += s["bias"].double()
        out = _curve(case["act"], pre)[0]
        if case["residual"]:
            out = out + s["residual"].double()
        return dict(out=out, pre=pre) if case["keep"] else dict(out=out)
    d = s["dout"].double()
    if case["act"] != "none":
        d = d * _curve(case["act"], s["pre"].double())[1]
    x, ends = s["x"].double(), [sum(s["b"][:i]) for i in range(len(s["b"]) + 1)]
    parts = [slice(i, j) for i, j in zip(ends, ends[1:])]
    found = dict(dx=d @ w.t(), dw=torch.stack([x[r].t() @ d[r] for r in parts]))
    if case["bias"]:
        found["db"] = torch.stack([d[r].sum(0) for r in parts])
    return found


def _exact_embedding(s, case):
    ids, V, K = s["ids"], case["vocabulary"], len(s["b"])
    if case["direction"] == "forward":
        out = torch.zeros(ids.shape[0], case["cols"], device=DEV, dtype=torch.float64)
        there = torch.nonzero((ids >= 0) & (ids < V))[:, 0]
        out[there] = s["table"][ids[there].long()].double() * case["scale"]
        return dict(out=out)
    # tokens in the order of (worker, id): differences of running sums at the ends of each run
    worker = torch.repeat_interleave(torch.arange(K, device=DEV), torch.tensor(s["b"], device=DEV))
    there = torch.nonzero((ids >= 0) & (ids < V))[:, 0]
    key = worker[there] * V + ids[there].long()
    key, order = torch.sort(key)
    found, counts = torch.unique_consecutive(key, return_counts=True)
    sums = torch.cumsum(s["dout"][there[order]].double(), 0)[torch.cumsum(counts, 0) - 1] if len(found) else None
    out = torch.zeros(K * V, case["cols"], device=DEV, dtype=torch.float64)
    if sums is not None:
        out[found] = torch.diff(sums, dim=0, prepend=torch.zeros_like(sums[:1])) * case["scale"]
    return dict(dtable=out.view(K, V, -1))


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    b = _workers(case)
    T, K, size = sum(b), len(b), {"f32": 4, "bf16": 2}[case["dtype"]]
    back = case["direction"] == "backward"
    if case["op"] == "embedding":
        V, H = case["vocabulary"], case["cols"]
        here = T * (1.0 - case["foreign"])
        if back:
            return {"bytes": 4 * T + here * H * size + K * V * H * 4, "flops": here * H}
        return {"bytes": 4 * T + (min(here, V) + T) * H * size, "flops": here * H}
    gsize = {"f32": 4, "bf16": 2}[case["grads"]]
    if case["op"] == "linear":
        n, m = case["n_in"], case["n_out"]
        if back:
            rows = T * (2 * n + m + (m if case["act"] != "none" else 0))
            return {"bytes": rows * size + n * m * size + K * (n * m + (m if case["bias"] else 0)) * gsize,
                    "flops": 4.0 * T * n * m}
        rows = T * (n + m + (m if case["residual"] else 0) + (m if case["keep"] else 0))
        return {"bytes": rows * size + n * m * size + (4 * m if case["bias"] else 0), "flops": 2.0 * T * n * m}
    E, H, F = case["experts"], case["cols"], case["hidden"]
    rows = T * case["top_k"] * (1.0 - case["dropped"])
    weights = min(E, T * case["top_k"]) * 3 * H * F
    if back:
        return {"bytes": rows * (3 * H + 2 * F) * size + weights * size + 3 * K * E * H * F * gsize,
                "flops": 12.0 * rows * H * F}
    return {"bytes": rows * (2 * H + (2 * F if case["keep"] else 0)) * size + weights * size, "flops": 6.0 * rows * H * F}
