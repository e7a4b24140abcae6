"""Timed operators of a residual block with routed experts, trained on ragged workers.

  op = "norm"   root-mean-square norm with the residual's addition: direction "forward" (the sum, the
                normalised rows in the input's type or in 8 bits with scales) or "backward" (the rows'
                gradient and each worker's gradient of the gain)
  op = "route"  tokens sorted by expert and back: "forward" (the plan, the sorted rows, the weighted
                sum of the experts' outputs with the residual) or "backward" (the gradients of all of them)
  op = "adamw"  a step over many tensors with the average of the workers' gradients inside, states in
                32 or 8 bits

Sizes are plain values: `b` are the workers' batch sizes, `dims` the widths of the dense layers whose
weights, biases and gains are updated, `repeat` times over.  With `own` false an operator is computed
from elementary torch operations in 32 bits; with `own` true by the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
RULE = dict(lr=1e-4, beta1=0.9, beta2=0.95, eps=1e-8)
DECAY = 0.1


# ---- the cases ------------------------------------------------------------------------------

def listed():
    return [
        # one token while an answer is written, the output in 8 bits for the product behind it: latency
        dict(name="norm token 4096 fp8", op="norm", direction="forward", dtype="bf16", out="fp8", block=0,
             b="1", cols=4096, pad=0, residual=True),
        # the widest rows of a long prompt or a large training batch, a scale for every 128 columns
        dict(name="norm 16384x8192 fp8/128", op="norm", direction="forward", dtype="bf16", out="fp8", block=128,
             b="16384", cols=8192, pad=0, residual=True),
        # fp32 rows of an odd count and width inside a wider tensor, no residual, 8-bit whole numbers
        dict(name="norm 1531x2050 f32 int8", op="norm", direction="forward", dtype="f32", out="int8", block=0,
             b="1531", cols=2050, pad=6, residual=False),
        # the backward pass at the width, batch and 16-worker split of the wide dense benchmark
        dict(name="norm grad 4096x4096 K16", op="norm", direction="backward", dtype="bf16", out="same", block=0,
             b="637,547,469,402,345,296,254,218,187,160,137,118,101,87,74,64", cols=4096, pad=0, residual=True),
        # the backward pass in fp32 at odd sizes, one of seven workers idle
        dict(name="norm grad 1531x777 f32 K7", op="norm", direction="backward", dtype="f32", out="same", block=0,
             b="600,399,266,0,133,90,43", cols=777, pad=5, residual=False),
        # sixteen sequences that write their next token, 8 of 64 experts each: latency
        dict(name="route 16 tokens of 64", op="route", direction="forward", dtype="bf16", b="16", top_k=8,
             experts=64, cols=2048, pad=0, residual=True, dropped=0.0),
        # a large training batch over 8 workers, 8 of 128 experts, some choices cut off by a capacity: the
        # largest case of the sorting
        dict(name="route 16384x2048 8 of 128", op="route", direction="forward", dtype="bf16",
             b="3300,1600,3300,800,1600,3300,800,1684", top_k=8, experts=128, cols=2048, pad=0, residual=True,
             dropped=0.02),
        # the gradients of a batch with few wide experts
        dict(name="route grad 8192x4096 2 of 8", op="route", direction="backward", dtype="bf16",
             b="4096,2048,1024,1024", top_k=2, experts=8, cols=4096, pad=0, residual=True, dropped=0.0),
        # gradients in fp32 at sizes that fit no vector access, many choices dropped (some tokens lose all)
        dict(name="route grad 1531x1001 3 of 11", op="route", direction="backward", dtype="f32",
             b="600,399,266,0,133,90,43", top_k=3, experts=11, cols=1001, pad=3, residual=False, dropped=0.2),
        # the small fp32 model of odd widths with its seven workers: few and tiny tensors
        dict(name="adamw 785-301-97-10 K7", op="adamw", dims="785,301,97,10", repeat=1, state="f32", grads="f32",
             copy=False, b="401,203,99,0,50,25,7"),
        # the wide dense benchmark model and its 16 workers' gradients
        dict(name="adamw 4096-4096-4096-4096-1000 K16", op="adamw", dims="4096,4096,4096,4096,1000", repeat=1,
             state="f32", grads="f32", copy=True,
             b="637,547,469,402,345,296,254,218,187,160,137,118,101,87,74,64"),
        # 235 million parameters in 20 tensors, gradients already averaged, 8-bit states: the largest step
        dict(name="adamw 235M 8-bit states", op="adamw", dims="4096,14336,4096", repeat=2, state="8bit", grads="bf16",
             copy=True, b="4096"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _split(rng, total, K):
    cut = [0] + sorted(rng.randint(0, total) for _ in range(K - 1)) + [total]
    return ",".join(str(cut[k + 1] - cut[k]) for k in range(K))


def draw(rng):
    most = {op: max(work(c)["bytes"] for c in listed() if c["op"] == op) for op in ("norm", "route", "adamw")}
    while True:
        op = rng.choice(["norm", "norm", "route", "route", "adamw"])
        workers = rng.choice([1, rng.randint(2, 8), rng.randint(2, 32)])
        direction = rng.choice(["forward", "backward"])
        tokens = _log_int(rng, 1, 16384)
        if op == "adamw":
            dims = [_log_int(rng, 16, 8192) for _ in range(rng.randint(2, 5))]
            c = dict(op=op, dims=",".join(map(str, dims)), repeat=rng.choice([1, 1, rng.randint(2, 24)]),
                     state=rng.choice(["f32", "8bit"]), grads=rng.choice(["f32", "bf16"]),
                     copy=rng.random() < 0.5, b=_split(rng, 4096, workers))
        else:
            cols = _log_int(rng, 64, 8192)
            if rng.random() < 0.6:
                cols = max(64, cols // 64 * 64)
            c = dict(op=op, direction=direction, dtype=rng.choice(["bf16", "bf16", "f32"]), b=_split(rng, tokens, workers),
                     cols=cols, pad=rng.choice([0, 0, 8, rng.randint(1, 31)]), residual=rng.random() < 0.7)
            if op == "norm":
                c["out"] = "same" if direction == "backward" else rng.choice(["same", "fp8", "fp8", "int8"])
                c["block"] = rng.choice([0, 32, 128]) if c["out"] in ("fp8", "int8") else 0
            else:
                c["top_k"] = rng.randint(1, 8)
                c["experts"] = max(c["top_k"], _log_int(rng, 4, 256))
                c["dropped"] = rng.choice([0.0, 0.02, 0.2])
        if work(c)["bytes"] <= most[op]:
            return c


# ---- what a program has in hand ---------------------------------------------------------------

def _workers(case):
    return [int(v) for v in case["b"].split(",")]


def _tensors(case):
    """(elements, weight decay) of each tensor: weight, bias and gain of every dense layer."""
    d = [int(v) for v in case["dims"].split(",")]
    one = []
    for n_in, n_out in zip(d, d[1:]):
        one += [(n_in * n_out, DECAY), (n_out, 0.0), (n_in, 0.0)]
    return one * int(case["repeat"])


def _layout(case):
    """First element of each tensor in the flat vectors (multiples of 256), and their length."""
    at, first = 0, []
    for n, _ in _tensors(case):
        first.append(at)
        at += (n + 255) // 256 * 256
    return first, at


def _rows(g, rows, cols, pad, dtype, scale=1.0):
    """[rows][cols] inside rows of cols + pad elements."""
    t = torch.empty(rows, cols + pad, device=DEV, dtype=dtype)
    t.copy_(torch.randn(rows, cols + pad, generator=g, device=DEV).mul_(scale))
    return t[:, :cols]


def _new(rows, cols, dtype):
    return torch.empty(rows, cols, device=DEV, dtype=dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s = dict(case=case, b=_workers(case))
    if case["op"] == "adamw":
        return _prepare_adamw(case, s, g, seed)
    T, H, dt, pad = sum(s["b"]), case["cols"], TYPES[case["dtype"]], case["pad"]
    if case["op"] == "norm":
        return _prepare_norm(case, s, g, T, H, dt, pad)
    return _prepare_route(case, s, g, T, H, dt, pad)


def _prepare_norm(case, s, g, T, H, dt, pad):
    # hidden states have a few columns that are much larger than the others
    wide = 1.0 + 20.0 * (torch.rand(H, generator=g, device=DEV) < 0.004)
    s["gain"] = 1.0 + 0.1 * torch.randn(H, generator=g, device=DEV)
    if case["direction"] == "forward":
        s["x"] = _rows(g, T, H, pad, dt)
        s["residual"] = _rows(g, T, H, pad, dt, 2.0).mul_(wide) if case["residual"] else None
    else:
        s["sum"] = _rows(g, T, H, pad, dt, 2.0).mul_(wide)
        s["rstd"] = (s["sum"].float().square().mean(1) + EPS).rsqrt()
        s["dy"] = _rows(g, T, H, pad, dt, 1e-2)
        s["dsum"] = _rows(g, T, H, pad, dt, 1e-2) if case["residual"] else None
        s["worker"] = torch.repeat_interleave(torch.arange(len(s["b"]), device=DEV), torch.tensor(s["b"], device=DEV))
    if own:
        from paper_2305_12213_amd import binding
        s["desc"] = d = binding.rms_norm_desc(
            case["dtype"], H, out=case["out"], scale_block=case["block"], eps=EPS, ld_x=H + pad,
            ld_residual=H + pad, ld_sum=H if case["direction"] == "forward" else H + pad, ld_y=H,
            ld_dy=H + pad, ld_dsum=H + pad, ld_dx=H)
        if case["direction"] == "forward":
            s["sum"] = _new(T, H, dt) if case["residual"] else None
            s["y"] = _new(T, H, {"same": dt, "fp8": torch.float8_e4m3fn, "int8": torch.int8}[case["out"]])
            s["scales"] = _new(T, binding.scale_blocks(d), torch.float32) if case["out"] != "same" else None
            s["values"] = _new(T, H, torch.bfloat16) if case["out"] != "same" else None
            s["rstd"] = torch.empty(T, device=DEV)
        else:
            s["dx"] = _new(T, H, dt)
            s["dgain"] = torch.empty(len(s["b"]), H, device=DEV)
            s["bytes"] = binding.rms_norm_backward_workspace_bytes(d, s["b"])
            s["workspace"] = torch.empty(max(1, s["bytes"]), device=DEV, dtype=torch.uint8)
    return s


def _prepare_route(case, s, g, T, H, dt, pad):
    E, k = case["experts"], case["top_k"]
    # experts are not equally popular: the best k of random scores on top of a bias of each expert
    score = torch.rand(T, E, generator=g, device=DEV).log().neg_().log_().neg_()
    score += 0.7 * torch.randn(E, generator=g, device=DEV)
    s["experts"] = score.topk(k, dim=1).indices.to(torch.int32)
    s["experts"][torch.rand(T, k, generator=g, device=DEV) < case["dropped"]] = -1
    s["weights"] = torch.softmax(torch.randn(T, k, generator=g, device=DEV), 1)
    s["bounds"] = torch.tensor([sum(s["b"][:i]) for i in range(len(s["b"]))], device=DEV, dtype=torch.int32)
    s["y"] = _new(T * k, H, dt).copy_(torch.randn(T * k, H, generator=g, device=DEV))   # the experts' outputs
    if case["direction"] == "forward":
        s["x"] = _rows(g, T, H, pad, dt)
        s["residual"] = _rows(g, T, H, pad, dt, 2.0) if case["residual"] else None
    else:
        s["offsets"], s["slot"], s["source"] = _plan(s["experts"], E)
        s["dout"] = _rows(g, T, H, pad, dt, 1e-2)
        s["dexpert"] = _new(T * k, H, dt).copy_(torch.randn(T * k, H, generator=g, device=DEV).mul_(1e-2))   # gradient of the sorted rows
        s["residual"] = s["dout"] if case["residual"] else None      # what reaches x past the experts
    if own:
        from paper_2305_12213_amd import binding
        s["desc"] = d = binding.route_desc(case["dtype"], H, T, k, E, ld_tokens=H + pad, ld_sorted=H, ld_addend=H + pad,
                                           ld_out=H)
        if case["direction"] == "forward":
            ints = dict(device=DEV, dtype=torch.int32)
            s["offsets"] = torch.empty(E + 1, **ints)
            s["slot"], s["source"] = torch.empty(T, k, **ints), torch.empty(T * k, **ints)
            s["segments"] = torch.empty(E, len(s["b"]) + 1, **ints)
            s["bytes"] = binding.route_workspace_bytes(d)
            s["workspace"] = torch.empty(max(1, s["bytes"]), device=DEV, dtype=torch.uint8)
            s["sorted"], s["out"] = _new(T * k, H, dt), _new(T, H, dt)
        else:
            s["dsorted"], s["dweights"], s["dx"] = _new(T * k, H, dt), torch.empty(T, k, device=DEV), _new(T, H, dt)
    return s


def _prepare_adamw(case, s, g, seed):
    tensors, (first, P) = _tensors(case), _layout(case)
    K, dt = len(s["b"]), TYPES[case["grads"]]
    n = torch.tensor([t[0] for t in tensors], device=DEV)
    span = (n + 255) // 256 * 256
    of = lambda v: torch.repeat_interleave(v, span)  # noqa: E731  (a tensor's value at each of its elements)
    s["index"] = torch.arange(P, device=DEV) - of(torch.tensor(first, device=DEV))
    live = s["index"] < of(n)
    s["ordinal"] = of(torch.arange(len(tensors), device=DEV, dtype=torch.int32))
    s["decay"] = of(torch.tensor([t[1] for t in tensors], device=DEV))
    s["param"] = torch.randn(P, generator=g, device=DEV).mul_(0.02).mul_(live)
    # the workers' gradients; their sizes span some orders of magnitude from row to row
    size = torch.exp(torch.randn(P // 256, generator=g, device=DEV)).mul_(1e-3)
    grads = torch.empty(K, P, device=DEV, dtype=dt)
    for k in range(K):
        grads[k] = torch.randn(P, generator=g, device=DEV).view(-1, 256).mul_(size[:, None]).view(-1).mul_(live)
    s["grads"] = grads
    m = torch.randn(P, generator=g, device=DEV).view(-1, 256).mul_(0.2 * size[:, None]).view(-1).mul_(live)
    r = torch.rand(P, generator=g, device=DEV).add_(0.5).view(-1, 256).mul_(size[:, None]).view(-1).mul_(live)
    s["step"], s["seed"] = 1000, int(seed) * 7919 % (1 << 31)
    if case["state"] == "f32":
        s["m"], s["v"] = m, r.square_()
    else:
        rnd = torch.full((P,), 1 << 15, device=DEV)
        s["m"], s["scale_m"] = _encode(m, 7, rnd)
        s["v"], s["scale_v"] = _encode(r, 8, rnd)
    if own:
        from paper_2305_12213_amd import binding
        s["copy"] = torch.zeros(P, device=DEV, dtype=torch.bfloat16) if case["copy"] else None
        eight = case["state"] == "8bit"
        at = lambda t, i: None if t is None else t[i:]  # noqa: E731
        s["adamw"] = h = binding.AdamW(
            [dict(param=at(s["param"], i), copy=at(s["copy"], i), state1=at(s["m"], i), state2=at(s["v"], i),
                  scale1=at(s.get("scale_m"), i // 256), scale2=at(s.get("scale_v"), i // 256), n=c, weight_decay=w)
             for i, (c, w) in zip(first, tensors)], param="f32", grad=case["grads"], state=case["state"])
        nbytes = h.workspace_bytes()
        h.bind(torch.empty(nbytes, device=DEV, dtype=torch.uint8), nbytes)
        s["pointers"] = binding.pointers([grads[0, i:] for i in first])
        if eight:
            s["values"] = [torch.zeros(P, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
            s["value_pointers"] = [binding.pointers([v[i:] for i in first]) for v in s["values"]]
    return s


# ---- one pass -----------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return {"norm": _own_norm, "route": _own_route, "adamw": _own_adamw}[case["op"]](s, case)
    return {"norm": _plain_norm, "route": _plain_route, "adamw": _plain_adamw}[case["op"]](s, case)


def _own_norm(s, case):
    from paper_2305_12213_amd import binding
    if case["direction"] == "backward":
        binding.rms_norm_backward(s["desc"], s["b"], s["sum"], s["rstd"], s["gain"], s["dy"], s["dsum"], s["dx"], s["dgain"],
                                  case["cols"], s["workspace"], s["bytes"])
        return dict(dx=s["dx"], dgain=s["dgain"])
    T = s["y"].shape[0]
    binding.rms_norm(s["desc"], T, s["x"], s["residual"], s["gain"], s["sum"], s["y"], s["scales"], s["rstd"])
    if case["out"] == "same":
        return dict(sum=s["sum"], y=s["y"], rstd=s["rstd"])
    binding.dequantise(s["desc"], T, s["y"], s["scales"], s["values"], "bf16", case["cols"])
    return dict(sum=s["sum"], y=s["values"], scales=s["scales"], rstd=s["rstd"])


def _own_route(s, case):
    from paper_2305_12213_amd import binding
    d = s["desc"]
    if case["direction"] == "backward":
        binding.route_combine_backward(d, s["dout"], s["y"], s["offsets"], s["slot"], s["weights"], s["dsorted"], s["dweights"])
        binding.route_combine(d, s["dexpert"], s["slot"], None, s["residual"], s["dx"])
        return dict(dsorted=s["dsorted"], dweights=s["dweights"], dx=s["dx"])
    binding.route_plan(d, s["experts"], s["offsets"], s["slot"], s["source"], s["workspace"], s["bytes"])
    binding.route_segments(d, s["offsets"], s["source"], s["b"], s["segments"])
    binding.route_gather(d, s["x"], s["offsets"], s["slot"], s["sorted"])
    binding.route_combine(d, s["y"], s["slot"], s["weights"], s["residual"], s["out"])
    return {k: s[k] for k in ("offsets", "slot", "source", "segments", "sorted", "out")}


def _own_adamw(s, case):
    from paper_2305_12213_amd import binding
    s["step"] += 1
    s["adamw"].step(s["pointers"], s["b"], s["grads"].stride(0), step=s["step"], seed=s["seed"] + s["step"], **RULE)
    m, v = s["m"], s["v"]
    if case["state"] == "8bit":
        s["adamw"].read_states(s["value_pointers"][0], s["value_pointers"][1], "bf16")
        m, v = s["values"]
    return dict(param=s["param"], copy=s["copy"], m=m, v=v)


# ---- the plain forms ------------------------------------------------------------------------------

def _plain_norm(s, case):
    dt, H = TYPES[case["dtype"]], case["cols"]
    if case["direction"] == "backward":
        dy, shat = s["dy"].float(), s["sum"].float() * s["rstd"][:, None]
        gdy = dy * s["gain"]
        dx = s["rstd"][:, None] * (gdy - shat * (gdy * shat).mean(1, keepdim=True))
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        of_worker = torch.arange(len(s["b"]), device=DEV)[:, None] == s["worker"]
        return dict(dx=dx.to(dt), dgain=of_worker.float() @ (dy * shat))
    x = s["x"].float()
    if s["residual"] is not None:
        x = x + s["residual"].float()
    rstd = (x.square().mean(1) + EPS).rsqrt()
    y = x * rstd[:, None] * s["gain"]
    total = None if s["residual"] is None else x.to(dt)
    if case["out"] == "same":
        return dict(sum=total, y=y.to(dt), rstd=rstd)
    width = case["block"] or H
    n = -(-H // width)
    if n * width != H:
        y = torch.cat([y, y.new_zeros(y.shape[0], n * width - H)], 1)
    y = y.view(-1, n, width)
    scales = y.abs().amax(2) / (448.0 if case["out"] == "fp8" else 127.0)
    q = torch.where(scales[:, :, None] > 0, y / scales[:, :, None], y.new_zeros(()))
    q = q.to(torch.float8_e4m3fn).float() if case["out"] == "fp8" else q.round()
    values = (q * scales[:, :, None]).view(-1, n * width)[:, :H].to(torch.bfloat16).contiguous()
    return dict(sum=total, y=values, scales=scales, rstd=rstd)


def _plan(experts, E):
    """(offsets, slot, source) of a stable sort of the choices by expert."""
    ids = experts.reshape(-1)
    key = torch.where((ids >= 0) & (ids < E), ids, E)
    order = torch.argsort(key, stable=True)
    offsets = torch.searchsorted(key[order], torch.arange(E + 1, device=DEV, dtype=torch.int32)).to(torch.int32)
    place = torch.arange(ids.numel(), device=DEV, dtype=torch.int32)
    dropped = place >= offsets[E]
    slot = torch.empty_like(place)
    slot[order] = torch.where(dropped, -1, place)
    return offsets, slot.view(experts.shape), torch.where(dropped, -1, order).to(torch.int32)


def _pick(rows, slot):
    """rows[slot] in 32 bits, zeros where there is no slot."""
    got = rows[slot.clamp(min=0).reshape(-1)].float().view(*slot.shape, rows.shape[1])
    return torch.where((slot >= 0)[:, :, None], got, got.new_zeros(()))


def _plain_route(s, case):
    dt, k, E = TYPES[case["dtype"]], case["top_k"], case["experts"]
    if case["direction"] == "backward":
        dout, kept = s["dout"].float(), s["source"] >= 0
        token = torch.where(kept, s["source"], 0)
        w = torch.where(kept, s["weights"].reshape(-1)[token], 0.0)
        dsorted = (w[:, None] * dout[token // k]).to(dt)
        dweights = (_pick(s["y"], s["slot"]) * dout[:, None, :]).sum(2)
        dx = _pick(s["dexpert"], s["slot"]).sum(1)
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        return dict(dsorted=dsorted, dweights=dweights, dx=dx.to(dt))
    offsets, slot, source = _plan(s["experts"], E)
    kept = source >= 0
    token = torch.where(kept, source, 0) // k
    rows = torch.where(kept[:, None], s["x"][token], s["x"].new_zeros(()))
    K = len(s["b"])
    worker = torch.searchsorted(s["bounds"], token.to(torch.int32), right=True) - 1
    expert = torch.searchsorted(offsets[1:].contiguous(), torch.arange(source.numel(), device=DEV, dtype=torch.int32), right=True)
    pair = torch.where(kept, expert * K + worker, E * K)
    begins = torch.searchsorted(pair, torch.arange(E * K, device=DEV)).to(torch.int32).view(E, K)
    out = (s["weights"][:, :, None] * _pick(s["y"], slot)).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return dict(offsets=offsets, slot=slot, source=source, segments=torch.cat([begins, offsets[1:, None]], 1),
                sorted=rows, out=out.to(dt))


MASK = (1 << 32) - 1
SMALLEST = 2.0 ** -15
SMALLEST_BITS = 112 << 23


def _random(s):
    """32 random bits for every element from its index, its tensor's ordinal and the step's seed."""
    x = s["index"] * 0x9E3779B1 + s["ordinal"] * 0x7F4A7C15 + (s["seed"] + s["step"])
    x = x & MASK
    x = ((x ^ (x >> 16)) * 0x6A09E667) & MASK
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & MASK
    return x ^ (x >> 16)


def _encode(x, bits, rnd):
    """8-bit codes of x in blocks of 256 and the blocks' scales: a sign for 7-bit magnitudes, then 16 octaves of
    equal steps each, with `rnd` of 65536ths of a step added before the rounding down."""
    top, shift = (1.875, 20) if bits == 7 else (1.9375, 19)
    amax = x.abs().view(-1, 256).amax(1)
    scale = torch.where(amax < 2.0 ** -100, 0.0, amax / top)
    inv = torch.where(amax < 2.0 ** -100, 0.0, top / amax)
    t = (x.abs().view(-1, 256) * inv[:, None]).view(-1) + SMALLEST
    code = (t.view(torch.int32) - SMALLEST_BITS + (rnd << (shift - 16)).to(torch.int32)) >> shift
    code = code.clamp(max=(1 << bits) - 1)
    if bits == 7:
        code = code | ((x < 0).to(torch.int32) << 7)
    return code.to(torch.uint8), scale


def _decode(code, scale, bits):
    code = code.to(torch.int32)
    shift = 20 if bits == 7 else 19
    t = (((code & ((1 << bits) - 1)) << shift) + SMALLEST_BITS).view(torch.float32) - SMALLEST
    t = (t.view(-1, 256) * scale[:, None]).view(-1)
    return torch.where(code > 127, -t, t) if bits == 7 else t


def _plain_adamw(s, case):
    s["step"] += 1
    eight, total = case["state"] == "8bit", float(sum(s["b"]))
    lam = torch.tensor([b / total for b in s["b"]], device=DEV)
    b1, b2 = RULE["beta1"], RULE["beta2"]
    c1, c2 = 1 - b1 ** s["step"], 1 - b2 ** s["step"]
    g = (lam[:, None] * s["grads"].float()).sum(0) if len(s["b"]) > 1 else s["grads"][0].float()
    m = _decode(s["m"], s["scale_m"], 7) if eight else s["m"]
    v = _decode(s["v"], s["scale_v"], 8).square() if eight else s["v"]
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    s["param"] = s["param"] - RULE["lr"] * (s["decay"] * s["param"] + (m / c1) / ((v / c2).sqrt() + RULE["eps"]))
    copy = s["param"].to(torch.bfloat16) if case["copy"] else None
    if not eight:
        s["m"], s["v"] = m, v
        return dict(param=s["param"], copy=copy, m=m, v=v)
    rnd = _random(s)
    s["m"], s["scale_m"] = _encode(m, 7, rnd >> 16)
    s["v"], s["scale_v"] = _encode(v.sqrt(), 8, rnd & 0xFFFF)
    return dict(param=s["param"], copy=copy, m=_decode(s["m"], s["scale_m"], 7).to(torch.bfloat16),
                v=_decode(s["v"], s["scale_v"], 8).square().to(torch.bfloat16))


# ---- work and definition ----------------------------------------------------------------------------

def work(case):
    if case["op"] == "adamw":
        n, K = sum(t[0] for t in _tensors(case)), len(_workers(case))
        state = 16 if case["state"] == "f32" else 4 + 16 / 256 + 4        # (8 bits: the values come back in 16)
        each = 8 + K * TYPES[case["grads"]].itemsize + state + (2 if case["copy"] else 0)
        return {"bytes": float(each * n), "flops": float((2 * K + 14) * n)}
    T, H, size = sum(_workers(case)), case["cols"], TYPES[case["dtype"]].itemsize
    if case["op"] == "norm":
        if case["direction"] == "backward":
            rows = 3 + bool(case["residual"])
            return {"bytes": float(T * (H * size * rows + 4) + 4 * H * (1 + len(_workers(case)))), "flops": float(11 * T * H)}
        out = size if case["out"] == "same" else 2 + 1                    # (8 bits: the values come back in 16)
        rows = size * (3 if case["residual"] else 1) + out
        scales = 0 if case["out"] == "same" else 4 * -(-H // (case["block"] or H))
        return {"bytes": float(T * (H * rows + 4 + scales) + 4 * H), "flops": float(8 * T * H)}
    k, res = case["top_k"], bool(case["residual"])
    if case["direction"] == "backward":
        # (the gradient past the experts is the output's gradient, read once)
        return {"bytes": float(T * H * size * (2 + 3 * k) + 16 * T * k), "flops": float(T * H * (4 * k + 1))}
    return {"bytes": float(T * H * size * (2 + res + 2 * k) + 16 * T * k + 4 * case["experts"] * (len(_workers(case)) + 2)),
            "flops": float(2 * T * H * k)}


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return {"norm": _exact_norm, "route": _exact_route, "adamw": _exact_adamw}[case["op"]](s, case)


def _d(t):
    return None if t is None else t.to(torch.float64)


def _exact_norm(s, case):
    gain = _d(s["gain"])
    if case["direction"] == "backward":
        z, rstd, dy = _d(s["sum"]), _d(s["rstd"]), _d(s["dy"])
        H, at, dgain = z.shape[1], 0, []
        for n in s["b"]:
            dgain.append((dy[at:at + n] * z[at:at + n] * rstd[at:at + n, None]).sum(0))
            at += n
        along = (dy * z * gain).sum(1) * rstd ** 3 / H
        dx = dy * gain * rstd[:, None] - z * along[:, None]
        return dict(dx=dx if s["dsum"] is None else dx + _d(s["dsum"]), dgain=torch.stack(dgain))
    z = _d(s["x"]) if s["residual"] is None else _d(s["x"]) + _d(s["residual"])
    rstd = 1 / torch.sqrt((z * z).sum(1) / z.shape[1] + EPS)
    y = gain * z * rstd[:, None]
    total = None if s["residual"] is None else z
    if case["out"] == "same":
        return dict(sum=total, y=y, rstd=rstd)
    values, scales = torch.empty_like(y), []
    for c in range(0, y.shape[1], case["block"] or y.shape[1]):
        part = y[:, c:c + (case["block"] or y.shape[1])]
        scale = part.abs().max(1, keepdim=True).values / (448 if case["out"] == "fp8" else 127)
        units = part / scale.clamp(min=1e-300)
        if case["out"] == "fp8":      # 3 bits behind the leading one, steps of 2^-9 below 2^-6
            step = torch.exp2(torch.floor(torch.log2(units.abs().clamp(min=2.0 ** -6))) - 3)
            units = torch.round(units / step) * step
        else:
            units = torch.round(units)
        values[:, c:c + part.shape[1]] = units * scale
        scales.append(scale)
    return dict(sum=total, y=values, scales=torch.cat(scales, 1), rstd=rstd)


def _exact_route(s, case):
    k, E = case["top_k"], case["experts"]
    T, y = sum(s["b"]), _d(s["y"])
    ids = s["experts"].cpu().tolist()
    of = [[] for _ in range(E)]
    for t, row in enumerate(ids):
        for j, e in enumerate(row):
            if 0 <= e < E:
                of[e].append(t * k + j)
    source = [i for e in of for i in e]
    total, ints = len(source), dict(device=DEV, dtype=torch.int32)
    slots = [-1] * (T * k)
    for r, i in enumerate(source):
        slots[i] = r
    slot = torch.tensor(slots, device=DEV).view(T, k)
    live = torch.tensor(source, device=DEV, dtype=torch.int64)
    token, w = live // k, _d(s["weights"]).reshape(-1)[live]
    H = y.shape[1]
    if case["direction"] == "backward":
        dout = _d(s["dout"])
        dsorted = torch.zeros_like(y)
        dsorted[:total] = dout[token] * w[:, None]
        dweights = torch.zeros(T * k, device=DEV, dtype=torch.float64)
        dweights[live] = (dout[token] * y[:total]).sum(1)
        dx = torch.zeros(T, H, device=DEV, dtype=torch.float64) if s["residual"] is None else _d(s["residual"])
        dx = dx.index_add(0, token, _d(s["dexpert"])[:total])
        return dict(dsorted=dsorted, dweights=dweights.view(T, k), dx=dx)
    rows = torch.zeros(T * k, H, device=DEV, dtype=torch.float64)
    rows[:total] = _d(s["x"])[token]
    out = torch.zeros(T, H, device=DEV, dtype=torch.float64) if s["residual"] is None else _d(s["residual"])
    out = out.index_add(0, token, y[:total] * w[:, None])
    starts = [0]
    for e in of:
        starts.append(starts[-1] + len(e))
    first = [sum(s["b"][:i]) * k for i in range(len(s["b"]))]
    segments = [[starts[e] + sum(i < f for i in of[e]) for f in first] + [starts[e + 1]] for e in range(E)]
    return dict(offsets=torch.tensor(starts, **ints), slot=slot.to(torch.int32),
                source=torch.tensor(source + [-1] * (T * k - total), **ints), segments=torch.tensor(segments, **ints),
                sorted=rows, out=out)


def _exact_adamw(s, case):
    eight, step = case["state"] == "8bit", s["step"] + 1
    lam = [b / sum(s["b"]) for b in s["b"]]
    g = sum(w * _d(s["grads"][k]) for k, w in enumerate(lam))
    if eight:
        table = _values_of_codes(7)
        m = torch.cat([table, -table])[s["m"].long()].view(-1, 256) * _d(s["scale_m"])[:, None]
        r = _values_of_codes(8)[s["v"].long()].view(-1, 256) * _d(s["scale_v"])[:, None]
        m, v = m.view(-1), r.view(-1) ** 2
    else:
        m, v = _d(s["m"]), _d(s["v"])
    m += (1 - RULE["beta1"]) * (g - m)
    v += (1 - RULE["beta2"]) * (g ** 2 - v)
    p = _d(s["param"])
    hat = m / (1 - RULE["beta1"] ** step) / (torch.sqrt(v / (1 - RULE["beta2"] ** step)) + RULE["eps"])
    p = p * (1 - RULE["lr"] * _d(s["decay"])) - RULE["lr"] * hat
    del g, hat
    if eight:
        bits = _random(dict(s, step=step))
        m = _nearest_below(m, 7, (bits >> 16).double() / 65536) * torch.sign(m)
        v = _nearest_below(v.sqrt(), 8, (bits & 0xFFFF).double() / 65536) ** 2
    return dict(param=p, copy=p if case["copy"] else None, m=m, v=v)


def _values_of_codes(bits):
    """What each magnitude code stands for, in units of the block's scale."""
    code, per = torch.arange(1 << bits, device=DEV, dtype=torch.float64), 8.0 if bits == 7 else 16.0
    octave = torch.floor(code / per)
    return torch.exp2(octave - 15) * (1 + code / per - octave) - 2.0 ** -15


def _nearest_below(x, bits, u):
    """|x| as the code at or below it once u of a step has been added."""
    table, top = _values_of_codes(bits), 1.875 if bits == 7 else 1.9375
    blocks = x.abs().view(-1, 256)
    scale = blocks.max(1, keepdim=True).values / top
    t = (blocks / scale.clamp(min=1e-300)).view(-1)
    code = (torch.searchsorted(table, t, right=True) - 1).clamp(0, len(table) - 2)
    part = (t - table[code]) / (table[code + 1] - table[code])
    code = code + ((part + u) >= 1)
    return (table[code].view(-1, 256) * scale).view(-1)
