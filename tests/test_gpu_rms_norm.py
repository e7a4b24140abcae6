"""The root-mean-square norm, its 8-bit outputs and its gradients against 64 bits.

Bounds, fixed before the first run.  A sum of n fp32 terms in any order that adds at most n / 64 + 20 terms one
behind the other is off by at most (n / 64 + 20) * 2^-24 of the sum of magnitudes; a handful of further roundings
are counted as 16 more; a stored value is rounded once (2^-24 or 2^-8 of it)."""
import numpy as np
import pytest

from oracle import operators as oo
from paper_2305_12213_amd import binding
from tests.operators_harness import EPS, STORED, assert_within, device_rows, empty_rows, host, torch_type, untouched

pytestmark = pytest.mark.gpu
NORM_EPS = 1e-5


def chain(cols):
    return (cols / 64 + 36) * EPS


def inputs(rows, cols, seed, scale=1.0):
    rng = np.random.default_rng([seed, rows, cols])
    wide = np.where(rng.random(cols) < 0.02, 30.0, 1.0)
    return rng, (rng.standard_normal((rows, cols)) * scale * wide).astype(np.float32)


def forward(rows, cols, dtype, out, block, residual, gain, pads=(0, 0, 0, 0), offset=0, x=None, res=None, alias=None,
            stats=True):
    import torch
    rng, xs = inputs(rows, cols, 1)
    _, rs = inputs(rows, cols, 2, 2.0)
    xs, rs = (xs if x is None else x), (rs if res is None else res)
    g = (1 + 0.2 * rng.standard_normal(cols)).astype(np.float32) if gain else None
    xd = device_rows(xs, dtype, pads[0], offset)
    rd = device_rows(rs, dtype, pads[1], offset) if residual else None
    gd = torch.from_numpy(g).cuda() if gain else None
    total = empty_rows(rows, cols, dtype, pads[2], offset)
    y = empty_rows(rows, cols, dtype if out == "same" else out, pads[3], offset)
    s, rstd, want = oo.rms_norm(host(xd), host(rd) if residual else None, g, NORM_EPS)     # (before anything is written)
    before = (xd, rd, total, y)
    if alias == "in place":          # the sum where the residual (or x) was, y where x was
        total = rd if residual else xd
        y = xd if residual and out == "same" else y
        pads = (pads[0], pads[1], pads[1] if residual else pads[0], pads[0] if residual and out == "same" else pads[3])
    d = binding.rms_norm_desc(dtype, cols, out, block, NORM_EPS, cols + pads[0], cols + pads[1], cols + pads[2],
                              cols + pads[3])
    n = binding.scale_blocks(d)
    scales = torch.full((rows, max(1, n)), -7.0, device="cuda")
    rstd_d = torch.full((rows,), -7.0, device="cuda") if stats else None
    binding.rms_norm(d, rows, xd, rd, gd, total if residual or alias else None, y, scales if n else None, rstd_d)
    torch.cuda.synchronize()
    rel = chain(cols)
    if stats:
        assert_within(host(rstd_d), rstd, rel * np.abs(np.nan_to_num(rstd)), "rstd")
    if residual or alias:
        assert_within(host(total), s, STORED[dtype] * 1.01 * np.abs(np.nan_to_num(s)) + EPS * np.abs(np.nan_to_num(s)), "sum")
    mag = np.nan_to_num(np.abs(want), posinf=0)
    if out == "same":
        assert_within(host(y), want, (rel + 1.01 * STORED[dtype]) * mag, "y")
    else:
        top = oo.FP8_TOP if out == "fp8" else oo.INT8_TOP
        ws = oo.block_scales(want, top, block)
        assert n == ws.shape[1]
        assert_within(host(scales), ws, 2 * rel * np.abs(np.nan_to_num(ws)), "scales")
        per = np.repeat(ws, block or cols, axis=1)[:, :cols]
        poor = np.nan_to_num(per)
        # half a step of the 8-bit type, and the fp32 error of y and of the scale
        half = 0.5 * poor if out == "int8" else np.maximum(mag * 2.0 ** -4, poor * 2.0 ** -10)
        for kind in ("f32", "bf16"):
            v = empty_rows(rows, cols, kind, 3, 1)
            binding.dequantise(d, rows, y, scales, v, kind, cols + 3)
            torch.cuda.synchronize()
            bound = half * (1 + 1e-3) + 4 * rel * mag + STORED[kind] * 1.01 * (mag + half)
            assert_within(host(v), np.where(np.isnan(per), np.nan, want), bound, "values " + kind)
            assert untouched(v)
    for t in before[2:]:
        assert untouched(t)
    return y, scales


COLS = [1, 3, 8, 31, 32, 33, 64, 65, 100, 127, 128, 129, 255, 257, 511, 512, 513, 777, 1000, 1024, 1025, 2047, 2050, 4096,
        4097, 8192, 8200, 12289, 16384, 16385, 32769, 65536, 65537, 70001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_widths(dynb, dtype, cols):
    forward(3, cols, dtype, "same", 0, residual=cols % 2 == 0, gain=cols % 3 != 0)


@pytest.mark.parametrize("dtype,out", [("f32", "fp8"), ("f32", "int8"), ("bf16", "fp8"), ("bf16", "int8")])
@pytest.mark.parametrize("cols", [1, 8, 33, 100, 129, 512, 777, 1025, 2050, 4096, 8200, 16385, 65537])
@pytest.mark.parametrize("block", [0, 32, 96, 128, 1024])
def test_eight_bit_outputs(dynb, dtype, out, cols, block):
    forward(3, cols, dtype, out, block, residual=block != 32, gain=True)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7, 64, 130, 1031])
@pytest.mark.parametrize("cols,out,block", [(96, "same", 0), (2050, "same", 0), (768, "fp8", 0), (520, "int8", 64)])
def test_row_counts(dynb, rows, cols, out, block):
    forward(rows, cols, "bf16", out, block, residual=True, gain=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("out,block", [("same", 0), ("fp8", 128), ("int8", 0)])
@pytest.mark.parametrize("pads,offset", [((1, 2, 3, 5), 1), ((8, 16, 8, 24), 0), ((4, 7, 1, 1), 3), ((5, 0, 0, 8), 8)])
@pytest.mark.parametrize("cols", [7, 250, 1032, 5001, 20003])
def test_pitches_and_starts(dynb, dtype, out, block, pads, offset, cols):
    forward(5, cols, dtype, out, block, residual=True, gain=True, pads=pads, offset=offset)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("out,block", [("same", 0), ("fp8", 0), ("int8", 32)])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("cols", [65, 4096, 70001])
def test_in_place(dynb, dtype, out, block, residual, cols):
    forward(4, cols, dtype, out, block, residual=residual, gain=True, pads=(3, 5, 0, 0), alias="in place")


@pytest.mark.parametrize("out,block", [("same", 0), ("fp8", 0), ("fp8", 32), ("int8", 0), ("int8", 64)])
@pytest.mark.parametrize("cols", [64, 200, 4100, 66000])
def test_zeros_infinities_and_nan(dynb, out, block, cols):
    rng, x = inputs(6, cols, 3)
    res = np.zeros_like(x)
    x[0] = 0
    x[1, 5] = np.inf
    x[2, 7] = np.nan
    x[3] = 1e-20                      # (squares vanish beside eps)
    x[4, :32] = 0
    x[4, 3] = -np.inf
    res[4, 3] = np.inf                # the sum is NaN
    x[5] = 3e18                       # squares overflow beyond cols of 38: rstd 0
    forward(6, cols, "f32", out, block, residual=True, gain=False, x=x, res=res, stats=cols != 200)


@pytest.mark.parametrize("rows,cols,dtype,out,block", [(40000, 96, "bf16", "same", 0), (40000, 250, "f32", "fp8", 64),
                                                       (34000, 1001, "bf16", "int8", 0), (9000, 2050, "bf16", "fp8", 128),
                                                       (9000, 2051, "bf16", "same", 0), (6000, 5001, "bf16", "fp8", 0),
                                                       (4200, 5000, "f32", "same", 0)])
def test_calls_beyond_the_caches(dynb, rows, cols, dtype, out, block):
    """More rows than workgroups, and beyond 64 MB rows pass the caches by."""
    forward(rows, cols, dtype, out, block, residual=True, gain=True, pads=(1, 0, 3, 0))


def test_no_rows(dynb):
    d = binding.rms_norm_desc("bf16", 64)
    binding.rms_norm(d, 0, None, None, None, None, None)


# ---- gradients --------------------------------------------------------------------------------------------------

def backward(b, cols, dtype, dsum, gain, pads=(0, 0, 0, 0), offset=0, stride=0, alias=None, want_gain=True, x=None):
    import torch
    rows = sum(b)
    rng, z = inputs(rows, cols, 4, 2.0)
    z = z if x is None else x
    _, dy = inputs(rows, cols, 5, 0.01)
    _, ds = inputs(rows, cols, 6, 0.01)
    g = (1 + 0.2 * rng.standard_normal(cols)).astype(np.float32) if gain else None
    zd, dyd = device_rows(z, dtype, pads[0], offset), device_rows(dy, dtype, pads[1], offset)
    dsd = device_rows(ds, dtype, pads[2], offset) if dsum else None
    gd = torch.from_numpy(g).cuda() if gain else None
    with np.errstate(all="ignore"):
        rstd = (1 / np.sqrt((host(zd) ** 2).mean(1) + NORM_EPS)).astype(np.float32)
    rd = torch.from_numpy(rstd).cuda()
    want, wgain = oo.rms_norm_grad(host(zd), rstd, g, host(dyd), host(dsd) if dsum else None, b)
    dyh, dsh, zh = host(dyd), host(dsd) if dsum else 0.0, host(zd)
    dx = {"dy": dyd, "dsum": dsd, None: None}[alias]
    if dx is None:
        dx = empty_rows(rows, cols, dtype, pads[3], offset)
    K, stride = len(b), stride or cols
    dgain = torch.full((K, stride), -7.0, device="cuda")
    d = binding.rms_norm_desc(dtype, cols, ld_sum=cols + pads[0], ld_dy=cols + pads[1], ld_dsum=cols + pads[2],
                              ld_dx=dx.stride(0) if rows > 1 else cols + pads[3], eps=NORM_EPS)
    nbytes = binding.rms_norm_backward_workspace_bytes(d, b)
    ws = torch.full((nbytes + 16,), 0x5a, device="cuda", dtype=torch.uint8)
    binding.rms_norm_backward(d, b, zd, rd, gd, dyd, dsd, dx, dgain if want_gain else None, stride, ws, nbytes)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0x5a).all())
    gdy, shat = dyh * (1.0 if g is None else g), zh * rstd[:, None].astype(np.float64)
    size = rstd[:, None] * (np.abs(gdy) + np.abs(shat) * np.abs(gdy * shat).mean(1, keepdims=True)) + np.abs(dsh)
    with np.errstate(all="ignore"):
        assert_within(host(dx), want, np.nan_to_num(chain(cols) * size + 1.01 * STORED[dtype] * np.abs(want), posinf=0), "dx")
    if alias is None:
        assert untouched(dx)
    if want_gain:
        at = 0
        for k, n in enumerate(b):
            size = np.abs(dyh[at:at + n] * shat[at:at + n]).sum(0)
            assert_within(host(dgain)[k, :cols], wgain[k], np.nan_to_num((n + 20) * EPS * size, posinf=0), "dgain %d" % k)
            at += n
        assert bool((dgain[:, cols:] == -7.0).all())
    return dgain


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_gradient_widths(dynb, dtype, cols):
    backward([2, 0, 5, 1], cols, dtype, dsum=cols % 2 == 0, gain=cols % 3 != 0)


@pytest.mark.parametrize("b", [[1], [0, 1], [1, 0], [3, 4, 0, 9], [0, 0, 64], [200], [37, 0, 1, 513, 129], [1] * 64,
                               [2500, 1, 700]])
@pytest.mark.parametrize("cols,dtype", [(96, "bf16"), (777, "f32"), (2048, "bf16")])
def test_gradient_workers(dynb, b, cols, dtype):
    backward(b, cols, dtype, dsum=True, gain=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pads,offset", [((1, 2, 3, 5), 1), ((8, 16, 8, 24), 0), ((5, 0, 0, 8), 8)])
@pytest.mark.parametrize("cols", [7, 250, 1032, 5001, 20003])
def test_gradient_pitches_and_starts(dynb, dtype, pads, offset, cols):
    backward([4, 0, 7], cols, dtype, dsum=True, gain=True, pads=pads, offset=offset, stride=cols + 3)


@pytest.mark.parametrize("b,cols,dtype", [([30000, 0, 17, 20001], 250, "f32"), ([34000], 1001, "bf16"), ([5000, 4000], 2050, "bf16"),
                                          ([3, 6000], 5001, "bf16"), ([2500, 1700], 5000, "f32")])
def test_gradients_beyond_the_caches(dynb, b, cols, dtype):
    backward(b, cols, dtype, dsum=True, gain=True, pads=(1, 0, 3, 0))


@pytest.mark.parametrize("alias", ["dy", "dsum"])
@pytest.mark.parametrize("cols,dtype", [(65, "f32"), (2048, "bf16"), (70001, "bf16")])
def test_gradient_in_place(dynb, alias, cols, dtype):
    backward([3, 0, 6], cols, dtype, dsum=True, gain=True, pads=(1, 3, 3, 0), alias=alias)


def test_gradient_without_gain_gradient_or_rows(dynb):
    import torch
    backward([3, 2], 300, "bf16", dsum=False, gain=True, want_gain=False)
    d = binding.rms_norm_desc("f32", 40)
    out = torch.full((2, 40), 5.0, device="cuda")
    n = binding.rms_norm_backward_workspace_bytes(d, [0, 0])
    ws = torch.empty(n + 16, device="cuda", dtype=torch.uint8)
    binding.rms_norm_backward(d, [0, 0], None, None, None, None, None, None, out, 40, ws, n)
    torch.cuda.synchronize()
    assert bool((out == 0).all())


def test_gradient_of_infinities_stays_in_its_row_and_worker(dynb):
    _, z = inputs(7, 500, 7)
    z[2, 3] = np.nan
    dgain = backward([2, 2, 3], 500, "f32", dsum=True, gain=True, x=z)
    assert np.isfinite(host(dgain)[[0, 2]]).all()


def test_gradient_against_differences(dynb):
    """The two passes against each other: a central difference of the forward pass in fp32."""
    import torch
    rows, cols, b = 4, 37, [1, 3]
    rng = np.random.default_rng(8)
    x = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).cuda()
    gain = torch.from_numpy((1 + rng.standard_normal(cols) * 0.1).astype(np.float32)).cuda()
    c = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).cuda()
    d = binding.rms_norm_desc("f32", cols, eps=NORM_EPS)

    def loss(v):
        y, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
        binding.rms_norm(d, rows, v, None, gain, None, y, None, rstd)
        return float((y.double() * c.double()).sum()), rstd

    _, rstd = loss(x)
    dx, dgain = torch.empty_like(x), torch.empty(2, cols, device="cuda")
    n = binding.rms_norm_backward_workspace_bytes(d, b)
    binding.rms_norm_backward(d, b, x, rstd, gain, c, None, dx, dgain, cols, torch.empty(n + 16, device="cuda", dtype=torch.uint8), n)
    for r, j in [(0, 0), (1, 5), (2, 36), (3, 20)]:
        h = 2.0 ** -6
        up, down = x.clone(), x.clone()
        up[r, j] += h
        down[r, j] -= h
        slope = (loss(up)[0] - loss(down)[0]) / (2 * h)
        # third derivative times h^2 / 6 (values of order 1), and 37 roundings of 2^-24 over 2 h
        assert abs(slope - float(dx[r, j])) < 10 * h * h / 6 + 37 * 4 * EPS / h


def test_results_repeat(dynb):
    """Sums over workers' rows are in a fixed order: bit for bit the same on every call and on another stream."""
    import torch
    first = backward([700, 0, 301, 1024], 1000, "bf16", dsum=True, gain=True).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = backward([700, 0, 301, 1024], 1000, "bf16", dsum=True, gain=True)
    assert torch.equal(first, again)


@pytest.mark.parametrize("out,block", [("same", 0), ("fp8", 0), ("fp8", 32), ("int8", 0), ("int8", 96)])
@pytest.mark.parametrize("cols", [64, 200, 2050, 4100, 66000])
@pytest.mark.parametrize("size,gain", [(1.0, 1e38), (1e30, 1e-15), (1e-10, 1e38), (3e18, 1e-20)])
def test_extreme_rows_and_gains(dynb, out, block, cols, size, gain):
    """Results near the largest fp32 value, and factors whose products would leave the range though the result does not."""
    import torch
    rng = np.random.default_rng([8, cols])
    x = (rng.uniform(0.5, 1.5, (5, cols)) * rng.choice([-1.0, 1.0], (5, cols)) * size).astype(np.float32)
    g = (rng.uniform(0.5, 1.5, cols) * gain).astype(np.float32)
    eps = 1e-30
    _, _, want = oo.rms_norm(x.astype(np.float64), None, g, eps)
    d = binding.rms_norm_desc("f32", cols, out, block, eps)
    n = binding.scale_blocks(d)
    y = empty_rows(5, cols, "f32" if out == "same" else out)
    scales = torch.full((5, max(1, n)), -7.0, device="cuda")
    binding.rms_norm(d, 5, torch.from_numpy(x).cuda(), None, torch.from_numpy(g).cuda(), None, y, scales if n else None, None)
    rel = chain(cols)
    if out == "same":
        assert_within(host(y), want, (rel + EPS) * np.abs(want), "y")
        return
    v = empty_rows(5, cols, "f32")
    binding.dequantise(d, 5, y, scales, v, "f32")
    ws = oo.block_scales(want, oo.FP8_TOP if out == "fp8" else oo.INT8_TOP, block)
    assert_within(host(scales), ws, 2 * rel * ws, "scales")
    per = np.repeat(ws, block or cols, axis=1)[:, :cols]
    half = 0.5 * per if out == "int8" else np.maximum(np.abs(want) * 2.0 ** -4, per * 2.0 ** -10)
    assert_within(host(v), want, half * (1 + 1e-3) + 4 * rel * np.abs(want) + EPS * (np.abs(want) + half), "values")


def test_offsets_beyond_32_bits(dynb):
    """Rows whose starts are 2^30 elements apart, forward and backward: the last one lies behind 4 GiB."""
    import torch
    rows, cols, ld = 4, 520, (1 << 30) + 3
    rng, x = inputs(rows, cols, 9)
    _, dy = inputs(rows, cols, 10)
    big = torch.empty((rows - 1) * ld + cols, device="cuda", dtype=torch.bfloat16).as_strided((rows, cols), (ld, 1))
    big.copy_(torch.from_numpy(x))
    xh = host(big)
    s, rstd, want = oo.rms_norm(xh, None, None, NORM_EPS)
    y, r = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16), torch.empty(rows, device="cuda")
    d = binding.rms_norm_desc("bf16", cols, "same", 0, NORM_EPS, ld, 0, ld, 0)
    binding.rms_norm(d, rows, big, None, None, None, y, None, r)
    rel = chain(cols)
    assert_within(host(y), want, (rel + 1.01 * STORED["bf16"]) * np.abs(want), "y")
    dyd = torch.from_numpy(dy).cuda().to(torch.bfloat16)
    dx, dgain = torch.empty_like(y), torch.empty(1, cols, device="cuda")
    n = binding.rms_norm_backward_workspace_bytes(d, [rows])
    ws = torch.empty(max(1, n), device="cuda", dtype=torch.uint8)
    binding.rms_norm_backward(d, [rows], big, r, None, dyd, None, dx, dgain, cols, ws, n)
    wdx, wdg = oo.rms_norm_grad(xh, host(r), None, host(dyd), None, [rows])
    mag = np.abs(host(dyd)) + np.abs(s * rstd[:, None]) * np.abs(host(dyd) * s * rstd[:, None]).mean(1)[:, None]
    assert_within(host(dx), wdx, 4 * rel * mag * rstd[:, None] + 1.01 * STORED["bf16"] * np.abs(wdx), "dx")
    assert_within(host(dgain), wdg, 4 * rel * np.abs(host(dyd) * s * rstd[:, None]).sum(0), "dgain")


def test_graph(dynb):
    """Forward with 8-bit rows, values and both gradients recorded into a graph: every replay gives what the calls give."""
    import torch
    rows, cols, b = 70, 1300, [40, 0, 30]
    x = torch.randn(rows, cols, device="cuda").to(torch.bfloat16)
    dy, gain = torch.randn_like(x), torch.randn(cols, device="cuda")
    d, same = binding.rms_norm_desc("bf16", cols, "fp8", 0, NORM_EPS), binding.rms_norm_desc("bf16", cols, "same", 0, NORM_EPS)
    n = binding.rms_norm_backward_workspace_bytes(same, b)
    ws = torch.empty(max(1, n), device="cuda", dtype=torch.uint8)

    def buffers():
        return dict(y=torch.zeros(rows, cols, device="cuda", dtype=torch.float8_e4m3fn), v=torch.zeros_like(x),
                    scales=torch.zeros(rows, 1, device="cuda"), rstd=torch.zeros(rows, device="cuda"), dx=torch.zeros_like(x),
                    dgain=torch.zeros(3, cols, device="cuda"))

    def calls(o):
        binding.rms_norm(d, rows, x, None, gain, None, o["y"], o["scales"], o["rstd"])
        binding.dequantise(d, rows, o["y"], o["scales"], o["v"], "bf16")
        binding.rms_norm_backward(same, b, x, o["rstd"], gain, dy, None, o["dx"], o["dgain"], cols, ws, n)

    one, two = buffers(), buffers()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        calls(two)
    for _ in range(3):
        x.normal_()
        for t in two.values():
            t.zero_()
        calls(one)
        graph.replay()
        torch.cuda.synchronize()
        for name in one:
            assert torch.equal(one[name].view(torch.uint8), two[name].view(torch.uint8)), name


@pytest.mark.parametrize("dtype,out", [("f32", "int8"), ("bf16", "fp8")])
@pytest.mark.parametrize("cols,block", [(12000, 8224), (40000, 8224), (20000, 8192), (66000, 33024), (300, 160), (2051, 224),
                                        (9000, 736), (17000, 1056), (5000, 512), (5000, 544), (100, 96), (30000, 32)])
@pytest.mark.parametrize("alias", [None, "in place"])
def test_blocks_of_any_width(dynb, dtype, out, cols, block, alias):
    forward(7, cols, dtype, out, block, residual=True, gain=cols % 3 == 0, pads=(1, 0, 0, 2), alias=alias)


@pytest.mark.parametrize("b", [[9], [0, 3, 130, 0, 5], [2] * 20])
@pytest.mark.parametrize("cols,dtype", [(16390, "f32"), (18432, "bf16"), (33001, "bf16")])
def test_gradient_workers_of_wide_rows(dynb, b, cols, dtype):
    backward(b, cols, dtype, dsum=True, gain=True)


@pytest.mark.parametrize("cols,out,block", [(18001, "same", 0), (20000, "fp8", 96), (1000, "int8", 96)])
def test_more_rows_than_workgroups_at_once(dynb, cols, out, block):
    forward(1500, cols, "bf16", out, block, residual=True, gain=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 7, 8, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 480, 512])
@pytest.mark.parametrize("rows", [1, 5, 31, 33, 4099])
def test_narrow_rows(dynb, dtype, cols, rows):
    """Several rows to a wave, some of them beyond the last: forward in each output, and the gradients of ragged workers."""
    forward(rows, cols, dtype, "same", 0, residual=True, gain=True, pads=(1, 0, 2, 0))
    forward(rows, cols, dtype, "fp8", 0, residual=False, gain=True)
    forward(rows, cols, dtype, "int8", 32, residual=True, gain=False, pads=(0, 1, 0, 3))
    backward([rows // 3, 0, rows - rows // 3], cols, dtype, dsum=True, gain=True)


@pytest.mark.parametrize("cols", [40, 100, 200])
def test_extremes_of_narrow_rows_stay_in_their_row(dynb, cols):
    rng, x = inputs(40, cols, 12)
    x[3] *= 1e30                      # squares overflow
    x[4] = 0
    x[5, 2] = np.inf
    x[6, cols - 1] = np.nan
    for out, block in (("same", 0), ("fp8", 0), ("int8", 32)):
        forward(40, cols, "f32", out, block, residual=False, gain=False, x=x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [8185, 8192, 8193, 8200, 12288, 16384])
@pytest.mark.parametrize("b,alias", [([3], None), ([1, 0, 70, 5], "dy"), ([40], "dsum")])
def test_gradients_around_the_widest_one_granule_rows(dynb, dtype, cols, b, alias):
    backward(b, cols, dtype, dsum=True, gain=True, pads=(1, 2, 0, 3) if alias is None else (0, 0, 0, 0), alias=alias)
