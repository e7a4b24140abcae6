"""Dense layers with bias, activation and residual, and their gradients, against plain forms in 64 bits, with bounds that
follow every rounding (products_harness)."""
import numpy as np
import pytest

from oracle import products as op
from paper_2305_12213_amd import binding
from tests.operators_harness import EPS, assert_within, device_rows, empty_rows, host, torch_type, untouched
from tests.products_harness import STEEPEST, act_off, slope_off, stored, summed

pytestmark = pytest.mark.gpu


def flat(values, dtype, offset):
    """A dense tensor whose first element is `offset` elements behind a fresh allocation."""
    import torch
    t = torch.full((offset + values.size + 64,), float("nan"), device="cuda").to(torch_type(dtype))
    v = t[offset:offset + values.size].view(values.shape)
    v.copy_(torch.from_numpy(values).cuda())
    return v


def room(nbytes):
    import torch
    return torch.full((nbytes + 64,), 0x7b, device="cuda", dtype=torch.uint8)


CASES = [  # rows of the workers, n_in, n_out, pad, offset
    ([1], 64, 64, 0, 0), ([1], 1, 1, 0, 0), ([2, 0, 1], 7, 5, 1, 1), ([1], 4096, 1024, 0, 0), ([16], 2048, 136, 8, 0),
    ([17, 0, 40], 264, 200, 0, 0), ([60, 1, 90], 301, 97, 3, 1), ([128], 128, 128, 0, 0), ([129, 127, 44], 136, 264, 8, 8),
    ([3, 5], 4099, 33, 0, 1), ([500, 20], 40, 513, 5, 0), ([70], 2048, 64, 0, 0),
]


def check(b, n, m, pad, offset, dtype, act, bias, residual, grad):
    import torch
    rows = sum(b)
    rng = np.random.default_rng([rows, n, m])
    x = device_rows(rng.standard_normal((rows, n)), dtype, pad, offset)
    w = flat(rng.standard_normal((n, m)) / n ** 0.5, dtype, offset)
    beta = flat(rng.standard_normal(m), "f32", offset) if bias else None
    res = device_rows(rng.standard_normal((rows, m)), dtype, pad, offset) if residual else None
    pre, out = (empty_rows(rows, m, dtype, pad, offset) for _ in range(2))
    d = binding.linear_desc(dtype, n, m, act, grad, ld_x=n + pad, ld_residual=m + pad, ld_pre=m + pad, ld_out=m + pad,
                            ld_dout=m + pad, ld_dx=n + pad)
    nbytes = binding.linear_workspace_bytes(d, rows)
    ws = room(nbytes)
    binding.linear(d, rows, x, w, beta, res, pre, out, ws, nbytes)
    torch.cuda.synchronize()
    assert untouched(pre) and untouched(out) and bool((ws[nbytes:] == 0x7b).all())
    hx, hw, hb, hr = host(x), host(w), None if beta is None else host(beta), None if res is None else host(res)
    want, want_pre = op.linear(hx, hw, hb, hr, act)
    e = summed(hx, hw) + 2 * EPS * np.abs(want_pre)
    assert_within(host(pre), want_pre, stored(dtype, want_pre, e), "pre")
    e = STEEPEST * e + act_off(act, want_pre) + EPS * np.abs(want)
    assert_within(host(out), want, stored(dtype, want, e), "out")
    # the residual's own memory for the output, nothing kept
    if residual:
        binding.linear(d, rows, x, w, beta, res, None, res, ws, nbytes)
        assert torch.equal(res, out)

    dout = device_rows(rng.standard_normal((rows, m)), dtype, pad, offset)
    K = len(b)

    def gradients(dx, dw, db):
        nbytes = binding.linear_backward_workspace_bytes(d, b)
        ws = room(nbytes)
        binding.linear_backward(d, b, x, w, pre if act != "none" else None, dout, dx, dw, n * m + 3, db, m + 1, ws, nbytes)
        torch.cuda.synchronize()
        assert bool((ws[nbytes:] == 0x7b).all())

    dx = empty_rows(rows, n, dtype, pad, offset)
    dw = torch.full((K, n * m + 3), float("nan"), device="cuda", dtype=torch_type(grad))
    db = torch.full((K, m + 1), float("nan"), device="cuda", dtype=torch_type(grad))
    gradients(dx, dw, db)
    assert untouched(dx) and bool(dw[:, n * m:].isnan().all()) and bool(db[:, m:].isnan().all())
    hd, hp = host(dout), host(pre)
    want_dx, want_dw, want_db = op.linear_gradients(b, hx, hw, hp, hd, act)
    dz = hd * op.slope(act, hp)
    edz = np.zeros_like(dz)
    fine = edz                                    # (the bias takes the sums of what has not been rounded)
    if act != "none":
        fine = np.abs(hd) * slope_off(act, hp) + EPS * np.abs(dz)
        edz = stored(dtype, dz, fine)
    assert_within(host(dx), want_dx, stored(dtype, want_dx, summed(dz, hw.T, edz)), "dx")
    ends = np.concatenate([[0], np.cumsum(b)])
    for k in range(K):
        r = slice(ends[k], ends[k + 1])
        off = summed(hx[r].T, dz[r]) + 1.01 * (np.abs(hx[r].T) @ edz[r])
        assert_within(host(dw[k, :n * m]).reshape(n, m), want_dw[k], stored(grad, want_dw[k], off), "dw %d" % k)
        off = 2 * (b[k] + 8) * EPS * np.abs(dz[r]).sum(0) + 1.01 * fine[r].sum(0)
        assert_within(host(db[k, :m]), want_db[k], stored(grad, want_db[k], off), "db %d" % k)
    # each alone gives the same
    for which in range(3):
        parts = [None, None, None]
        parts[which] = empty_rows(rows, n, dtype, pad, offset) if which == 0 else torch.full_like((dx, dw, db)[which], float("nan"))
        gradients(*parts)
        assert torch.equal(parts[which].nan_to_num(), (dx, dw, db)[which].nan_to_num())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_layers(dynb, case, dtype):
    act = ["none", "relu", "silu", "gelu"][case % 4]
    check(*CASES[case], dtype, act, case % 3 != 0, case % 2 == 0, "f32")
    check(*CASES[case], dtype, "gelu", True, True, dtype)


def test_large_tiles(dynb):
    check([1100, 0, 1900], 136, 4096, 0, 0, "bf16", "silu", True, True, "bf16")
    check([500, 200], 2048, 1600, 8, 0, "bf16", "none", True, False, "f32")


@pytest.mark.parametrize("odd", [0, 1])
def test_large_tiles_of_fp32(dynb, odd):
    """768 tiles of 128 x 128 and more: of the outputs, of the inputs' gradients, of the weights'."""
    pad = 4 - 3 * odd
    check([5000, 0, 200], 40 + odd, 2440 + odd, pad, odd, "f32", "silu", True, True, "f32")
    check([5000, 200], 2440 - odd, 40 + odd, pad, odd, "f32", "none", False, True, "f32")
    check([700, 260], 2600 - odd, 2440 + odd, pad, odd, "f32", "none", True, False, "f32")


def test_pitches_and_rows_of_more_than_32_bits(dynb):
    """Rows 2^22 elements apart (256 of them are 2^31 bytes), 600 of them: the last ones are 2^32 bytes from the first."""
    import torch
    rows, n, m, ld = 600, 72, 40, 1 << 22
    g = torch.Generator("cuda").manual_seed(2)
    wide = torch.empty(rows * ld, device="cuda", dtype=torch.bfloat16)
    x = wide.view(rows, ld)[:, :n]
    x.copy_(torch.randn(rows, n, generator=g, device="cuda"))
    near, w = x.contiguous(), torch.randn(n, m, generator=g, device="cuda").to(torch.bfloat16)
    dout = torch.randn(rows, m, generator=g, device="cuda").to(torch.bfloat16)
    found = []
    for t, pitch in ((x, ld), (near, 0)):
        d = binding.linear_desc("bf16", n, m, "none", "f32", ld_x=pitch)
        out, dw = torch.empty(rows, m, device="cuda", dtype=torch.bfloat16), torch.empty(n * m, device="cuda")
        nb = max(binding.linear_workspace_bytes(d, rows), binding.linear_backward_workspace_bytes(d, [rows]))
        binding.linear(d, rows, t, w, None, None, None, out, room(nb), nb)
        binding.linear_backward(d, [rows], t, w, None, dout, None, dw, 0, None, 0, room(nb), nb)
        torch.cuda.synchronize()
        hx, hw, hd = host(near), host(w), host(dout)
        assert_within(host(out), hx @ hw, stored("bf16", hx @ hw, summed(hx, hw)), "out")
        assert_within(host(dw).reshape(n, m), hx.T @ hd, summed(hx.T, hd) + EPS * np.abs(hx.T @ hd), "dw")


def test_pitches_of_more_than_32_bits_in_fp32(dynb):
    """Rows 2^21 + 1 elements apart (256 of them pass 2^31 bytes), 600 of them."""
    import torch
    rows, n, m, ld = 600, 72, 41, (1 << 21) + 1
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.empty(rows * ld, device="cuda").view(rows, ld)[:, :n]
    x.copy_(torch.randn(rows, n, generator=g, device="cuda"))
    w = torch.randn(n, m, generator=g, device="cuda")
    dout = torch.randn(rows, m, generator=g, device="cuda")
    d = binding.linear_desc("f32", n, m, "none", "f32", ld_x=ld)
    out, dw = torch.empty(rows, m, device="cuda"), torch.empty(n * m, device="cuda")
    nb = max(binding.linear_workspace_bytes(d, rows), binding.linear_backward_workspace_bytes(d, [rows]))
    binding.linear(d, rows, x, w, None, None, None, out, room(nb), nb)
    binding.linear_backward(d, [rows], x, w, None, dout, None, dw, 0, None, 0, room(nb), nb)
    torch.cuda.synchronize()
    hx, hw, hd = host(x.contiguous()), host(w), host(dout)
    assert_within(host(out), hx @ hw, stored("f32", hx @ hw, summed(hx, hw)), "out")
    assert_within(host(dw).reshape(n, m), hx.T @ hd, summed(hx.T, hd) + EPS * np.abs(hx.T @ hd), "dw")


def test_no_rows_and_idle_workers(dynb):
    import torch
    d = binding.linear_desc("bf16", 40, 24, "silu")
    binding.linear(d, 0, None, None, None, None, None, None, None, 0)
    dw, db = torch.full((2, 960), float("nan"), device="cuda"), torch.full((2, 24), float("nan"), device="cuda")
    n = binding.linear_backward_workspace_bytes(d, [0, 0])
    binding.linear_backward(d, [0, 0], None, None, None, None, None, dw, 960, db, 24, room(n), n)
    assert not bool(dw.isnan().any() | dw.any()) and not bool(db.isnan().any() | db.any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_extreme_pre_activations(dynb, dtype):
    """Where exponentials overflow or vanish, activations and slopes have their limits; a NaN stays one."""
    import torch
    v = torch.tensor([-3e38, -1e4, -200.0, -90.0, 90.0, 200.0, 1e4, 3e38, float("nan")], device="cuda").to(torch_type(dtype))
    x, one = v[:, None].contiguous(), torch.ones(1, 1, device="cuda", dtype=v.dtype)
    for act in ("relu", "silu", "gelu"):
        d = binding.linear_desc(dtype, 1, 1, act)
        out, pre, dx = (torch.empty(9, 1, device="cuda", dtype=v.dtype) for _ in range(3))
        binding.linear(d, 9, x, one, None, None, pre, out, room(64), binding.linear_workspace_bytes(d, 9))
        n = binding.linear_backward_workspace_bytes(d, [9])
        binding.linear_backward(d, [9], x, one, pre, torch.ones_like(x), dx, None, 0, None, 0, room(n), n)
        assert bool(out[8].isnan()) and bool((out[4:8] == x[4:8]).all()) and bool((out[:4].abs() <= 1e-35).all())
        assert bool((dx[4:8] == 1).all()) and bool((dx[:4].abs() <= 1e-35).all())


def test_replays_on_another_stream(dynb):
    import torch
    d = binding.linear_desc("bf16", 2048, 136, "gelu", "f32")
    g = torch.Generator("cuda").manual_seed(2)
    x, w = (torch.randn(s, device="cuda", generator=g).to(torch.bfloat16) for s in ((12, 2048), (2048, 136)))
    dout, bias = torch.randn(12, 136, device="cuda", generator=g).to(torch.bfloat16), torch.randn(136, device="cuda", generator=g)
    pre, out, dx = torch.empty_like(dout), torch.empty_like(dout), torch.empty_like(x)
    dw, db = torch.empty(2, 2048 * 136, device="cuda"), torch.empty(2, 136, device="cuda")
    n = max(binding.linear_workspace_bytes(d, 12), binding.linear_backward_workspace_bytes(d, [5, 7]))
    ws = room(n)

    def step():
        binding.linear(d, 12, x, w, bias, None, pre, out, ws, n)
        binding.linear_backward(d, [5, 7], x, w, pre, dout, dx, dw, 2048 * 136, db, 136, ws, n)

    step()
    want = [t.clone() for t in (pre, out, dx, dw, db)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(4):
        for t in (pre, out, dx, dw, db, ws):
            t.fill_(3)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((pre, out, dx, dw, db), want))
        step()
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_pre_activations(dynb, dtype):
    """Activations and slopes at the infinities are their limits there, so that a pre-activation which has become infinite by its
    rounding gives no NaN.  A product of zeros with an infinite bias is that bias."""
    import torch
    m, rows = 24, 40
    z = torch.zeros(m, device="cuda")
    z[::3], z[1::3] = float("inf"), float("-inf")
    t = torch_type(dtype)
    x, w = torch.zeros(rows, 16, device="cuda", dtype=t), torch.zeros(16, m, device="cuda", dtype=t)
    dout = torch.randn(rows, m, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(t)
    one = torch.eye(m, device="cuda", dtype=t)
    for act, middle in (("none", 1.0), ("relu", 0.0), ("silu", 0.5), ("gelu", 0.5)):
        d = binding.linear_desc(dtype, 16, m, act)
        out, pre, dx = (torch.empty(rows, m, device="cuda", dtype=t) for _ in range(3))
        n = binding.linear_workspace_bytes(d, rows)
        binding.linear(d, rows, x, w, z, None, pre, out, room(n), n)
        assert torch.equal(pre, z.to(t).expand(rows, m))
        want = z.clone()
        if act != "none":
            want[1::3] = 0.0
        assert torch.equal(out, want.to(t).expand(rows, m)), act
        # through a unit weight dx is dz, whose slopes are 1, 0 and the middle one (all exact)
        d = binding.linear_desc(dtype, m, m, act)
        n = binding.linear_backward_workspace_bytes(d, [rows])
        db = torch.empty(m, device="cuda")
        binding.linear_backward(d, [rows], dx, one, pre, dout, dx, None, 0, db, m, room(n), n)
        slope = torch.ones(m, device="cuda")
        if act != "none":
            slope[1::3], slope[2::3] = 0.0, middle
        assert torch.equal(dx, dout * slope.to(t)), act
        assert bool(db.isfinite().all()), act
