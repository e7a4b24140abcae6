"""More rows than the norm's workgroups take at once: what a workgroup carries from one row to the next (the rows it has asked
for, its alternating buffers in LDS) must not show.  A workgroup that takes a single row carries nothing, and results are
the same bits in any call, so the rows of one large call are compared with those of calls on pieces of them."""
import numpy as np
import pytest

from paper_2305_12213_amd import binding
from tests.operators_harness import torch_type

pytestmark = pytest.mark.gpu
MOST = 1024                        # rows that every kernel of the norm takes at once, whatever its width


def rows_of(rows, cols, dtype, seed):
    """Ordinary rows, and some whose squares overflow or vanish."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x[5::7] *= 1e25
    x[6::11] *= 1e-25
    return x.to(torch_type(dtype))


def at_once(threads, rows_of_block=1):
    return 1024 * (2048 // threads) * rows_of_block


# rows that stay in registers: lanes of a row, granules per thread, waves; then the kernel that goes over a row again:
# blocks of any width (an odd and an even number of them), of powers of two, whole rows taken block by block
FORWARD = [(64, "same", 0, at_once(256, 32)), (100, "fp8", 32, at_once(256, 16)), (250, "int8", 0, at_once(256, 8)),
           (500, "same", 0, at_once(256, 4)), (1000, "fp8", 128, at_once(256, 4)), (1300, "int8", 0, at_once(192)),
           (4096, "same", 0, at_once(512)), (8200, "same", 0, at_once(576)), (8200, "fp8", 128, at_once(704)),
           (16000, "int8", 0, at_once(1024)), (16400, "same", 0, at_once(1024)), (17000, "fp8", 128, at_once(1024)),
           (20000, "fp8", 96, at_once(1024)), (1000, "int8", 96, at_once(128)), (100, "fp8", 96, at_once(64)),
           (20000, "int8", 8224, at_once(1024)), (20000, "fp8", 10016, at_once(1024)), (9000, "fp8", 8224, at_once(1024))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols,out,block,held", FORWARD)
def test_forward(dynb, dtype, cols, out, block, held):
    import torch
    rows = held + held // 2 + 301                       # (some workgroups take two rows, some one)
    if cols <= 1000 and held < 20000:
        rows += 2 * held                                # (and more of them)
    x, res = rows_of(rows, cols, dtype, 1), rows_of(rows, cols, dtype, 2)
    gain = torch.rand(cols, device="cuda") + 0.5
    d = binding.rms_norm_desc(dtype, cols, out, block, 0.0)
    n = max(1, binding.scale_blocks(d))

    def buffers():
        return dict(s=torch.zeros_like(x), y=torch.zeros(rows, cols, device="cuda", dtype=torch_type(dtype if out == "same" else out)),
                    scales=torch.zeros(rows, n, device="cuda"), rstd=torch.zeros(rows, device="cuda"), values=torch.zeros_like(x))

    def call(o, a, b):
        binding.rms_norm(d, b - a, x[a:b], res[a:b], gain, o["s"][a:b], o["y"][a:b], o["scales"][a:b], o["rstd"][a:b])
        if out != "same":
            binding.dequantise(d, b - a, o["y"][a:b], o["scales"][a:b], o["values"][a:b], dtype)

    whole, pieces = buffers(), buffers()
    call(whole, 0, rows)
    for a in range(0, rows, MOST):
        call(pieces, a, min(rows, a + MOST))
    torch.cuda.synchronize()
    assert bool(whole["rstd"].isfinite().all()) and bool((whole["rstd"] > 0).all())
    for name in whole:
        assert torch.equal(whole[name].view(torch.uint8), pieces[name].view(torch.uint8)), name


def test_rows_beyond_a_grid_in_one_direction(dynb):
    """2^20 workgroups lie in one direction of a grid of one row each, the next rows in the other: in place, 34 GB a matrix."""
    import torch
    rows, cols = (1 << 20) + 3, 16400
    new = lambda seed: torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16).normal_(  # noqa: E731
        generator=torch.Generator(device="cuda").manual_seed(seed))
    some = [slice(0, 2), slice(rows - 6, rows)]
    d = binding.rms_norm_desc("bf16", cols)
    x, rstd = new(1), torch.zeros(rows, device="cuda")
    before = [x[r].clone() for r in some]
    binding.rms_norm(d, rows, x, None, None, None, x, None, rstd)
    for r, v in zip(some, before):
        y, q = torch.zeros_like(v), torch.zeros(len(v), device="cuda")
        binding.rms_norm(d, len(v), v, None, None, None, y, None, q)
        assert torch.equal(x[r], y) and torch.equal(rstd[r], q)
    dy = new(2)
    before = [dy[r].clone() for r in some]
    binding.rms_norm_backward(d, [rows], x, rstd, None, dy, None, dy, None, 0, None, 0)
    for r, v in zip(some, before):
        dx = torch.zeros_like(v)
        binding.rms_norm_backward(d, [len(v)], x[r], rstd[r], None, v, None, dx, None, 0, None, 0)
        assert torch.equal(dy[r], dx)


@pytest.mark.parametrize("dtype,cols", [("bf16", 16400), ("bf16", 20001), ("f32", 8200), ("f32", 16390)])
def test_gradients_of_wide_rows(dynb, dtype, cols):
    """The rows' gradients of the kernel that takes a row at a time (the gain's come from another one)."""
    import torch
    rows = at_once(1024) * 2 + 301
    x, dy, ds = (rows_of(rows, cols, dtype, seed) for seed in (3, 4, 5))
    gain = torch.rand(cols, device="cuda") + 0.5
    rstd = (x.float() * 2.0 ** -90).square().mean(1).rsqrt() * 2.0 ** -90
    rstd = torch.where(rstd.isfinite(), rstd, 1.0)
    d = binding.rms_norm_desc(dtype, cols)
    whole, pieces = torch.zeros_like(x), torch.zeros_like(x)
    for to, step in ((whole, rows), (pieces, MOST)):
        for a in range(0, rows, step):
            b = min(rows, a + step)
            binding.rms_norm_backward(d, [b - a], x[a:b], rstd[a:b], gain, dy[a:b], ds[a:b], to[a:b], None, 0, None, 0)
    torch.cuda.synchronize()
    assert bool(whole.isfinite().any(1).all())
    assert torch.equal(whole.view(torch.uint8), pieces.view(torch.uint8))
