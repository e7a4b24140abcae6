"""Shared plumbing of the tests of the norm, the expert sorting and AdamW: device rows with a pitch and an
offset, and how far fp32 arithmetic with one rounding may be from 64 bits."""
import numpy as np

EPS = 2.0 ** -24            # half a step of fp32
STORED = {"f32": EPS, "bf16": 2.0 ** -8}


def torch_type(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}[dtype]


def device_rows(values, dtype, pad=0, offset=0, fill=float("nan")):
    """A view [rows][cols] of device memory whose rows are `pad` elements apart and whose first element is
    `offset` elements behind a fresh allocation; everything around the rows is `fill`."""
    import torch
    rows, cols = values.shape
    flat = torch.full((offset + rows * (cols + pad) + 64,), fill, device="cuda", dtype=torch.float32).to(torch_type(dtype))
    view = flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.from_numpy(np.ascontiguousarray(values)).cuda().to(torch_type(dtype)))
    return view


def empty_rows(rows, cols, dtype, pad=0, offset=0):
    """The same, all of it marked, to be written by a call; untouched() says whether only the rows were."""
    import torch
    size = torch.empty(0, dtype=torch_type(dtype)).element_size()
    flat = torch.full(((offset + rows * (cols + pad) + 64) * size,), 0x7b, device="cuda", dtype=torch.uint8)
    view = flat.view(torch_type(dtype))[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    return view


def untouched(view):
    """Whether everything around a view of empty_rows() still holds the mark."""
    import torch
    size = view.element_size()
    base = torch.empty(0, dtype=torch.uint8, device="cuda").set_(view.untyped_storage())
    marked = base == 0x7b
    inside = torch.zeros_like(marked).view(view.dtype if size > 1 else torch.int8)
    inside.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(1)
    inside = inside.view(torch.uint8).view(-1, size).any(1, keepdim=True).expand(-1, size).reshape(-1)
    return bool((marked | inside).all())


def host(t):
    return t.detach().to("cpu").double().numpy()


def assert_within(got, want, bound, what):
    """|got - want| <= bound where want is finite; the same infinities and NaN elsewhere."""
    got, want, bound = np.asarray(got, np.float64), np.asarray(want, np.float64), np.broadcast_to(bound, np.shape(want))
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), (what, "NaN elsewhere")
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), (what, "infinities")
    off = np.abs(got - want)
    bad = fine & ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), tuple(np.argwhere(bad)[0]), got[bad][0], want[bad][0], bound[bad][0])
