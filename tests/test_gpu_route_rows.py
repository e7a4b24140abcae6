"""More tokens than the kernels of the rows have workgroups for (2^20): narrow rows, sixteen to a workgroup, and rows of a whole
workgroup.  The values are exact in bf16, the sums checked against torch's in float32."""
import pytest

from paper_2305_12213_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,cols", [((1 << 24) + 5000, 8), ((1 << 20) + 300, 1640)])
def test_more_rows_than_workgroups(dynb, tokens, cols):
    import torch
    E, n = 5, tokens
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(-1, E, (n, 1), generator=g, device="cuda", dtype=torch.int32)
    ints = dict(device="cuda", dtype=torch.int32)
    d = binding.route_desc("bf16", cols, n, 1, E)
    offsets, slot, source = torch.zeros(E + 1, **ints), torch.zeros(n, 1, **ints), torch.zeros(n, **ints)
    size = binding.route_workspace_bytes(d)
    binding.route_plan(d, ids, offsets, slot, source, torch.empty(size + 16, device="cuda", dtype=torch.uint8), size)
    order = torch.sort(torch.where(ids[:, 0] < 0, E, ids[:, 0]), stable=True).indices
    kept = int((ids >= 0).sum())
    assert int(offsets[E]) == kept and torch.equal(source[:kept].long(), order[:kept]) and bool((source[kept:] == -1).all())
    new = lambda seed: torch.empty(n, cols, device="cuda", dtype=torch.bfloat16).normal_(  # noqa: E731
        generator=torch.Generator(device="cuda").manual_seed(seed))
    x, out = new(1), torch.zeros(n, cols, device="cuda", dtype=torch.bfloat16)
    binding.route_gather(d, x, offsets, slot, out)
    step = 1 << 20 if cols < 100 else 1 << 16
    pieces = [slice(a, min(n, a + step)) for a in range(0, n, step)]

    def of_choice(rows, r):               # a matrix of sorted rows, seen from tokens r (dropped: zeros)
        s = slot[r, 0].long()
        return rows[s.clamp(min=0)] * (s >= 0)[:, None]

    for r in pieces:
        assert torch.equal(of_choice(out, r), x[r] * (ids[r] >= 0))
    assert not bool(out[kept:].any())
    w = torch.rand(n, 1, generator=g, device="cuda") + 0.5
    y = out
    binding.route_combine(d, y, slot, w, None, x)
    for r in pieces:
        assert torch.equal(x[r], (w[r] * of_choice(y, r).float()).to(torch.bfloat16))
    dout, dw = new(2), torch.full((n, 1), -7.0, device="cuda")
    dy = x.fill_(float("nan"))
    binding.route_combine_backward(d, dout, y, offsets, slot, w, dy, dw)
    for r in pieces:
        assert torch.equal(of_choice(dy, r), (w[r] * dout[r].float()).to(torch.bfloat16) * (ids[r] >= 0))
        product = dout[r].float() * of_choice(y, r).float()
        # sums of `cols` products in fp32 in two orders
        assert bool(((dw[r, 0] - product.sum(1)).abs() <= 2 * (cols / 8 + 20) * 2.0 ** -24 * product.abs().sum(1)).all())
    assert not bool(dy[kept:].any())
