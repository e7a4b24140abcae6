"""Tokens sorted by expert and back, and the gradients, against plain forms in 64 bits.

Whole numbers are equal.  Bounds, fixed before the first run: a weighted sum of k rows in fp32 is off by at most
(k + 2) * 2^-24 of the sum of magnitudes, a product of two rows by (cols / 64 + 20) * 2^-24 of it, and a stored
value is rounded once (2^-24 or 2^-8 of it)."""
import numpy as np
import pytest

from oracle import operators as oo
from paper_2305_12213_amd import binding
from tests.operators_harness import EPS, STORED, assert_within, device_rows, empty_rows, host, untouched

pytestmark = pytest.mark.gpu


def ids_of(tokens, k, experts, kind, seed=0):
    rng = np.random.default_rng([seed, tokens, k, experts])
    if kind == "one":
        return np.full((tokens, k), experts - 1, np.int32)
    if kind == "none":
        return np.full((tokens, k), -1, np.int32)
    ids = rng.integers(0, experts, (tokens, k)).astype(np.int32)
    if kind == "skewed":
        ids = np.minimum(ids, rng.integers(0, experts, (tokens, k))).astype(np.int32) // 3
    if kind == "holes":                        # dropped choices of all kinds, some tokens without any
        bad = np.array([-1, experts, -2 ** 31, 2 ** 31 - 1, experts + 1], np.int64).astype(np.int32)
        hit = rng.random((tokens, k)) < 0.3
        ids[hit] = rng.choice(bad, hit.sum())
        ids[rng.random(tokens) < 0.1] = -1
    return ids


def plan(tokens, k, experts, ids):
    import torch
    d = binding.route_desc("f32", 8, tokens, k, experts)
    ints = dict(device="cuda", dtype=torch.int32)
    out = [torch.full((n,), -77, **ints) for n in (experts + 1 + 3, tokens * k + 3, tokens * k + 3)]
    nbytes = binding.route_workspace_bytes(d)
    ws = torch.full((nbytes + 16,), 0x5a, device="cuda", dtype=torch.uint8)
    binding.route_plan(d, torch.from_numpy(ids).cuda(), *out, ws, nbytes)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0x5a).all())
    for t in out:
        assert t[-3:].tolist() == [-77] * 3
    return d, [t[:-3] for t in out]


def fast_plan(ids, experts):
    """oracle.route_plan for many choices: one stable sort."""
    flat = ids.reshape(-1).astype(np.int64)
    key = np.where((flat >= 0) & (flat < experts), flat, experts)
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(experts + 1))
    source = np.where(np.arange(len(flat)) < offsets[-1], order, -1)
    slot = np.full(len(flat), -1, np.int64)
    slot[order[:offsets[-1]]] = np.arange(offsets[-1])
    return offsets, slot.reshape(ids.shape), source


def test_the_sorted_plan_is_the_plain_one():
    ids = ids_of(50, 3, 7, "holes")
    for a, b in zip(fast_plan(ids, 7), oo.route_plan(ids, 7)):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("tokens", [1, 2, 63, 64, 65, 341, 1024, 1365, 2731, 5000, 16383, 40000])
@pytest.mark.parametrize("k,experts", [(1, 1), (1, 8), (2, 3), (3, 11), (8, 64), (6, 257), (8, 1024)])
@pytest.mark.parametrize("kind", ["even", "skewed", "holes"])
def test_plan(dynb, tokens, k, experts, kind):
    ids = ids_of(tokens, k, experts, kind)
    _, (offsets, slot, source) = plan(tokens, k, experts, ids)
    want = fast_plan(ids, experts)
    assert np.array_equal(offsets.cpu().numpy(), want[0])
    assert np.array_equal(source.cpu().numpy(), want[2])
    assert np.array_equal(slot.cpu().numpy().reshape(tokens, k), want[1])


@pytest.mark.parametrize("tokens,k,experts", [(1, 64, 1024), (700, 64, 5), (33, 1, 1), (9000, 4, 1000), (300000, 2, 16)])
@pytest.mark.parametrize("kind", ["one", "none", "holes"])
def test_plan_extremes(dynb, tokens, k, experts, kind):
    ids = ids_of(tokens, k, experts, kind)
    _, got = plan(tokens, k, experts, ids)
    want = fast_plan(ids, experts)
    for a, b in zip(got, (want[0], want[1].reshape(-1), want[2])):
        assert np.array_equal(a.cpu().numpy(), b)


def test_plan_without_tokens(dynb):
    import torch
    d = binding.route_desc("f32", 8, 0, 2, 5)
    offsets = torch.full((6,), -7, device="cuda", dtype=torch.int32)
    n = binding.route_workspace_bytes(d)
    binding.route_plan(d, None, offsets, None, None, torch.empty(n + 16, device="cuda", dtype=torch.uint8), n)
    torch.cuda.synchronize()
    assert offsets.tolist() == [0] * 6
    segments = torch.full((5, 3), -7, device="cuda", dtype=torch.int32)
    binding.route_segments(d, offsets, None, [0, 0], segments)
    torch.cuda.synchronize()
    assert bool((segments == 0).all())


@pytest.mark.parametrize("b", [[1], [5, 0, 3], [0, 0, 400, 7], [100] * 8, [1] * 64, [700, 0, 0, 300, 24]])
@pytest.mark.parametrize("k,experts,kind", [(1, 3, "even"), (4, 37, "holes"), (2, 256, "skewed"), (2, 5, "none")])
def test_segments(dynb, b, k, experts, kind):
    import torch
    tokens = sum(b)
    d, (offsets, _, source) = plan(tokens, k, experts, ids_of(tokens, k, experts, kind))
    segments = torch.full((experts, len(b) + 1), -7, device="cuda", dtype=torch.int32)
    binding.route_segments(d, offsets, source, b, segments)
    torch.cuda.synchronize()
    want = oo.route_segments(offsets.cpu().numpy(), source.cpu().numpy(), b, k)
    assert np.array_equal(segments.cpu().numpy(), want)


def rows_case(tokens, k, experts, cols, dtype, kind, pads=(0, 0, 0, 0), offset=0, addend=True, seed=0):
    import torch
    rng = np.random.default_rng([seed, tokens, k, cols])
    ids = ids_of(tokens, k, experts, kind)
    offsets, slot, source = fast_plan(ids, experts)
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()  # noqa: E731
    offd, slotd = ints(offsets), ints(slot)
    x = device_rows(rng.standard_normal((tokens, cols)).astype(np.float32), dtype, pads[0], offset)
    y = rng.standard_normal((tokens * k, cols)).astype(np.float32)
    y[offsets[-1]:] = np.nan                   # rows that no choice has are not read
    y = device_rows(y, dtype, pads[1], offset)
    res = device_rows(rng.standard_normal((tokens, cols)).astype(np.float32), dtype, pads[2], offset) if addend else None
    w = rng.random((tokens, k)).astype(np.float32)
    w[slot < 0] = np.nan                       # nor are the weights of dropped choices
    wd = torch.from_numpy(w).cuda()
    d = binding.route_desc(dtype, cols, tokens, k, experts, cols + pads[0], cols + pads[1], cols + pads[2], cols + pads[3])
    xh, yh, rh = host(x), host(y), host(res) if addend else None
    total = int(offsets[-1])
    # there
    out = empty_rows(tokens * k, cols, dtype, pads[1], offset)
    binding.route_gather(d, x, offd, slotd, out)
    torch.cuda.synchronize()
    flat = source[:total] // k
    want = np.zeros((tokens * k, cols))
    want[:total] = xh[flat]
    assert np.array_equal(host(out), want) and untouched(out)
    # and back
    for weights in (w, None):
        back = empty_rows(tokens, cols, dtype, pads[3], offset)
        binding.route_combine(d, y, slotd, wd if weights is not None else None, res, back)
        torch.cuda.synchronize()
        terms = np.where((slot >= 0)[:, :, None], yh[np.maximum(slot, 0)], 0.0)
        if weights is not None:
            terms = np.where((slot >= 0)[:, :, None], terms * np.nan_to_num(w)[:, :, None].astype(np.float64), 0.0)
        want = terms.sum(1) + (rh if addend else 0.0)
        size = np.abs(terms).sum(1) + (np.abs(rh) if addend else 0.0)
        assert_within(host(back), want, (k + 2) * EPS * size + 1.01 * STORED[dtype] * np.abs(want), "combine")
        assert untouched(back)
    if addend:                                 # in place
        copy = device_rows(rh.astype(np.float32), dtype, pads[3], offset)
        d2 = binding.route_desc(dtype, cols, tokens, k, experts, cols + pads[0], cols + pads[1], cols + pads[3], cols + pads[3])
        binding.route_combine(d2, y, slotd, None, copy, copy)
        torch.cuda.synchronize()
        assert np.array_equal(host(copy), host(back))
    # gradients of the way back
    dsorted = empty_rows(tokens * k, cols, dtype, pads[1], offset)
    dw = torch.full((tokens * k + 3,), -7.0, device="cuda")
    binding.route_combine_backward(d, x, y, offd, slotd, wd, dsorted, dw)
    torch.cuda.synchronize()
    want = np.zeros((tokens * k, cols))
    want[:total] = xh[flat] * w.reshape(-1)[source[:total]].astype(np.float64)[:, None]
    assert_within(host(dsorted), want, 1.01 * (STORED[dtype] + EPS) * np.abs(want), "dsorted")
    assert untouched(dsorted) and dw[-3:].tolist() == [-7.0] * 3
    prod = np.where((slot >= 0)[:, :, None], yh[np.maximum(slot, 0)] * xh[:, None, :], 0.0)
    assert_within(host(dw)[:-3].reshape(tokens, k), prod.sum(2), (cols / 64 + 20) * EPS * np.abs(prod).sum(2), "dweights")
    first = dw.clone()
    binding.route_combine_backward(d, x, y, offd, slotd, wd, y, dw)        # over the experts' outputs themselves
    torch.cuda.synchronize()
    assert torch.equal(first, dw) and np.array_equal(host(y), host(dsorted))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 7, 8, 9, 64, 100, 511, 512, 513, 1000, 1024, 2050, 4096, 4100, 8195, 20001])
def test_row_widths(dynb, dtype, cols):
    rows_case(21, 3, 5, cols, dtype, "holes", addend=cols % 2 == 0)


@pytest.mark.parametrize("tokens", [1, 2, 5, 16, 100, 701])
@pytest.mark.parametrize("k", [1, 2, 3, 4, 7, 8, 9, 13, 16, 17, 64])
def test_tokens_and_choices(dynb, tokens, k):
    rows_case(tokens, k, 70, 264, "bf16", "holes" if tokens > 2 else "even")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pads,offset", [((1, 2, 3, 5), 1), ((8, 16, 8, 24), 0), ((4, 7, 1, 1), 3)])
@pytest.mark.parametrize("cols", [7, 250, 1032, 5001])
def test_pitches_and_starts(dynb, dtype, pads, offset, cols):
    rows_case(19, 4, 6, cols, dtype, "holes", pads=pads, offset=offset)


@pytest.mark.parametrize("cols,dtype,tokens,k", [(100, "f32", 36000, 4), (201, "bf16", 58000, 2), (500, "bf16", 8000, 9),
                                                 (1001, "f32", 4500, 3), (2000, "bf16", 5600, 2), (2051, "bf16", 9000, 1)])
def test_calls_beyond_the_caches(dynb, cols, dtype, tokens, k):
    """More than 64 MB per call, where rows pass the caches by and gradients go token by token."""
    assert (1 + k) * tokens * cols * (4 if dtype == "f32" else 2) > 64e6
    rows_case(tokens, k, 37, cols, dtype, "holes", pads=(1, 0, 3, 0))


@pytest.mark.parametrize("kind", ["none", "one"])
def test_nothing_kept_and_all_to_one(dynb, kind):
    rows_case(40, 2, 9, 520, "bf16", kind)


def test_infinities_of_kept_rows_reach_their_tokens_only(dynb):
    import torch
    slot = torch.tensor([[0, 2], [1, -1]], device="cuda", dtype=torch.int32)
    y = torch.ones(4, 16, device="cuda")
    y[1] = float("inf")
    y[3] = float("nan")
    d = binding.route_desc("f32", 16, 2, 2, 3)
    out = torch.empty(2, 16, device="cuda")
    binding.route_combine(d, y, slot, torch.tensor([[0.5, 0.25], [0.0, float("nan")]], device="cuda"), None, out)
    torch.cuda.synchronize()
    assert out[0].tolist() == [0.75] * 16 and bool(out[1].isnan().all())       # (0 * infinity)


def test_offsets_beyond_32_bits(dynb):
    """Sorted rows whose bytes pass 2^32: the last rows of 2 x 130000 x 8200 bf16 elements."""
    import torch
    tokens, k, cols = 130000, 2, 8200
    ids = np.zeros((tokens, k), np.int32)
    ids[:, 1] = 1
    d = binding.route_desc("bf16", cols, tokens, k, 2)
    _, (offsets, slot, _) = plan(tokens, k, 2, ids)
    x = torch.zeros(tokens, cols, device="cuda", dtype=torch.bfloat16)
    x[:, 0] = (torch.arange(tokens, device="cuda") % 251).to(torch.bfloat16)
    x[:, -1] = x[:, 0] + 1
    out = torch.empty(tokens * k, cols, device="cuda", dtype=torch.bfloat16)
    binding.route_gather(d, x, offsets, slot, out)
    back = torch.empty_like(x)
    binding.route_combine(d, out, slot, None, None, back)
    dw = torch.empty(tokens, k, device="cuda")
    binding.route_combine_backward(d, x, out, offsets, slot, torch.ones(tokens, k, device="cuda"), out, dw)
    torch.cuda.synchronize()
    n = (torch.arange(tokens, device="cuda") % 251).float()
    for half in (0, tokens):
        assert torch.equal(out[half:half + tokens, 0].float(), n)
        assert torch.equal(out[half:half + tokens, -1], x[:, -1])
    assert torch.equal(back[:, 0], (2 * n).to(torch.bfloat16))
    want = x[:, 0].float() ** 2 + x[:, -1].float() ** 2
    assert torch.equal(dw[:, 0], want) and torch.equal(dw[:, 1], want)


def test_segments_of_almost_2_31_rows(dynb):
    """One expert with 2^31 - 1 rows: where the workers begin."""
    import torch
    n = (1 << 31) - 1
    b = [1 << 30, 7, 0, n - (1 << 30) - 7 - 1, 1]
    d = binding.route_desc("bf16", 8, n, 1, 1)
    source = torch.arange(n, device="cuda", dtype=torch.int32)
    offsets = torch.tensor([0, n], device="cuda", dtype=torch.int32)
    segments = torch.full((1, 6), -7, device="cuda", dtype=torch.int32)
    binding.route_segments(d, offsets, source, b, segments)
    torch.cuda.synchronize()
    assert segments[0].tolist() == [0] + np.cumsum(np.array(b, np.int64)).tolist()


def test_graph(dynb):
    """Plan, sorting, combination and gradients recorded into a graph: every replay gives what the calls give."""
    import torch
    tokens, k, experts, cols, b = 900, 6, 40, 260, [500, 0, 400]
    ids = torch.zeros(tokens, k, device="cuda", dtype=torch.int32)
    x, w = torch.zeros(tokens, cols, device="cuda", dtype=torch.bfloat16), torch.rand(tokens, k, device="cuda")
    d = binding.route_desc("bf16", cols, tokens, k, experts)
    n = binding.route_workspace_bytes(d)
    ws = torch.empty(max(16, n), device="cuda", dtype=torch.uint8)

    def buffers():
        ints = lambda *s: torch.full(s, -7, device="cuda", dtype=torch.int32)  # noqa: E731
        rows = lambda r: torch.zeros(r, cols, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        return dict(offsets=ints(experts + 1), slot=ints(tokens, k), source=ints(tokens * k), segments=ints(experts, 4),
                    there=rows(tokens * k), back=rows(tokens), dsorted=rows(tokens * k), dw=torch.zeros(tokens, k, device="cuda"))

    def calls(o):
        binding.route_plan(d, ids, o["offsets"], o["slot"], o["source"], ws, n)
        binding.route_segments(d, o["offsets"], o["source"], b, o["segments"])
        binding.route_gather(d, x, o["offsets"], o["slot"], o["there"])
        binding.route_combine(d, o["there"], o["slot"], w, x, o["back"])
        binding.route_combine_backward(d, o["back"], o["there"], o["offsets"], o["slot"], w, o["dsorted"], o["dw"])

    one, two = buffers(), buffers()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        calls(two)
    for i in range(3):
        x.normal_()
        ids.copy_(torch.from_numpy(ids_of(tokens, k, experts, ("even", "holes", "skewed")[i])))
        calls(one)
        graph.replay()
        torch.cuda.synchronize()
        for name in one:
            assert torch.equal(one[name].view(torch.uint8), two[name].view(torch.uint8)), name
