"""Embeddings and their gradients against plain forms in 64 bits.

A looked-up row is one product in fp32 and one rounding.  A sum of n gradients in fp32 is off by at most n * 2^-24 of the sum of
magnitudes, and a product with the scale by 2^-24 more."""
import numpy as np
import pytest

from oracle import products as op
from paper_2305_12213_amd import binding
from tests.operators_harness import EPS, STORED, assert_within, device_rows, empty_rows, host, torch_type, untouched

pytestmark = pytest.mark.gpu


def ids_of(kind, tokens, vocabulary, seed=0):
    rng = np.random.default_rng([seed, tokens, vocabulary])
    ids = rng.integers(0, vocabulary, tokens)
    if kind == "one":
        ids[:] = vocabulary - 1
    if kind == "few":
        ids = rng.integers(0, min(3, vocabulary), tokens)
    if kind == "zipf":
        ids = np.minimum((vocabulary ** rng.random(tokens)).astype(np.int64) - 1, vocabulary - 1)
    if kind == "foreign":
        ids = np.where(rng.random(tokens) < 0.4, rng.choice([-1, vocabulary, -2 ** 31, 2 ** 31 - 1], tokens), ids)
    if kind == "none":
        ids[:] = -1
    return ids.astype(np.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocabulary,cols,pad,offset", [(1, 1, 1, 0, 0), (5, 3, 64, 0, 0), (130, 1000, 77, 3, 1),
                                                             (33, 50, 1024, 8, 0), (2, 7, 8191, 1, 1)])
def test_lookup(dynb, tokens, vocabulary, cols, pad, offset, dtype):
    import torch
    ids = ids_of("foreign", tokens, vocabulary)
    table = device_rows(np.random.default_rng(1).standard_normal((vocabulary, cols)), dtype, pad, offset)
    out = empty_rows(tokens, cols, dtype, pad, offset)
    d = binding.embedding_desc(dtype, cols, vocabulary, tokens, 0.3, ld_table=cols + pad, ld_out=cols + pad)
    binding.embedding(d, torch.from_numpy(ids).cuda(), table, out)
    torch.cuda.synchronize()
    scale = float(np.float32(0.3))
    want = op.embedding(ids, host(table), scale)
    assert_within(host(out), want, (EPS + STORED[dtype]) * (1 + EPS) * np.abs(want), "rows")
    assert untouched(out)


def gradient(b, ids, dout, vocabulary, cols, pad, scale, dtype):
    import torch
    K = len(b)
    d = binding.embedding_desc(dtype, cols, vocabulary, sum(b), scale, ld_dout=cols + pad)
    g = torch.full((K, vocabulary * cols + 3), float("nan"), device="cuda")
    n = binding.embedding_backward_workspace_bytes(d, K)
    ws = torch.full((n + 64,), 0x7b, device="cuda", dtype=torch.uint8)
    binding.embedding_backward(d, b, ids, dout, g, g.stride(0), ws, n)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0x7b).all()) and bool(g[:, vocabulary * cols:].isnan().all())
    return g[:, :vocabulary * cols].view(K, vocabulary, cols)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,b,vocabulary,cols,pad", [
    ("any", [1], 1, 1, 0), ("none", [3, 4], 5, 64, 0), ("any", [0, 7, 0], 9, 40, 1), ("one", [300, 0, 500], 31, 77, 3),
    ("few", [1000, 33], 600, 128, 0), ("zipf", [700, 0, 31, 900], 2000, 136, 0), ("foreign", [64, 64, 65], 1000, 513, 2),
    ("zipf", [6000, 1, 3000], 70000, 8, 0), ("one", [5000], 3, 24, 0), ("any", [4097], 513, 16, 0), ("zipf", [200], 300, 1100, 0),
    ("any", [2] * 64, 20, 16, 0)])
def test_gradient(dynb, kind, b, vocabulary, cols, pad, dtype):
    import torch
    tokens = sum(b)
    ids = ids_of(kind, tokens, vocabulary)
    rows = np.random.default_rng(2).standard_normal((tokens, cols))
    rows[(ids < 0) | (ids >= vocabulary)] = np.nan               # (not read into any sum)
    dout, dev = device_rows(rows, dtype, pad), torch.from_numpy(ids).cuda()
    got = gradient(b, dev, dout, vocabulary, cols, pad, 0.3, dtype)
    scale, hd = float(np.float32(0.3)), np.nan_to_num(host(dout))
    want = op.embedding_gradient(b, ids, hd, vocabulary, scale)
    size = op.embedding_gradient(b, ids, np.abs(hd), vocabulary, scale)
    most = max([1] + [np.bincount(part[(part >= 0) & (part < vocabulary)], minlength=1).max()
                      for part in np.split(ids, np.cumsum(b)[:-1]) if len(part)])
    assert_within(host(got), want, (most + 2) * EPS * size, "dtable")
    assert torch.equal(got, gradient(b, dev, dout, vocabulary, cols, pad, 0.3, dtype))


def test_large_vocabulary(dynb):
    """Three passes of the sort, rows past the caches."""
    import torch
    V, H, b = 1 << 19, 72, [3000, 5001]
    ids = ids_of("zipf", sum(b), V)
    dout = torch.randn(sum(b), H, device="cuda")
    got = gradient(b, torch.from_numpy(ids).cuda(), dout, V, H, 0, 1.0, "f32")
    worker = torch.arange(2, device="cuda").repeat_interleave(torch.tensor(b, device="cuda"))
    key = worker * V + torch.from_numpy(ids).cuda().long()
    want, size = (torch.zeros(2 * V, H, device="cuda", dtype=torch.float64).index_add_(0, key, t.double())
                  for t in (dout, dout.abs()))
    most = int(torch.bincount(key).max())
    assert bool(((got.reshape(-1, H).double() - want).abs() <= (most + 2) * EPS * size).all())


def test_table_of_more_than_32_bits(dynb):
    """2^21 tokens of 1100 columns: the last rows are 2^31 elements from the first."""
    import torch
    V, H = (1 << 21) + 3, 1100
    table = torch.empty(V, H, device="cuda", dtype=torch.bfloat16)
    ids = torch.tensor([V - 1, 0, V // 2, V - 1, V, 7], device="cuda", dtype=torch.int32)
    some = ids[[0, 1, 2, 5]].long()
    table[some] = torch.randn(4, H, device="cuda").to(torch.bfloat16)
    out = torch.empty(6, H, device="cuda", dtype=torch.bfloat16)
    d = binding.embedding_desc("bf16", H, V, 6)
    binding.embedding(d, ids, table, out)
    assert torch.equal(out[[0, 1, 2, 3, 5]], table[ids[[0, 1, 2, 3, 5]].long()]) and not bool(out[4].any())
    g = torch.empty(V * H, device="cuda")
    n = binding.embedding_backward_workspace_bytes(d, 1)
    binding.embedding_backward(d, [6], ids, out, g, V * H, torch.empty(n + 16, device="cuda", dtype=torch.uint8), n)
    g = g.view(V, H)
    assert torch.equal(g[V - 1], out[0].float() + out[3].float()) and torch.equal(g[V // 2], out[2].float())
    assert int((g != 0).any(1).sum()) == 4


def test_no_tokens(dynb):
    import torch
    d = binding.embedding_desc("bf16", 16, 10, 0)
    binding.embedding(d, None, None, None)
    g = torch.full((2, 160), float("nan"), device="cuda")
    n = binding.embedding_backward_workspace_bytes(d, 2)
    binding.embedding_backward(d, [0, 0], None, None, g, 160, torch.empty(n + 16, device="cuda", dtype=torch.uint8), n)
    assert not bool(g.any()) and not bool(g.isnan().any())


def test_replays(dynb):
    import torch
    V, H, b = 500, 40, [5000, 200]
    d = binding.embedding_desc("f32", H, V, sum(b), 2.0)
    ids, dout = torch.empty(sum(b), device="cuda", dtype=torch.int32), torch.empty(sum(b), H, device="cuda")
    g, out, table = torch.empty(2, V * H, device="cuda"), torch.empty_like(dout), torch.randn(V, H, device="cuda")
    n = binding.embedding_backward_workspace_bytes(d, 2)
    ws = torch.empty(n + 16, device="cuda", dtype=torch.uint8)
    ids.zero_(), dout.zero_()

    def step():
        binding.embedding(d, ids, table, out)
        binding.embedding_backward(d, b, ids, dout, g, V * H, ws, n)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        new = torch.from_numpy(ids_of("zipf", sum(b), V, i)).cuda()
        ids.copy_(new), dout.copy_(torch.randn(sum(b), H, device="cuda", generator=torch.Generator("cuda").manual_seed(i)))
        graph.replay()
        torch.cuda.synchronize()
        a, c = g.clone(), out.clone()
        g.fill_(float("nan")), out.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert torch.equal(a, g) and torch.equal(c, out)



def test_narrow_tables_of_many_rows(dynb):
    """64 workers, 2^23 tokens of one column: 2^29 rows of gradients."""
    import torch
    K, V, T = 64, 1 << 23, 6000
    g = torch.Generator("cuda").manual_seed(5)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    ids[:4] = torch.tensor([0, V - 1, V, -1], device="cuda")
    ids[-2:] = V - 1
    dout = torch.randn(T, 1, generator=g, device="cuda")
    b = [T // K] * (K - 1)
    b.append(T - sum(b))
    d = binding.embedding_desc("f32", 1, V, T)
    out = torch.full((K * V,), float("nan"), device="cuda")
    n = binding.embedding_backward_workspace_bytes(d, K)
    binding.embedding_backward(d, b, ids, dout, out, V, torch.empty(n + 16, device="cuda", dtype=torch.uint8), n)
    worker = torch.arange(K, device="cuda").repeat_interleave(torch.tensor(b, device="cuda"))
    live = (ids >= 0) & (ids < V)
    key = (worker * V + ids.long())[live]
    want = torch.zeros(K * V, device="cuda", dtype=torch.float64).index_add_(0, key, dout[live, 0].double())
    size = torch.zeros_like(want).index_add_(0, key, dout[live, 0].double().abs())
    most = int(torch.bincount(key - key.min()).max())
    assert bool(((out.double() - want).abs() <= (most + 2) * EPS * size).all())


@pytest.mark.parametrize("dtype,tokens", [("f32", 1 << 20), ("bf16", 1 << 22), ("f32", (1 << 18) + 777)])
def test_one_id_in_a_long_batch(dynb, dtype, tokens):
    """Equal rows, whose roundings all point the same way.  A row is in a sum of 16, then in sums of 64 while more than 1024 are
    left, then in one sum of what is left with at most 63 of each shorter kind and 15 rows on either side: at most
    16 + 64 n + 2 (63 n + 15) + 1024 + 2 roundings with n levels of 64, each of 2^-24."""
    import torch
    V, H, b = 5, 24, [3, tokens - 3]
    ids = torch.full((tokens,), 3, device="cuda", dtype=torch.int32)
    ids[:40] = torch.arange(40, device="cuda") % 5
    ids[-1] = 0
    dout = torch.full((tokens, H), 1.1, device="cuda").to(torch_type(dtype)) * (1 + torch.arange(H, device="cuda") % 8 / 8).to(torch_type(dtype))
    got = gradient(b, ids, dout, V, H, 0, 1.0, dtype)
    here = ids[3:] == 3
    want = float(here.sum()) * dout[0].double()
    levels, left = 0, tokens // 16
    while left > 1024:
        levels, left = levels + 1, left // 64
    most = 16 + 64 * levels + 2 * (63 * levels + 15) + 1024 + 2
    assert bool(((got[1, 3].double() - want).abs() <= most * EPS * want).all()), float(((got[1, 3].double() - want).abs() / want).max())
    for v in (0, 1, 2, 4):
        many = float((ids[3:] == v).sum())
        assert bool(((got[1, v].double() - many * dout[0].double()).abs() <= 40 * EPS * many * dout[0].double()).all())
    assert torch.equal(got, gradient(b, ids, dout, V, H, 0, 1.0, dtype))
