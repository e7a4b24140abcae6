"""What dense layers, gated blocks and embeddings refuse, before anything is launched: no GPU is needed.  The addresses are
made up and never read."""
import pytest

from paper_2305_12213_amd import binding

A = [0x10000 * (i + 1) for i in range(16)]           # multiples of 16
WS = 0x4000000
BADARG = -1
BIG = 1 << 40


def refused(call, *args, **kw):
    with pytest.raises(binding.DynbError) as e:
        call(*args, stream=0, **kw)
    assert e.value.code == BADARG and str(e.value)


def with_one(args, k, value):
    return args[:k] + [value] + args[k + 1:]


@pytest.mark.parametrize("field,value", [("dtype", 2), ("dtype", -1), ("grad_dtype", 2), ("grad_dtype", 1), ("activation", 4),
                                         ("activation", -1), ("n_in", 0), ("n_in", (1 << 20) + 1), ("n_out", -1),
                                         ("n_out", (1 << 20) + 1), ("ld_x", 63), ("ld_residual", 31), ("ld_pre", 1),
                                         ("ld_out", -32), ("ld_dout", 31), ("ld_dx", 63)])
def test_linear_descriptions(field, value):
    d = binding.linear_desc("f32", 64, 32)
    setattr(d, field, value)
    refused(binding.linear, d, 4, *A[:6], WS, BIG)
    refused(binding.linear_backward, d, [4], *A[:6], 2048, A[6], 32, WS, BIG)
    assert binding.linear_workspace_bytes(d, 4) == 0 and binding.linear_backward_workspace_bytes(d, [4]) == 0


def test_linear_arguments():
    d = binding.linear_desc("f32", 4096, 32, activation="gelu")
    need = binding.linear_workspace_bytes(d, 4)
    assert need > 0
    for rows in (-1, 1 << 31):
        refused(binding.linear, d, rows, *A[:6], WS, BIG)
    for k in range(6):
        if k not in (2, 3, 4):
            refused(binding.linear, d, 4, *with_one(A[:6], k, None), WS, BIG)
        refused(binding.linear, d, 4, *with_one(A[:6], k, A[k] + 2), WS, BIG)
    for ws, n in ((None, need), (WS, need - 1), (WS + 8, need)):
        refused(binding.linear, d, 4, *A[:6], ws, n)


def test_linear_gradient_arguments():
    d = binding.linear_desc("bf16", 64, 32, activation="silu", grad="f32")
    b = [300, 4]
    need = binding.linear_backward_workspace_bytes(d, b)
    assert need > 0
    good = A[:6] + [2048, A[6], 32]
    for bad in ([], [-1, 2], [1] * 65, [(1 << 31) - 1, 1]):
        refused(binding.linear_backward, d, bad, *good, WS, BIG)
        assert binding.linear_backward_workspace_bytes(d, bad) == 0
    for k in (0, 1, 2, 3):                        # (x and weight are read, pre belongs to the activation)
        refused(binding.linear_backward, d, b, *with_one(good, k, None), WS, BIG)
    for k in (0, 1, 2, 3, 4, 5, 7):
        refused(binding.linear_backward, d, b, *with_one(good, k, good[k] + 1), WS, BIG)
    for k, value in ((5, A[5] + 2), (7, A[6] + 2), (6, 2047), (8, 31)):
        refused(binding.linear_backward, d, b, *with_one(good, k, value), WS, BIG)
    for ws, n in ((None, need), (WS, need - 1), (WS + 8, need)):
        refused(binding.linear_backward, d, b, *good, ws, n)


@pytest.mark.parametrize("field,value", [("dtype", 2), ("grad_dtype", 1), ("activation", 4), ("cols", 0), ("cols", (1 << 20) + 1),
                                         ("hidden", 0), ("hidden", (1 << 20) + 1), ("n_experts", 0), ("n_experts", 1025),
                                         ("rows", -1), ("rows", 1 << 31), ("ld_x", 63), ("ld_y", 1), ("ld_dy", -64), ("ld_dx", 60),
                                         ("ld_kept", 31)])
def test_gated_descriptions(field, value):
    d = binding.gated_block_desc("f32", 64, 32, 4, 100)
    setattr(d, field, value)
    refused(binding.gated_block, d, *A[:8], WS, BIG)
    refused(binding.gated_block_backward, d, 1, *A[:13], BIG, WS, BIG)
    assert binding.gated_block_workspace_bytes(d) == 0 and binding.gated_block_backward_workspace_bytes(d, 1) == 0


def test_gated_arguments():
    d = binding.gated_block_desc("f32", 64, 32, 4, 100)
    need = binding.gated_block_workspace_bytes(d)
    for k in range(8):
        refused(binding.gated_block, d, *with_one(A[:8], k, None), WS, BIG)     # (one of the two kept ones included)
        refused(binding.gated_block, d, *with_one(A[:8], k, A[k] + 2), WS, BIG)
    for ws, n in ((None, need), (WS, need - 1), (WS + 8, need)):
        refused(binding.gated_block, d, *A[:8], ws, n)


def test_gated_gradient_arguments():
    d = binding.gated_block_desc("f32", 64, 32, 4, 100)
    size = 4 * 64 * 32
    need = binding.gated_block_backward_workspace_bytes(d, 2)
    for K in (0, -1, 65):
        refused(binding.gated_block_backward, d, K, *A[:13], size, WS, BIG)
        assert binding.gated_block_backward_workspace_bytes(d, K) == 0
    for k in range(13):
        if k != 9:                                # (dx may be left out)
            refused(binding.gated_block_backward, d, 2, *with_one(A[:13], k, None), size, WS, BIG)
        refused(binding.gated_block_backward, d, 2, *with_one(A[:13], k, A[k] + 2), size, WS, BIG)
    refused(binding.gated_block_backward, d, 2, *A[:13], size - 1, WS, BIG)
    for ws, n in ((None, need), (WS, need - 1), (WS + 8, need)):
        refused(binding.gated_block_backward, d, 2, *A[:13], size, ws, n)


@pytest.mark.parametrize("field,value", [("dtype", 2), ("cols", 0), ("cols", (1 << 20) + 1), ("vocabulary", 0),
                                         ("vocabulary", (1 << 24) + 1), ("tokens", -1), ("tokens", 1 << 31),
                                         ("scale", float("nan")), ("scale", float("inf")), ("ld_table", 63), ("ld_out", -1),
                                         ("ld_dout", 1)])
def test_embedding_descriptions(field, value):
    d = binding.embedding_desc("f32", 64, 100, 10)
    setattr(d, field, value)
    refused(binding.embedding, d, *A[:3])
    refused(binding.embedding_backward, d, [10], *A[:3], BIG, WS, BIG)
    assert binding.embedding_backward_workspace_bytes(d, 1) == 0


def test_embedding_arguments():
    d = binding.embedding_desc("f32", 64, 100, 10)
    need = binding.embedding_backward_workspace_bytes(d, 2)
    assert need > 0
    for K in (0, 65):
        assert binding.embedding_backward_workspace_bytes(d, K) == 0
    for k in range(3):
        for value in (None, A[k] + 2):
            refused(binding.embedding, d, *with_one(A[:3], k, value))
            refused(binding.embedding_backward, d, [4, 6], *with_one(A[:3], k, value), 6400, WS, BIG)
    for b in ([], [11], [10, -1, 1], [0] * 65):
        refused(binding.embedding_backward, d, b, *A[:3], 6400, WS, BIG)
    refused(binding.embedding_backward, d, [4, 6], *A[:3], 6399, WS, BIG)
    for ws, n in ((None, need), (WS, need - 1), (WS + 8, need)):
        refused(binding.embedding_backward, d, [4, 6], *A[:3], 6400, ws, n)


@pytest.mark.parametrize("dtype,n,activation", [("f32", 1, "none"), ("f32", 64, "none"), ("bf16", 1, "gelu"), ("bf16", 4096, "none")])
def test_backward_workspace_of_the_most_rows(dtype, n, activation):
    """About 128 chunks of rows have a sum of n each; parts of a weight's gradient are at most 16 (a row's gradient of so many
    tiles has one); what belongs to an activation is a value per element, in rows of whole granules."""
    for b in ([1 << 30], [2130000000], [2140000000], [(1 << 31) - 1], [(1 << 31) - 2, 1], [1 << 30, (1 << 30) - 1]):
        K, T, size = len(b), sum(b), 2 if dtype == "bf16" else 4
        got = binding.linear_backward_workspace_bytes(binding.linear_desc(dtype, n, n, activation=activation), b)
        kept = T * -(-n * size // 16) * 16 if activation != "none" else 0
        least, most = kept + 100 * n * 4, kept + (130 + K) * n * 4 + 16 * K * n * n * 4 + 64
        assert least <= got <= most, (b, got, least, most)


UNSUPPORTED = -2


def too_large(call, *args):
    with pytest.raises(binding.DynbError) as e:
        call(*args, stream=0)
    assert e.value.code == UNSUPPORTED and str(e.value)


def test_all_products_of_a_call_are_looked_at_before_its_first_launch():
    """A later product of more tiles than one launch holds: the call is refused as a whole (without a GPU a launch would be
    another error)."""
    d = binding.linear_desc("bf16", 64, 4, "none", "f32")           # dx by tiles of 32 rows, 2^24 of them
    too_large(binding.linear, d, 1 << 30, *A[:6], WS, BIG)
    too_large(binding.linear_backward, d, [1 << 29], A[0], A[1], None, A[2], A[3], A[4], 256, A[5], 4, WS, BIG)
    too_large(binding.linear_backward, d, [1 << 29], A[0], A[1], None, A[2], A[3], None, 0, A[5], 4, WS, BIG)
    d = binding.gated_block_desc("bf16", 4096, 64, 1, 1 << 28)      # 2^20 tiles of hidden, 2^24 of y and dx
    too_large(binding.gated_block, d, None, *A[:7], WS, BIG)
    too_large(binding.gated_block_backward, d, 1, None, None, *A[:11], BIG, WS, BIG)


def test_more_looked_up_rows_than_one_launch_holds():
    """Pieces of 8 columns: 2^31 - 256 at most."""
    for tokens, cols in (((1 << 31) - 255, 1), ((1 << 31) - 1, 8), (1 << 30, 9), (1 << 29, 25)):
        too_large(binding.embedding, binding.embedding_desc("bf16", cols, 10, tokens), *A[:3])
