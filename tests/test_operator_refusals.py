"""What the norm, the expert sorting and AdamW refuse, before anything is launched: no GPU is needed.  The addresses
are made up and never read."""
import ctypes

import pytest

from paper_2305_12213_amd import binding

A, B, D, E = 0x10000, 0x20000, 0x30000, 0x40000        # multiples of 16
BADARG, STATE = -1, -4


def refused(code, call, *args, **kw):
    with pytest.raises(binding.DynbError) as e:
        call(*args, stream=0, **kw)
    assert e.value.code == code and str(e.value)


@pytest.mark.parametrize("field,value", [("dtype", 2), ("dtype", -1), ("out", 3), ("out", -1), ("cols", 0), ("cols", -4),
                                         ("cols", (1 << 20) + 1), ("eps", -1e-6), ("eps", float("nan")), ("eps", float("inf")),
                                         ("ld_x", 63), ("ld_residual", 1), ("ld_sum", -64), ("ld_y", 60), ("ld_dy", 63),
                                         ("ld_dsum", 63), ("ld_dx", 63)])
def test_norm_descriptions(field, value):
    d = binding.rms_norm_desc("f32", 64)
    setattr(d, field, value)
    refused(BADARG, binding.rms_norm, d, 4, A, B, D, E, A)
    refused(BADARG, binding.rms_norm_backward, d, [4], A, B, D, E, None, A, None, 64, None, 0)
    assert binding.rms_norm_backward_workspace_bytes(d, [4]) == 0
    with pytest.raises(binding.DynbError):
        binding.scale_blocks(d)


def test_norm_arguments():
    d = binding.rms_norm_desc("f32", 64)
    refused(BADARG, binding.rms_norm, d, -1, A, B, D, E, A)
    refused(BADARG, binding.rms_norm, d, 1 << 31, A, B, D, E, A)
    refused(BADARG, binding.rms_norm, d, 4, None, B, D, E, A)
    refused(BADARG, binding.rms_norm, d, 4, A, B, D, E, None)
    for k in range(6):
        args = [A, B, D, E, A, None, A]
        args[k if k < 5 else 6] += 2
        refused(BADARG, binding.rms_norm, d, 4, *args)
    refused(BADARG, binding.rms_norm, binding.rms_norm_desc("bf16", 64), 4, A + 1, B, D, E, A)
    for out in ("fp8", "int8"):
        refused(BADARG, binding.rms_norm, binding.rms_norm_desc("f32", 64, out), 4, A, B, D, E, A + 1)     # no scales
        for block in (-32, 16, 33):
            refused(BADARG, binding.rms_norm, binding.rms_norm_desc("f32", 64, out, block), 4, A, B, D, E, A, B)
    assert binding.scale_blocks(binding.rms_norm_desc("f32", 100, "fp8", 32)) == 4
    assert binding.scale_blocks(binding.rms_norm_desc("f32", 100, "fp8", 4096)) == 1
    assert binding.scale_blocks(binding.rms_norm_desc("f32", 100, "int8")) == 1
    assert binding.scale_blocks(binding.rms_norm_desc("f32", 100)) == 0


def test_dequantise_arguments():
    d = binding.rms_norm_desc("f32", 64, "fp8")
    refused(BADARG, binding.dequantise, binding.rms_norm_desc("f32", 64), 4, A, B, D)
    refused(BADARG, binding.dequantise, d, -1, A, B, D)
    refused(BADARG, binding.dequantise, d, 4, None, B, D)
    refused(BADARG, binding.dequantise, d, 4, A, None, D)
    refused(BADARG, binding.dequantise, d, 4, A, B, None)
    refused(BADARG, binding.dequantise, d, 4, A, B, D + 2)
    refused(BADARG, binding.dequantise, d, 4, A, B + 1, D)
    refused(BADARG, binding.dequantise, d, 4, A, B, D, "f32", 63)


def test_norm_gradient_arguments():
    d = binding.rms_norm_desc("f32", 64)
    ws = binding.rms_norm_backward_workspace_bytes(d, [300, 4])
    good = [A, B, D, E, A, B, D, 64, 0x50000, ws]
    for b in ([], [-1, 2], [1] * 65, [(1 << 31) - 1, 1]):
        refused(BADARG, binding.rms_norm_backward, d, b, *good)
        assert binding.rms_norm_backward_workspace_bytes(d, b) == 0
    for k, bad in ((0, None), (1, None), (3, None), (5, None), (0, A + 2), (1, B + 2), (2, D + 2), (3, E + 2), (4, A + 2),
                   (5, B + 2), (6, D + 2), (7, 63)):
        args = list(good)
        args[k] = bad
        refused(BADARG, binding.rms_norm_backward, d, [300, 4], *args)
    if ws:
        refused(BADARG, binding.rms_norm_backward, d, [300, 4], *good[:8], None, ws)
        refused(BADARG, binding.rms_norm_backward, d, [300, 4], *good[:8], 0x50000, ws - 1)
        refused(BADARG, binding.rms_norm_backward, d, [300, 4], *good[:8], 0x50008, ws)


@pytest.mark.parametrize("field,value", [("dtype", 2), ("cols", 0), ("cols", (1 << 20) + 1), ("top_k", 0), ("top_k", 65),
                                         ("n_experts", 0), ("n_experts", 1025), ("tokens", -1), ("tokens", 1 << 30),
                                         ("ld_tokens", 63), ("ld_sorted", 63), ("ld_addend", 1), ("ld_out", -64)])
def test_route_descriptions(field, value):
    d = binding.route_desc("bf16", 64, 10, 2, 8)
    setattr(d, field, value)
    ws = (0x50000, 1 << 30)
    refused(BADARG, binding.route_plan, d, A, B, D, E, *ws)
    refused(BADARG, binding.route_segments, d, A, B, [10], D)
    refused(BADARG, binding.route_gather, d, A, B, D, E)
    refused(BADARG, binding.route_combine, d, A, B, D, E, A)
    refused(BADARG, binding.route_combine_backward, d, A, B, D, E, A, B, D)
    assert binding.route_workspace_bytes(d) == 0


def test_route_arguments():
    for tokens in (10, 100000):
        d = binding.route_desc("bf16", 64, tokens, 2, 8)
        ws = binding.route_workspace_bytes(d)
        calls = [(binding.route_plan, [A, B, D, E], [0x50000, ws], 4, ()), (binding.route_gather, [A, B, D, E], [], 2, ()),
                 (binding.route_combine, [A, B, D, E, A], [], 2, (2, 3)),
                 (binding.route_combine_backward, [A, B, D, E, A, B, D], [], 2, ())]
        for call, args, rest, size, optional in calls:
            for k in range(len(args)):
                if k not in optional:
                    refused(BADARG, call, d, *args[:k], None, *args[k + 1:], *rest)
                refused(BADARG, call, d, *args[:k], args[k] + 1, *args[k + 1:], *rest)
        if ws:
            refused(BADARG, binding.route_plan, d, A, B, D, E, None, ws)
            refused(BADARG, binding.route_plan, d, A, B, D, E, 0x50000, ws - 1)
            refused(BADARG, binding.route_plan, d, A, B, D, E, 0x50004, ws)
        for b in ([], [tokens + 1], [tokens, -1, 1], [0] * 65):
            refused(BADARG, binding.route_segments, d, A, B, b, D)
        for k in range(3):
            args = [A, B, [tokens], D]
            args[k if k < 2 else 3] = None
            refused(BADARG, binding.route_segments, d, *args)


def tensor(**kw):
    return {**dict(param=A, state1=B, state2=D, scale1=E, scale2=A, n=100, weight_decay=0.0), **kw}


def test_adamw_descriptions():
    for kw, t in ((dict(), tensor(n=-1)), (dict(), tensor(n=1 << 41)), (dict(), tensor(param=None)), (dict(), tensor(state1=None)),
                  (dict(), tensor(state2=None)), (dict(state="8bit"), tensor(scale1=None)), (dict(state="8bit"), tensor(scale2=None)),
                  (dict(), tensor(weight_decay=-0.1)), (dict(), tensor(weight_decay=float("nan"))), (dict(), tensor(param=A + 2)),
                  (dict(), tensor(state2=D + 1)), (dict(state="8bit"), tensor(scale1=E + 2)), (dict(), tensor(copy=A + 1)),
                  (dict(param="bf16"), tensor(copy=E)), (dict(param="bf16"), tensor(param=A + 1))):
        with pytest.raises(binding.DynbError) as e:
            binding.AdamW([tensor(), t], **kw)
        assert e.value.code == BADARG
    with pytest.raises(binding.DynbError):
        binding.AdamW([])
    lib, out = binding.load(), ctypes.c_void_p()
    assert lib.dynb_adamw_create(None, ctypes.byref(out)) == BADARG
    assert lib.dynb_adamw_workspace_bytes(None) == 0
    lib.dynb_adamw_destroy(None)


def test_adamw_arguments():
    h = binding.AdamW([tensor(), tensor(n=0, param=None, state1=None, state2=None)])
    assert h.workspace_bytes() > 0
    refused(BADARG, h.bind, None, 1 << 20)
    refused(BADARG, h.bind, A, h.workspace_bytes() - 1)
    refused(BADARG, h.bind, A + 8, 1 << 20)
    refused(STATE, h.step, [A, None])
    refused(BADARG, h.step, [None, None])
    refused(BADARG, h.step, [A + 2, None])
    for b in ([], [0], [1, -1], [1] * 65):
        refused(BADARG, h.step, [A, None], b)
    refused(BADARG, h.step, [A, None], [1, 1], -5)
    for kw in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(step=0), dict(eps=-1.0),
               dict(eps=float("inf")), dict(lr=float("nan"))):
        refused(BADARG, h.step, [A, None], **kw)
    refused(BADARG, h.read_states, [A, A], [A, A])              # fp32 states
    with pytest.raises(ValueError):
        h.step([A])
    h = binding.AdamW([tensor()], state="8bit")
    refused(STATE, h.read_states, [A], [A])
