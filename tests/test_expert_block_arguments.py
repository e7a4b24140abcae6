"""What the block with routed experts refuses before the library sees an address: no GPU is needed, the library's calls
are replaced by one that says it was reached."""
import pytest

from paper_2305_12213_amd import expert_block


class Reached(Exception):
    pass


@pytest.fixture
def block(monkeypatch):
    import torch

    def reached(*args, **kw):
        raise Reached

    for name in ("rms_norm", "route_plan", "rms_norm_backward"):
        monkeypatch.setattr(expert_block.binding, name, reached)
    b = expert_block.ExpertBlock.__new__(expert_block.ExpertBlock)
    b.width, b.hidden, b.experts, b.top_k, b.classes = 48, 40, 5, 2, 7
    b.dtype, b.t, b.device, b.max_tokens, b.max_workers, b.steps = "f32", torch.float32, "cpu", 20, 2, 0
    b.place, b.param = {"gain1": (0, 48, (48,))}, torch.ones(48)
    b.size, b.pointers = 48, None

    class Optimizer:
        step = staticmethod(reached)

    b.optimizer = Optimizer()
    return b


def test_rows(block):
    import torch
    labels = torch.zeros(12, dtype=torch.int32)
    good = torch.zeros(12, 48)
    for h in (good, torch.zeros(48, 12).t(), torch.zeros(12, 60)[:, 5:53]):      # (other strides are copied)
        with pytest.raises(Reached):
            block.gradients(h, labels, [5, 7])
    for h in (good.to(torch.bfloat16), good.double(), good.to("meta"), torch.zeros(12, 47), torch.zeros(12, 49),
              torch.zeros(12 * 48), torch.zeros(12, 48, 1)):
        with pytest.raises(ValueError):
            block.gradients(h, labels, [5, 7])
    for b in ([5, 6], [13, -1], [4, 4, 4], []):
        with pytest.raises(ValueError):
            block.gradients(good, labels, b)


def test_strided_rows_are_read_where_they_are(block, monkeypatch):
    import torch
    seen = []

    def norm(desc, rows, x, *rest):
        seen.append(x)
        raise Reached

    monkeypatch.setattr(expert_block.binding, "rms_norm", norm)
    h = torch.arange(12 * 60.0).view(12, 60)[:, 5:53]
    with pytest.raises(Reached):
        block.gradients(h, torch.zeros(12, dtype=torch.int64), [12])
    assert seen[0].is_contiguous() and torch.equal(seen[0], h)


def test_labels(block):
    import torch
    h = torch.zeros(12, 48)
    for labels in (torch.zeros(11, dtype=torch.int32), torch.zeros(12), torch.zeros(12, 1, dtype=torch.int32),
                   torch.zeros(12, dtype=torch.int32, device="meta")):
        with pytest.raises(ValueError):
            block.gradients(h, labels, [12])


def test_workers_of_a_step(block):
    with pytest.raises(Reached):
        block.step([3, 4], 1e-3)
    for b in ([1, 1, 1], [1] * 64):
        with pytest.raises(ValueError):
            block.step(b, 1e-3)
