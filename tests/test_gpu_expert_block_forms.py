"""Every form of the block with routed experts (gated or not, on tokens or on rows, fp32 and bf16): the workers' gradients
against automatic differentiation in 64 bits of the weights as the products read them."""
import numpy as np
import pytest

from paper_2305_12213_amd import expert_block

pytestmark = pytest.mark.gpu

EXACT = ("gain1", "router", "gain2")       # read in fp32 whatever the block's type


def autograd(block, given, labels, b):
    """Each worker's gradient of its mean loss, from torch in float64 on the CPU.  Experts are chosen from the norm's output as it
    is stored."""
    import torch
    rows = [sum(b[:i]) for i in range(len(b) + 1)]
    out = []
    for i, n in enumerate(b):
        P = {name: (block.view(block.param, name) if name in EXACT else block.weight(name)).double().cpu().requires_grad_()
             for name in block.place}
        part, y = given[rows[i]:rows[i + 1]].cpu(), labels[rows[i]:rows[i + 1]].long().cpu()
        if block.vocabulary:
            here = (part >= 0) & (part < block.vocabulary)
            x = P["table"][torch.where(here, part, 0).long()] * here[:, None]
        else:
            x = part.double()
        norm = lambda v, g: v * (v.square().mean(1, keepdim=True) + expert_block.EPS).rsqrt() * g  # noqa: E731
        n1 = norm(x, P["gain1"])
        chosen = (n1.detach().to(block.t).double() @ P["router"].detach()).topk(block.top_k, dim=1).indices
        w = torch.softmax((n1 @ P["router"]).gather(1, chosen), 1)
        rows_out = x
        for j in range(block.top_k):
            e = chosen[:, j]
            times = lambda v, name: (v[:, None, :] @ P[name][e])[:, 0]  # noqa: E731
            if block.gated:
                gate = times(n1, "w_gate")
                y_e = times(gate * torch.sigmoid(gate) * times(n1, "w_up"), "w_down")
            else:
                y_e = times(torch.relu(times(n1, "w1")), "w2")
            rows_out = rows_out + w[:, j:j + 1] * y_e
        if n:
            torch.nn.functional.cross_entropy(norm(rows_out, P["gain2"]) @ P["head"], y).backward()
        out.append({k: v.grad.numpy() if n else np.zeros(v.shape) for k, v in P.items()})
    return out


def gradients(dtype, gated, vocabulary, b):
    import torch
    block = expert_block.ExpertBlock(48, 40, 5, 2, 7, sum(b), len(b), dtype=dtype, state="f32", seed=3, gated=gated,
                                     vocabulary=vocabulary)
    g = torch.Generator(device="cuda").manual_seed(1)
    if vocabulary:
        given = torch.randint(0, vocabulary, (sum(b),), generator=g, device="cuda", dtype=torch.int32)
        given[5], given[-2] = -1, vocabulary
    else:
        given = torch.randn(sum(b), 48, generator=g, device="cuda").to(block.t)
    labels = torch.randint(0, 7, (sum(b),), generator=g, device="cuda", dtype=torch.int32)
    block.gradients(given, labels, b)
    torch.cuda.synchronize()
    for i, want in enumerate(autograd(block, given, labels, b)):
        for name in block.place:
            yield i, name, block.view(block.grads[i], name).double().cpu().numpy(), want[name]


@pytest.mark.parametrize("b", [[13, 0, 30, 5], [64]])
@pytest.mark.parametrize("gated,vocabulary", [(True, 0), (False, 19)])
def test_fp32(dynb, gated, vocabulary, b):
    """Sums of up to 64 rows and 48 columns through six products in fp32: a relative error of 1e-5 of the tensor's largest
    element is twenty times their roundings."""
    for i, name, got, want in gradients("f32", gated, vocabulary, b):
        assert np.abs(got - want).max() <= 1e-5 * np.abs(want).max(), (i, name)


@pytest.mark.parametrize("b", [[13, 0, 30, 5], [64]])
@pytest.mark.parametrize("gated,vocabulary", [(True, 0), (False, 19), (True, 19), (False, 0)])
def test_bf16(dynb, gated, vocabulary, b):
    """Sixteen tensors at most are stored in bf16 between the rows and a gradient, each off by 2^-8 of its norm at most; a
    layer passes on a relative error in the norm less than doubled: an eighth in all."""
    for i, name, got, want in gradients("bf16", gated, vocabulary, b):
        assert np.linalg.norm(got - want) <= 2 * 16 * 2.0 ** -8 * np.linalg.norm(want), (i, name)
