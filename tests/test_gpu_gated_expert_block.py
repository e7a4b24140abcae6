"""The block with gated experts on tokens: embedding, norm, expert sorting, gated block, dense layer and AdamW in one run,
every worker's gradient against automatic differentiation in 64 bits."""
import numpy as np
import pytest

from paper_2305_12213_amd import expert_block

pytestmark = pytest.mark.gpu


def autograd(block, tokens, labels, b):
    """Each worker's gradient of its mean loss, from torch in float64 on the CPU."""
    import torch
    out = []
    rows = [sum(b[:i]) for i in range(len(b) + 1)]
    for i, n in enumerate(b):
        P = {name: block.view(block.param, name).double().cpu().requires_grad_() for name in block.place}
        t = tokens[rows[i]:rows[i + 1]].long().cpu()
        y = labels[rows[i]:rows[i + 1]].long().cpu()
        here = (t >= 0) & (t < block.vocabulary)
        x = P["table"][torch.where(here, t, 0)] * here[:, None]
        norm = lambda v, g: v * (v.square().mean(1, keepdim=True) + expert_block.EPS).rsqrt() * g  # noqa: E731
        n1 = norm(x, P["gain1"])
        top = (n1 @ P["router"]).topk(block.top_k, dim=1)
        w = torch.softmax(top.values, 1)
        out_rows = x
        for j in range(block.top_k):
            e = top.indices[:, j]
            gate, up = (n1[:, None, :] @ P["w_gate"][e])[:, 0], (n1[:, None, :] @ P["w_up"][e])[:, 0]
            a = gate * torch.sigmoid(gate) * up
            out_rows = out_rows + w[:, j:j + 1] * (a[:, None, :] @ P["w_down"][e])[:, 0]
        logits = norm(out_rows, P["gain2"]) @ P["head"]
        if n:
            torch.nn.functional.cross_entropy(logits, y).backward()
        out.append({k: v.grad.numpy() if n else np.zeros(v.shape) for k, v in P.items()})
    return out


@pytest.mark.parametrize("width,hidden", [(48, 40), (45, 33)])
@pytest.mark.parametrize("b", [[13, 0, 30, 5], [64]])
def test_gradients_are_those_of_the_workers_losses(dynb, b, width, hidden):
    import torch
    block = expert_block.ExpertBlock(width, hidden, 5, 2, 7, sum(b), len(b), dtype="f32", state="f32", seed=3, gated=True,
                                     vocabulary=19)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(0, 19, (sum(b),), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(0, 7, (sum(b),), generator=g, device="cuda", dtype=torch.int32)
    block.gradients(tokens, labels, b)
    torch.cuda.synchronize()
    for i, want in enumerate(autograd(block, tokens, labels, b)):
        for name in block.place:
            got = block.view(block.grads[i], name).double().cpu().numpy()
            # sums of up to 64 rows and 48 columns through six products in fp32: a relative error of 1e-5 of the
            # tensor's largest element is twenty times their roundings
            assert np.abs(got - want[name]).max() <= 1e-5 * np.abs(want[name]).max(), (i, name)


def test_it_runs_on_ragged_workers(dynb):
    losses = expert_block.main(iterations=12, width=64, hidden=96, experts=6, top_k=2, classes=8, tokens=256, vocabulary=50)
    assert bool(losses.isfinite().all())


def test_tokens_outside_the_vocabulary(dynb):
    import torch
    block = expert_block.ExpertBlock(48, 40, 5, 2, 7, 20, 2, gated=True, vocabulary=9)
    labels = torch.arange(20, device="cuda") % 7
    tokens = (torch.arange(20, device="cuda") % 9).to(torch.int32)
    tokens[3], tokens[11] = -1, 9
    assert bool(block.gradients(tokens, labels, [12, 8]).isfinite().all()) and bool(block.grads.isfinite().all())
    block.step([12, 8], 1e-3)
    for bad in (tokens.long(), tokens[:, None], tokens.cpu()):
        with pytest.raises(ValueError):
            block.gradients(bad, labels, [12, 8])
    labels[4] = 7
    with pytest.raises(ValueError):
        block.gradients(tokens, labels, [12, 8])
