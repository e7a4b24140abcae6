"""A residual block with routed experts and a linear classifier, trained on ragged workers: the norm, the
expert sorting and AdamW of the library as a training program uses them together, with the controller that
resizes the workers' batches.

    h -> norm -> router, sort by expert -> relu(z W1[e]) W2[e] -> weighted sum + h -> norm -> logits -> loss

The products between them are torch's, unless the experts are gated: then the experts, (silu(z Wg[e]) * (z Wu[e])) Wd[e],
and the logits are the library's, and no size of a group is read on the host.  With a vocabulary, h are rows of a table
that is trained too.

Worker k's gradient is that of the mean loss over its own b_k rows, as everywhere in this library; AdamW forms the
weighted average of Eq. 2 itself.  Run `python -m paper_2305_12213_amd.expert_block` for a few iterations on synthetic
data, `... expert_block tokens` for gated experts on tokens.
"""
from __future__ import annotations

import sys

import torch

from paper_2305_12213_amd import binding, synth

EPS = 1e-5


class ExpertBlock:
    """Parameters, gradients [K][P] and optimizer states as flat vectors, for at most `max_tokens` rows of
    `max_workers` workers.  gated: the experts' and the last layer's products are the library's; vocabulary: number of tokens
    in the table that the rows are taken from, 0 for rows as they are given."""

    gated, vocabulary = False, 0

    def __init__(self, width, hidden, experts, top_k, classes, max_tokens, max_workers, dtype="bf16",
                 state="8bit", seed=0, device="cuda", gated=False, vocabulary=0):
        self.width, self.hidden, self.experts, self.top_k, self.classes = width, hidden, experts, top_k, classes
        self.dtype, self.device, self.max_tokens, self.max_workers = dtype, device, max_tokens, max_workers
        self.t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.gated, self.vocabulary = bool(gated), int(vocabulary)
        if self.gated:
            products = dict(w_gate=(experts, width, hidden), w_up=(experts, width, hidden), w_down=(experts, hidden, width))
        else:
            products = dict(w1=(experts, width, hidden), w2=(experts, hidden, width))
        shapes = dict(gain1=(width,), router=(width, experts), **products, gain2=(width,), head=(width, classes))
        if self.vocabulary:
            shapes["table"] = (self.vocabulary, width)
        decay = dict(gain1=0.0, gain2=0.0)
        at, self.place = 0, {}
        for name, shape in shapes.items():
            n = 1
            for v in shape:
                n *= v
            self.place[name] = (at, n, shape)
            at += -(-n // 256) * 256
        self.size = at
        new = lambda *shape, **kw: torch.zeros(*shape, device=device, **kw)  # noqa: E731
        self.param, self.grads = new(at), new(max_workers, at)
        self.copy = new(at, dtype=torch.bfloat16)
        g = torch.Generator(device=device).manual_seed(seed)
        for name, (o, n, shape) in self.place.items():
            v = self.view(self.param, name)
            if len(shape) == 1:
                v.fill_(1.0)
            elif name == "table":
                v.copy_(torch.randn(shape, generator=g, device=device))
            else:
                v.copy_(torch.randn(shape, generator=g, device=device) * (2.0 / shape[-2]) ** 0.5)
        self.copy.copy_(self.param)
        eight = state == "8bit"
        kind = dict(dtype=torch.uint8) if eight else {}
        self.m, self.v = new(at, **kind), new(at, **kind)
        self.scales = [new(at // 256), new(at // 256)]
        self.optimizer = binding.AdamW(
            [dict(param=self.param[o:], copy=self.copy[o:], state1=self.m[o:], state2=self.v[o:],
                  scale1=self.scales[0][o // 256:] if eight else None,
                  scale2=self.scales[1][o // 256:] if eight else None, n=n,
                  weight_decay=decay.get(name, 0.01)) for name, (o, n, _) in self.place.items()],
            param="f32", grad="f32", state=state)
        nbytes = self.optimizer.workspace_bytes()
        self.optimizer.bind(new(nbytes, dtype=torch.uint8), nbytes)
        self.pointers = binding.pointers([self.grads[0, o:] for o, _, _ in self.place.values()])
        self.steps = 0

    def view(self, flat, name):
        o, n, shape = self.place[name]
        return flat[..., o:o + n].view(*flat.shape[:-1], *shape)

    def weight(self, name):
        """A weight as the products read it."""
        return self.view(self.param if self.dtype == "f32" else self.copy, name)

    def empty(self, *shape, dtype=None):
        return torch.empty(*shape, device=self.device, dtype=dtype or self.t)

    def _check(self, h, labels, b):
        """What the library cannot see from addresses: it reads width * T elements of the block's type."""
        device = torch.device(self.device).type
        if self.vocabulary:
            if h.dim() != 1 or h.dtype != torch.int32 or h.device.type != device:
                raise ValueError("tokens must be [rows] of int32 on %s" % device)
        elif h.dim() != 2 or h.shape[1] != self.width or h.dtype != self.t or h.device.type != device:
            raise ValueError("h must be [rows][%d] of %s on %s" % (self.width, self.t, device))
        T, K = h.shape[0], len(b)
        if T > self.max_tokens or K > self.max_workers or sum(b) != T or any(n < 0 for n in b):
            raise ValueError("more rows or workers than the block was made for, or batch sizes that are not the rows")
        if labels.shape != (T,) or labels.is_floating_point() or labels.device != h.device:
            raise ValueError("labels must be whole numbers, one per row, where the rows are")

    def gradients(self, h, labels, b):
        """Every worker's gradient into self.grads[:K]; returns the workers' mean losses (device).  h: [sum(b)][width] of
        the block's type, any strides, or with a vocabulary the tokens, [sum(b)] int32 (one outside it has a row of
        zeros); labels: [sum(b)] in [0, classes)."""
        self._check(h, labels, b)
        if self.gated and bool(((labels < 0) | (labels >= self.classes)).any()):
            raise ValueError("a label is not one of the %d classes" % self.classes)
        h = h.contiguous()
        T, H, K, k, E = h.shape[0], self.width, len(b), self.top_k, self.experts
        if self.vocabulary:
            tokens, h = h, self.empty(T, H)
            lookup = binding.embedding_desc(self.dtype, H, self.vocabulary, T)
            binding.embedding(lookup, tokens, self.weight("table"), h)
        ints = dict(dtype=torch.int32)
        norm = binding.rms_norm_desc(self.dtype, H, eps=EPS)
        route = binding.route_desc(self.dtype, H, T, k, E)
        rows = [sum(b[:i]) for i in range(K + 1)]
        # forward
        n1, rstd1 = self.empty(T, H), self.empty(T, dtype=torch.float32)
        binding.rms_norm(norm, T, h, None, self.view(self.param, "gain1"), None, n1, None, rstd1)
        top = (n1.float() @ self.view(self.param, "router")).topk(k, dim=1)
        weights, ids = torch.softmax(top.values, 1), top.indices.to(torch.int32)
        offsets, slot = self.empty(E + 1, **ints), self.empty(T, k, **ints)
        source, segments = self.empty(T * k, **ints), self.empty(E, K + 1, **ints)
        nbytes = binding.route_workspace_bytes(route)
        binding.route_plan(route, ids, offsets, slot, source, self.empty(nbytes + 16, dtype=torch.uint8), nbytes)
        binding.route_segments(route, offsets, source, b, segments)
        z, y = self.empty(T * k, H), self.empty(T * k, H)
        binding.route_gather(route, n1, offsets, slot, z)
        if self.gated:
            kept = self._gated_forward(offsets, z, y)
        else:
            strange = ((labels < 0) | (labels >= self.classes)).sum().to(torch.int32)
            cut = torch.cat([segments.flatten(), strange[None]]).tolist()   # the products below need the sizes on the host
            if cut.pop():
                raise ValueError("a label is not one of the %d classes" % self.classes)
            cut = [cut[i:i + K + 1] for i in range(0, len(cut), K + 1)]
            w1, w2, a = self.weight("w1"), self.weight("w2"), self.empty(T * k, self.hidden)
            for e in range(E):
                r = slice(cut[e][0], cut[e][K])
                a[r] = torch.relu(z[r] @ w1[e])
                y[r] = a[r] @ w2[e]
        out, n2, rstd2 = self.empty(T, H), self.empty(T, H), self.empty(T, dtype=torch.float32)
        binding.route_combine(route, y, slot, weights, h, out)
        binding.rms_norm(norm, T, out, None, self.view(self.param, "gain2"), None, n2, None, rstd2)
        logits = self._logits(n2).float()
        # the loss and its gradient, means over each worker's own rows
        p = torch.softmax(logits, 1)
        picked = torch.log_softmax(logits, 1).gather(1, labels.long()[:, None])[:, 0]
        losses = torch.stack([-picked[rows[i]:rows[i + 1]].sum() / max(1, b[i]) for i in range(K)])
        p[torch.arange(T, device=p.device), labels.long()] -= 1.0
        for i in range(K):
            p[rows[i]:rows[i + 1]] /= max(1, b[i])
        dlogits = p.to(self.t)
        # backward
        G = self.grads[:K]
        if self.gated:
            dn2 = self._head_backward(b, n2, dlogits)
        else:
            for i in range(K):
                r = slice(rows[i], rows[i + 1])
                self.view(G, "head")[i] = (n2[r].t() @ dlogits[r]).float()
            dn2 = dlogits @ self.weight("head").t()
        dout = self.empty(T, H)
        self._norm_backward(norm, b, out, rstd2, "gain2", dn2.contiguous(), None, dout)
        dy, dweights = self.empty(T * k, H), self.empty(T, k, dtype=torch.float32)
        binding.route_combine_backward(route, dout, y, offsets, slot, weights, dy, dweights)
        if self.gated:
            dz = self._gated_backward(K, offsets, segments, z, dy, kept)
        else:
            dz = torch.zeros_like(z)
            for e in range(E):
                r = slice(cut[e][0], cut[e][K])
                da = (dy[r] @ w2[e].t()) * (a[r] > 0)
                dz[r] = da @ w1[e].t()
                for i in range(K):
                    q = slice(cut[e][i], cut[e][i + 1])
                    self.view(G, "w2")[i, e] = (a[q].t() @ dy[q]).float()
                    self.view(G, "w1")[i, e] = (z[q].t() @ da[q.start - r.start:q.stop - r.start]).float()
        dtop = weights * (dweights - (weights * dweights).sum(1, keepdim=True))
        drouter = torch.zeros(T, E, device=h.device).scatter_(1, ids.long(), dtop)
        for i in range(K):
            r = slice(rows[i], rows[i + 1])
            self.view(G, "router")[i] = n1[r].float().t() @ drouter[r]
        past = (drouter @ self.view(self.param, "router").t()).to(self.t)
        dn1, dh = self.empty(T, H), self.empty(T, H)
        binding.route_combine(route, dz, slot, None, past, dn1)
        self._norm_backward(norm, b, h, rstd1, "gain1", dn1, dout, dh)
        self.input_gradient = dh
        if self.vocabulary:
            nbytes = binding.embedding_backward_workspace_bytes(lookup, K)
            binding.embedding_backward(lookup, b, tokens, dh, self._gradient("table"), self.size, *self._room(nbytes))
        return losses

    def _room(self, nbytes):
        """A workspace, and its size."""
        return self.empty(nbytes + 16, dtype=torch.uint8), nbytes

    def _gradient(self, name):
        """Worker 0's gradient of a parameter; the other workers' are self.size elements apart."""
        return self.grads[0, self.place[name][0]:]

    def _logits(self, n2):
        if not self.gated:
            return n2 @ self.weight("head")
        d = binding.linear_desc(self.dtype, self.width, self.classes)
        logits = self.empty(n2.shape[0], self.classes)
        binding.linear(d, n2.shape[0], n2, self.weight("head"), None, None, None, logits,
                       *self._room(binding.linear_workspace_bytes(d, n2.shape[0])))
        return logits

    def _head_backward(self, b, n2, dlogits):
        d, dn2 = binding.linear_desc(self.dtype, self.width, self.classes), torch.empty_like(n2)
        binding.linear_backward(d, b, n2, self.weight("head"), None, dlogits, dn2, self._gradient("head"), self.size, None, 0,
                                *self._room(binding.linear_backward_workspace_bytes(d, b)))
        return dn2

    def _gated_forward(self, offsets, z, y):
        rows = z.shape[0]
        d = binding.gated_block_desc(self.dtype, self.width, self.hidden, self.experts, rows)
        gate, up = self.empty(rows, self.hidden), self.empty(rows, self.hidden)
        binding.gated_block(d, offsets, z, self.weight("w_gate"), self.weight("w_up"), self.weight("w_down"), gate, up, y,
                            *self._room(binding.gated_block_workspace_bytes(d)))
        return d, gate, up

    def _gated_backward(self, K, offsets, segments, z, dy, kept):
        (d, gate, up), dz = kept, torch.empty_like(z)
        binding.gated_block_backward(d, K, offsets, segments, z, self.weight("w_gate"), self.weight("w_up"),
                                     self.weight("w_down"), gate, up, dy, dz, self._gradient("w_gate"),
                                     self._gradient("w_up"), self._gradient("w_down"), self.size,
                                     *self._room(binding.gated_block_backward_workspace_bytes(d, K)))
        return dz

    def _norm_backward(self, norm, b, total, rstd, gain, dy, dsum, dx):
        nbytes = binding.rms_norm_backward_workspace_bytes(norm, b)
        binding.rms_norm_backward(norm, b, total, rstd, self.view(self.param, gain), dy, dsum, dx,
                                  self.grads[0, self.place[gain][0]:], self.size,
                                  self.empty(nbytes + 16, dtype=torch.uint8), nbytes)

    def step(self, b, lr):
        """The weighted average of the workers' gradients, applied."""
        if len(b) > self.max_workers:
            raise ValueError("more workers than the block was made for")
        self.steps += 1
        self.optimizer.step(self.pointers, b, self.size, lr=lr, beta1=0.9, beta2=0.95, eps=1e-8, step=self.steps,
                            seed=self.steps)


def main(iterations=30, width=256, hidden=512, experts=8, top_k=2, classes=32, tokens=1024, vocabulary=0):
    speeds = [1.0, 0.5, 0.5, 0.25]
    b = [tokens // len(speeds)] * len(speeds)
    control = binding.Controller(b, tokens, dict(kp=1.0, deadband=0.05, b_min=1, b_max=tokens))
    block = ExpertBlock(width, hidden, experts, top_k, classes, tokens, len(speeds), gated=vocabulary > 0, vocabulary=vocabulary)
    g = torch.Generator(device="cuda").manual_seed(7)
    centres = torch.randn(classes, width, generator=g, device="cuda")
    for it in range(iterations):
        labels = torch.randint(0, classes, (tokens,), generator=g, device="cuda", dtype=torch.int32)
        if vocabulary:                   # a token's class is its number's remainder, but for one in four
            h = torch.randint(0, vocabulary, (tokens,), generator=g, device="cuda", dtype=torch.int32)
            labels = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.75, h % classes, labels)
        else:
            h = (centres[labels.long()] + 1.5 * torch.randn(tokens, width, generator=g, device="cuda")).to(torch.bfloat16)
        losses = block.gradients(h, labels, b)
        block.step(b, 3e-3)
        if it % 5 == 0 or it == iterations - 1:
            print("iteration %d: batches %s, losses %s" % (it, b, ["%.3f" % v for v in losses.tolist()]), flush=True)
        b, _ = control.observe(synth.iteration_times(b, speeds))
    return losses


if __name__ == "__main__":
    main(vocabulary=1000 if sys.argv[1:] == ["tokens"] else 0)
