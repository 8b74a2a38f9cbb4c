"""Learners of a residual network in 8 bits, end to end: weights pulled in FP8, every block a norm with the residual's
addition, two 8-bit products and a gelu between them, the backward pass into the vector that is pushed, clipped by its global
norm, updates under n-softsync.

    python examples/learner_block.py [updates]

The data is synthetic: the labels come from a fixed random linear map.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1509_04210_b200 import binding as rb  # noqa: E402
from paper_1509_04210_b200 import learner as ln  # noqa: E402


class Network:
    """width -> (norm, width -> hidden, gelu, hidden -> width, added to the stream) * blocks -> norm -> classes, in one flat vector."""

    def __init__(self, width, hidden, classes, blocks):
        self.width, self.hidden, self.blocks = width, hidden, blocks
        self.parts, at = {}, 0               # name: (offset, shape)
        for i in range(blocks):
            for name, shape in (("norm", (width,)), ("up", (hidden, width)), ("down", (width, hidden))):
                self.parts[name, i], at = (at, shape), at + shape[0] * (shape[1] if len(shape) > 1 else 1)
        self.parts["norm", blocks], at = (at, (width,)), at + width
        self.parts["head", 0], at = (at, (classes, width)), at + classes * width
        self.nparams = at

    def views(self, vector):
        return {k: vector[at:at + torch.Size(shape).numel()].view(shape) for k, (at, shape) in self.parts.items()}

    def initial(self, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        theta = torch.ones(self.nparams, device="cuda")
        for (name, _), v in self.views(theta).items():
            if name != "norm":
                v.normal_(0.0, v.shape[1] ** -0.5, generator=gen)
        return theta


class Learner:
    """One learner: the matrices it last pulled, in FP8 as they stand and transposed, the norms' weights, its gradients."""

    def __init__(self, net, seed):
        self.net, self.gen = net, torch.Generator(device="cuda").manual_seed(seed)
        self.pushed = torch.empty(net.nparams, device="cuda")
        self.grads = net.views(self.pushed)
        self.theta = torch.empty(net.nparams, device="cuda")      # of which the norms' weights are used
        self.weights, self.turned, self.ts = {}, {}, 0

    def pull(self, ps):
        self.ts = ps.pull(self.theta)
        self.norms = {k: v for k, v in self.net.views(self.theta).items() if k[0] == "norm"}
        for k, (at, shape) in self.net.parts.items():
            if k[0] != "norm":
                self.weights[k], _ = ln.pull_fp8(ps, at, *shape, out=self.weights.get(k))
                self.turned[k], _ = ln.pull_fp8(ps, at, *shape, transpose=True, out=self.turned.get(k))

    def compute(self, x, label):
        """Forward and backward over a mini-batch; the gradients land in ``grads``.  Returns the mean loss."""
        net, kept = self.net, []
        stream, branch = x, None
        for i in range(net.blocks + 1):
            # the stream with the branch before added to it, and what the next product and its weight's gradient read
            if branch is None:
                s = stream
                y, kept_y = ln.rms_norm(s, self.norms["norm", i], fp8=True, keep=True)
            else:
                y, s, kept_y = ln.rms_norm(branch, self.norms["norm", i], residual=stream, fp8=True, keep=True)
            stream = s
            if i == net.blocks:
                break
            h = ln.fp8_matmul(y, self.weights["up", i])
            a, kept_h = ln.act8_forward("gelu", h)
            branch = ln.fp8_matmul(a, self.weights["down", i])
            kept.append((s, kept_y, kept_h, a))
        logits = ln.fp8_matmul(y, self.weights["head", 0], torch.float32)

        logp = torch.log_softmax(logits, 1)
        loss = -logp.gather(1, label.unsqueeze(1)).mean()
        dz = torch.exp(logp)
        dz.scatter_add_(1, label.unsqueeze(1), torch.full_like(label, -1.0, dtype=torch.float32).unsqueeze(1))
        dz /= len(label)

        ln.act8_weight_grad(dz, kept_y, out=self.grads["head", 0])
        dy = ln.fp8_matmul(dz, self.turned["head", 0])
        ds, _ = ln.rms_norm_backward(dy, stream, self.norms["norm", net.blocks], out_weight=self.grads["norm", net.blocks])
        for i in reversed(range(net.blocks)):
            s, kept_y, kept_h, a = kept[i]
            # ds is the gradient of the stream and of the branch that was added to it
            ln.fp8_matmul(ln.fp8_quantize(ds, transpose=True), ln.fp8_quantize(a, transpose=True), out=self.grads["down", i])
            dh = ln.act8_backward("gelu", ln.fp8_matmul(ds, self.turned["down", i]), kept_h)
            ln.act8_weight_grad(dh, kept_y, out=self.grads["up", i])
            dy = ln.fp8_matmul(dh, self.turned["up", i])
            ds, _ = ln.rms_norm_backward(dy, s, self.norms["norm", i], dsum=ds, out=ds, out_weight=self.grads["norm", i])
        return loss

    def clip(self, most):
        """Scales the gradients, in the vector that is pushed, to a norm of ``most``.  Returns the norm they had."""
        return ln.clip_gradients(list(self.grads.values()), most)


def train(updates=100, learners=4, n=2, batch=128, width=256, hidden=512, classes=40, blocks=2, rate=0.05, most=1.0, seed=1):
    """The losses the learners saw, in the order of their pushes."""
    net = Network(width, hidden, classes, blocks)
    teacher = torch.randn(width, classes, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + 1000))
    ps = rb.ParameterServer(net.nparams, learners, n, rate * n, 0.9, 0.0, stream=torch.cuda.current_stream())
    ps.set_weights(net.initial(seed))
    group = [Learner(net, seed + 1 + i) for i in range(learners)]
    for l in group:
        l.pull(ps)
    sched = rb.Scheduler(learners, n, rb.SCHED_SOFTSYNC_ROUNDS, seed)
    losses = []
    while ps.timestamp() < updates:
        event = sched.next(1)[0]
        l = group[int(event["learner"])]
        if event["kind"] == rb.EV_PUSH:
            x = torch.randn(batch, width, device="cuda", generator=l.gen)
            losses.append(l.compute(x.bfloat16(), (x @ teacher).argmax(1)))
            l.clip(most)
            ps.push(l.pushed, l.ts)
        elif event["kind"] == rb.EV_STEP:
            assert ps.step() == 1
        elif event["kind"] == rb.EV_PULL:
            l.pull(ps)
    ln.sync()
    ps.close()
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    got = train(int(sys.argv[1]) if len(sys.argv) > 1 else 100)
    tenth = max(1, len(got) // 10)
    for k in range(0, len(got), tenth):
        part = got[k:k + tenth]
        print("pushes %4d to %4d: loss %.3f" % (k, k + len(part) - 1, sum(part) / len(part)))
