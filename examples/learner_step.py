"""Learners that share the server's GPU, end to end: weights pulled in 4 bits, a two-layer network forward on
them, checkpoints in 8 bits, the backward pass into the vector that is pushed, updates under n-softsync.

    python examples/learner_step.py [updates]

The data is synthetic: the labels come from a fixed random network of the same shape.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1509_04210_b200 import binding as rb  # noqa: E402
from paper_1509_04210_b200 import learner as ln  # noqa: E402


class Network:
    """inputs -> hidden (gelu) -> classes, as two matrices in one flat vector of weights."""

    def __init__(self, inputs, hidden, classes):
        self.layers = [(0, hidden, inputs), (hidden * inputs, classes, hidden)]
        self.nparams = hidden * inputs + classes * hidden

    def initial(self, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        theta = torch.empty(self.nparams, device="cuda")
        for offset, rows, cols in self.layers:
            theta[offset:offset + rows * cols].normal_(0.0, cols ** -0.5, generator=gen)
        return theta

    def matrix(self, theta, i):
        offset, rows, cols = self.layers[i]
        return theta[offset:offset + rows * cols].view(rows, cols)


class Learner:
    """One learner: the weights it last pulled, in 4 bits, and the buffer its gradient is pushed from."""

    def __init__(self, net, seed):
        self.net, self.gen = net, torch.Generator(device="cuda").manual_seed(seed)
        self.grad = torch.empty(net.nparams, device="cuda")
        self.weights = [None, None]      # as they stand, for the forward products
        self.transposed = None           # the second layer's, for the backward product
        self.ts = 0

    def pull(self, ps):
        for i, (offset, rows, cols) in enumerate(self.net.layers):
            self.weights[i], self.ts = ln.pull_mx4(ps, offset, rows, cols, out=self.weights[i])
        offset, rows, cols = self.net.layers[1]
        self.transposed, _ = ln.pull_mx4(ps, offset, rows, cols, transpose=True, out=self.transposed)

    def compute(self, x, label):
        """Forward and backward over a mini-batch; the gradient lands in ``grad``.  Returns the mean loss."""
        kept_x = ln.act8_save(x)
        h = ln.mx4_matmul(x, self.weights[0])
        y, kept_h = ln.act8_forward("gelu", h)
        kept_y = ln.act8_save(y)
        logits = ln.mx4_matmul(y, self.weights[1], torch.float32)

        logp = torch.log_softmax(logits, 1)
        loss = -logp.gather(1, label.unsqueeze(1)).mean()
        dz = torch.exp(logp)
        dz.scatter_add_(1, label.unsqueeze(1), torch.full_like(label, -1.0, dtype=torch.float32).unsqueeze(1))
        dz /= len(label)

        ln.act8_weight_grad(dz, kept_y, out=self.net.matrix(self.grad, 1))
        dy = ln.mx4_matmul(dz, self.transposed)
        dh = ln.act8_backward("gelu", dy, kept_h)
        ln.act8_weight_grad(dh, kept_x, out=self.net.matrix(self.grad, 0))
        return loss


def train(updates=200, learners=4, n=2, batch=128, inputs=256, hidden=512, classes=40, rate=0.05, seed=1):
    """The losses the learners saw, in the order of their pushes."""
    net = Network(inputs, hidden, classes)
    teacher = Network(inputs, hidden, classes).initial(seed + 1000)
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
            x = torch.randn(batch, inputs, device="cuda", generator=l.gen)
            h = torch.nn.functional.gelu(x @ net.matrix(teacher, 0).t())
            label = (h @ net.matrix(teacher, 1).t()).argmax(1)
            losses.append(l.compute(x.bfloat16(), label))
            ps.push(l.grad, l.ts)
        elif event["kind"] == rb.EV_STEP:
            assert ps.step() == 1
        elif event["kind"] == rb.EV_PULL:
            l.pull(ps)
    ln.sync()
    ps.close()
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    got = train(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
    tenth = max(1, len(got) // 10)
    for k in range(0, len(got), tenth):
        part = got[k:k + tenth]
        print("pushes %4d to %4d: loss %.3f" % (k, k + len(part) - 1, sum(part) / len(part)))
