"""An 8-bit dense head on the activities of Forward-Forward layers.

Two FF layers are trained on the learnable synthetic task, one after another
and without a gradient between them.  On the last one's activities h a head is
trained by backpropagation:

    z = relu(W1 d + b1),   d = dropout(silu(group_norm(h))),   logits = W2 z + b2

Both of its products, and the four of its backward pass, are 8-bit: the
master weights stay fp32 and are quantized once a step, both ways round; the
activities and their gradients are quantized as they come.  Then the weights
are quantized for good and single samples are answered from a CUDA graph.

    python examples/eight_bit_head.py [--steps N] [--batch B]
"""

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2404_08573_gb300 import ff, synth  # noqa: E402

CLASSES = 10


class EightBitHead:
    """group norm, silu, dropout and two 8-bit linear layers, with their gradient."""

    def __init__(self, features: int, hidden: int, groups: int, p: float = 0.2, seed: int = 0, lr: float = 2e-3):
        dev = "cuda"
        self.features, self.hidden, self.groups, self.p, self.seed = features, hidden, groups, p, seed
        self.gamma, self.beta = torch.ones(features, device=dev), torch.zeros(features, device=dev)
        self.w1 = torch.from_numpy(synth.he_uniform(seed, hidden, features)).to(dev)
        self.w2 = torch.from_numpy(synth.he_uniform(seed + 1, CLASSES, hidden)).to(dev)
        self.b1, self.b2 = torch.zeros(hidden, device=dev), torch.zeros(CLASSES, device=dev)
        self.offset = 0  # position in the masks' generator
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.optimizer = torch.optim.Adam(self.parameters, lr=lr)
        self.served = None

    @property
    def parameters(self):
        return [self.gamma, self.beta, self.w1, self.b1, self.w2, self.b2]

    def gradients(self, h, y):
        """Mean cross-entropy of a batch (h bf16 [B, features], y int64 [B]) and the parameters' gradients."""
        B, act = h.shape[0], "silu"
        w1, w1t = ff.fp8_quantize_both(self.w1, tile=True)
        w2, w2t = ff.fp8_quantize_both(self.w2, tile=True)
        a, mean, rstd = ff.group_norm_act(h, self.gamma, self.beta, self.groups, act=act)
        d = ff.dropout(a, self.p, self.seed, self.offset)
        dq, dqt = ff.fp8_quantize_both(d)
        z = ff.fp8_matmul(dq, w1, bias=self.b1, relu=True, status=self.status)
        zq, zqt = ff.fp8_quantize_both(z)
        logits = ff.fp8_matmul(zq, w2, bias=self.b2, out_dtype=torch.float32, status=self.status)
        loss = torch.nn.functional.cross_entropy(logits, y)

        g = torch.softmax(logits, dim=1)
        g[torch.arange(B, device=h.device), y] -= 1.0
        g /= B
        gq, gqt = ff.fp8_quantize_both(g)
        dw2 = ff.fp8_matmul(gqt, zqt, out_dtype=torch.float32, status=self.status)
        dz = ff.fp8_matmul(gq, w2t, status=self.status) * (z > 0)
        dzq, dzqt = ff.fp8_quantize_both(dz)
        dw1 = ff.fp8_matmul(dzqt, dqt, out_dtype=torch.float32, status=self.status)
        da = ff.dropout(ff.fp8_matmul(dzq, w1t, status=self.status), self.p, self.seed, self.offset)
        _, dgamma, dbeta = ff.group_norm_act_backward(da, h, mean, rstd, self.gamma, self.beta, self.groups, act=act)
        return loss, [dgamma, dbeta, dw1, dz.float().sum(0), dw2, g.sum(0)]

    def train_step(self, h, y):
        loss, grads = self.gradients(h, y)
        for p, g in zip(self.parameters, grads):
            p.grad = g
        self.optimizer.step()
        self.offset += ff.dropout_words(h.shape[0], self.features)
        self.served = None
        return loss

    def logits(self, h):
        """Logits [n, 10] without dropout; the weights are quantized at the first call after a step."""
        if self.served is None:
            self.served = ff.fp8_quantize(self.w1, tile=True), ff.fp8_quantize(self.w2, tile=True)
        w1, w2 = self.served
        a, _, _ = ff.group_norm_act(h, self.gamma, self.beta, self.groups)
        z = ff.fp8_matmul(ff.fp8_quantize(a), w1, bias=self.b1, relu=True, status=self.status)
        return ff.fp8_matmul(ff.fp8_quantize(z), w2, bias=self.b2, out_dtype=torch.float32, status=self.status)

    def check(self):
        if int(self.status.item()):
            raise RuntimeError("a wait of an 8-bit product timed out")


def ff_layers(x, y, widths, batch: int, lr: float = 0.001, seed: int = 0):
    """FF layers trained for one pass over x, y (numpy), greedily, layer by layer."""
    layers, fan_in = [], x.shape[1]
    for i, width in enumerate(widths):
        layers.append(ff.Layer(fan_in, width, prec="bf16", lr=lr, init_seed=seed + i, max_rows=2 * batch))
        fan_in = width
    net = ff.Net(layers, max_B=batch)
    for i in range(0, len(x) - batch + 1, batch):
        xb, yb = x[i:i + batch], y[i:i + batch]
        x2, l2 = synth.pair_batch(xb, yb, synth.negative_labels(yb, seed=seed + 1 + i))
        net.train_step(torch.from_numpy(x2).cuda(), torch.from_numpy(l2).cuda(), B=batch)
        net.sync()
    net.close()
    return layers


def activities(layers, x):
    """The last layer's activities [n, features] of images x (numpy), with the neutral label."""
    a = layers[0].new_activation(len(x), layers[0].in_features)
    a[:, :x.shape[1]] = torch.from_numpy(x).cuda()
    a[:, :CLASSES] = 0.1
    for layer in layers:
        h = layer.new_activation(len(x))
        layer.forward(a, h_out=h)
        a = h
    return a[:, :layers[-1].out_features]


def serve(head, features):
    """A graph that answers one sample: (its input [1, features], its logits, the graph)."""
    x = torch.zeros(1, features, dtype=torch.bfloat16, device="cuda")
    head.logits(x)  # the weights' 8-bit forms are made before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = head.logits(x)
    return x, out, graph


def run(samples: int = 8192, batch: int = 512, steps: int = 120, widths=(500, 500), hidden: int = 256, groups: int = 10,
        seed: int = 0, report=print):
    x, y = synth.learnable_task(samples + 1024, seed=seed)
    layers = ff_layers(x[:samples], y[:samples], widths, batch, seed=seed)
    h, hy = activities(layers, x), torch.from_numpy(y.astype(np.int64)).cuda()
    head = EightBitHead(widths[-1], hidden, groups, seed=seed)
    losses = []
    for step in range(steps):
        i = step * batch % (samples - batch + 1)
        losses.append(head.train_step(h[i:i + batch], hy[i:i + batch]))
    losses = torch.stack(losses).cpu().numpy()
    logits = head.logits(h[samples:])
    accuracy = float((logits.argmax(1) == hy[samples:]).float().mean())
    one, out, graph = serve(head, widths[-1])
    same = 0
    for i in range(16):
        one.copy_(h[samples + i:samples + i + 1])
        graph.replay()
        same += int(out.argmax().item() == int(logits[i].argmax().item()))
    head.check()
    for layer in layers:
        layer.check()
        layer.close()
    report(f"cross-entropy {losses[:8].mean():.3f} -> {losses[-8:].mean():.3f}, accuracy on 1024 held-out samples "
           f"{accuracy:.3f}, {same} of 16 single answers as in the batch")
    return losses, accuracy, same


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=120)
    parser.add_argument("--batch", type=int, default=512)
    args = parser.parse_args()
    run(batch=args.batch, steps=args.steps)
