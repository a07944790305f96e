"""A deep head with a residual stream on the activities of Forward-Forward layers.

On the last FF layer's activities a head of residual blocks is trained by
backpropagation:

    x0 = W0 h
    s_i = s_(i-1) + x_(i-1),  y_i = rms_norm(s_i),  x_i = W2_i relu(W1_i y_i)
    logits = W rms_norm(s + x) + b

to the labels' log-probabilities and, a little, to the entropy of its answers.
Its products are 8-bit in training (weights quantized once a step, both ways
round); the gradients are clipped together.  Then the weights are quantized for
good, to 8 or to 4 bits, and samples are answered with their likeliest classes,
single ones from a CUDA graph.

    python examples/deep_head.py [--steps N] [--batch B]
"""

import argparse
import os
import sys

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [os.path.join(HERE, ".."), HERE]

from eight_bit_head import activities, ff_layers  # noqa: E402
from paper_2404_08573_gb300 import ff, synth  # noqa: E402

CLASSES = 10


class DeepHead:
    def __init__(self, features: int, width: int, hidden: int, blocks: int, seed: int = 0, lr: float = 1e-3, bonus: float = 0.01,
                 max_norm: float = 1.0):
        def weight(i, rows, cols):
            return torch.from_numpy(synth.he_uniform(seed + i, rows, cols)).cuda()

        self.bonus, self.max_norm = bonus, max_norm
        self.w0 = weight(0, width, features)
        self.gammas = [torch.ones(width, device="cuda") for _ in range(blocks + 1)]
        self.w1 = [weight(10 + i, hidden, width) for i in range(blocks)]
        self.w2 = [weight(50 + i, width, hidden) * 0.5 for i in range(blocks)]
        self.w, self.b = weight(99, CLASSES, width), torch.zeros(CLASSES, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.optimizer = torch.optim.Adam(self.parameters, lr=lr)
        self.served = {}

    @property
    def weights(self):
        return [self.w0] + self.w1 + self.w2 + [self.w]

    @property
    def parameters(self):
        return self.weights + self.gammas + [self.b]

    def _mm(self, a, b, **kw):
        return ff.fp8_matmul(a, b, status=self.status, **kw)

    def gradients(self, h, y):
        """Mean of -logp - bonus * entropy over a batch (h bf16 [B, features], y int32 [B]; a label of -1 counts for
        nothing), and the gradients of the parameters, in their order."""
        n, B = len(self.w1), h.shape[0]
        q = [ff.fp8_quantize_both(w, tile=True) for w in self.weights]
        (w0, _), w1, w2, (w, wt) = q[0], q[1:1 + n], q[1 + n:1 + 2 * n], q[-1]
        hq, hqt = ff.fp8_quantize_both(h)
        x, s, kept = self._mm(hq, w0), None, []
        for i in range(n):
            v, s, rstd = ff.rms_norm(x, self.gammas[i], residual=s)
            vq, vqt = ff.fp8_quantize_both(v)
            z = self._mm(vq, w1[i][0], relu=True)
            zq, zqt = ff.fp8_quantize_both(z)
            x = self._mm(zq, w2[i][0])
            kept.append((s, rstd, vqt, z, zqt))
        v, s, rstd = ff.rms_norm(x, self.gammas[n], residual=s)
        vq, vqt = ff.fp8_quantize_both(v)
        logits = self._mm(vq, w, bias=self.b, out_dtype=torch.float32)
        r = ff.label_logprobs(logits, y)
        loss = -(r.logp + self.bonus * r.entropy).mean()

        each = torch.full((B,), -1.0 / B, device=h.device)
        g = ff.label_logprobs_backward(logits, y, r.stats, each, entropy=r.entropy, dentropy=self.bonus * each)
        gq, gqt = ff.fp8_quantize_both(g)
        dw, db = self._mm(gqt, vqt, out_dtype=torch.float32), g.sum(0)
        ds, dgamma = ff.rms_norm_backward(self._mm(gq, wt), s, rstd, self.gammas[n])
        dgammas, dw1, dw2 = [dgamma], [], []
        for i in reversed(range(n)):  # ds: the gradient of the stream and of the block's output alike
            s, rstd, vqt, z, zqt = kept[i]
            dq, dqt = ff.fp8_quantize_both(ds)
            dw2.append(self._mm(dqt, zqt, out_dtype=torch.float32))
            dzq, dzqt = ff.fp8_quantize_both(self._mm(dq, w2[i][1]) * (z > 0))
            dw1.append(self._mm(dzqt, vqt, out_dtype=torch.float32))
            ds, dgamma = ff.rms_norm_backward(self._mm(dzq, w1[i][1]), s, rstd, self.gammas[i], dh=ds)
            dgammas.append(dgamma)
        _, dqt = ff.fp8_quantize_both(ds)
        dw0 = self._mm(dqt, hqt, out_dtype=torch.float32)
        return loss, [dw0] + dw1[::-1] + dw2[::-1] + [dw] + dgammas[::-1] + [db]

    def train_step(self, h, y):
        """One clipped Adam step; returns the loss and the gradients' norm before clipping."""
        loss, grads = self.gradients(h, y)
        norm = ff.clip_grad_norm(grads, self.max_norm)
        for p, g in zip(self.parameters, grads):
            p.grad = g
        self.optimizer.step()
        self.served = {}
        return loss, norm

    def logits(self, h, bits: int = 4):
        """Logits [n, 10] with weights of 8 or 4 bits, quantized at the first call after a step."""
        if bits not in self.served:
            self.served[bits] = [ff.fp8_quantize(w, tile=True) if bits == 8 else ff.fp4_quantize(w) for w in self.weights]
        quantize, mm = (ff.fp8_quantize, self._mm) if bits == 8 else (ff.fp4_quantize, self._mm4)
        n, q = len(self.w1), self.served[bits]
        x, s = mm(quantize(h), q[0]), None
        for i in range(n + 1):
            if bits == 8:
                v, s, _ = ff.rms_norm_fp8(x, self.gammas[i], residual=s)
            else:
                v, s, _ = ff.rms_norm(x, self.gammas[i], residual=s)
                v = quantize(v)
            if i == n:
                return mm(v, q[-1], bias=self.b, out_dtype=torch.float32)
            x = mm(quantize(mm(v, q[1 + i], relu=True)), q[1 + n + i])

    def _mm4(self, a, b, **kw):
        return ff.fp4_matmul(a, b, status=self.status, **kw)

    def answer(self, h, bits: int = 4, top: int = 3):
        """The `top` likeliest classes, their log-probabilities and the answers' entropy."""
        r = ff.label_logprobs(self.logits(h, bits), None, top=top)
        return r.top_index, r.top_logp, r.entropy

    def check(self):
        if int(self.status.item()):
            raise RuntimeError("a wait of a product timed out")


def serve(head, features, bits: int = 4):
    """A graph that answers one sample: (its input [1, features], its outputs, the graph)."""
    x = torch.zeros(1, features, dtype=torch.bfloat16, device="cuda")
    head.answer(x, bits)  # the weights' small forms are made before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = head.answer(x, bits)
    return x, out, graph


def run(samples: int = 8192, batch: int = 512, steps: int = 120, widths=(500, 500), width: int = 384, hidden: int = 512,
        blocks: int = 2, seed: int = 0, report=print):
    x, y = synth.learnable_task(samples + 1024, seed=seed)
    layers = ff_layers(x[:samples], y[:samples], widths, batch, seed=seed)
    h, hy = activities(layers, x), torch.from_numpy(y.astype(np.int32)).cuda()
    head = DeepHead(widths[-1], width, hidden, blocks, seed=seed)
    losses, norms = [], []
    for step in range(steps):
        i = step * batch % (samples - batch + 1)
        loss, norm = head.train_step(h[i:i + batch], hy[i:i + batch])
        losses.append(loss)
        norms.append(norm)
    losses, norms = torch.stack(losses).cpu().numpy(), torch.cat(norms).cpu().numpy()
    accuracy = {}
    for bits in (8, 4):
        index, _, _ = head.answer(h[samples:], bits)
        accuracy[bits] = float((index[:, 0] == hy[samples:]).float().mean())
    one, out, graph = serve(head, widths[-1])
    one.copy_(h[samples:samples + 1])
    graph.replay()
    answer = [t[0].cpu().numpy() for t in out]
    head.check()
    for layer in layers:
        layer.check()
        layer.close()
    report(f"loss {losses[:8].mean():.3f} -> {losses[-8:].mean():.3f}, accuracy on 1024 held-out samples {accuracy[8]:.3f} in 8 bits, "
           f"{accuracy[4]:.3f} in 4; one sample: classes {answer[0].tolist()}, log-probabilities {np.round(answer[1], 3).tolist()}")
    return losses, norms, accuracy, answer


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=120)
    parser.add_argument("--batch", type=int, default=512)
    args = parser.parse_args()
    run(batch=args.batch, steps=args.steps)
