"""The middle step of quantizing a whole network (Sec. 4.2.3 of the paper): the conv layers
are quantized, the FC layers behind them are still dense and are fine-tuned on the
quantized layers' outputs, then quantized too.

A small network on synthetic images, labelled by a fixed random teacher.  Each step runs
the quantized conv stack, two dense layers with dropout between them, softmax cross entropy
with its gradient, the backward pass, and updates the weights along their orthogonalised
momentum.  The trained layers are then quantized in both ways: with codebooks, and to 8-bit integers.

    python examples/finetune_fc.py [--steps 60] [--dtype fp32|bf16] [--dropout 0.0]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_1512_06473_gb300 as q  # noqa: E402

IMAGES, SIDE, HIDDEN, CLASSES = 512, 27, 256, 10


def conv_stack(g):
    """Two product-quantized conv layers with pools: [N, 8, 27, 27] -> [N, 24, 6, 6]."""
    def layer(cs, ct, k, stride, pad, csp, K, std):
        D = torch.randn(cs // csp, K, csp, generator=g, device="cuda") * std
        codes = torch.randint(0, K, (ct, k * k, cs // csp), generator=g, device="cuda", dtype=torch.uint8)
        return q.ConvLayer(D, codes, torch.zeros(ct, device="cuda"), ct, k, k, stride, pad, relu=True)
    return q.Net([layer(8, 32, 5, 2, 2, 4, 128, 0.1), q.PoolLayer(3, 2),
                  layer(32, 24, 5, 1, 2, 4, 64, 0.05)], (8, SIDE, SIDE))


class Update:
    """Weights along their orthogonalised momentum (a step of the Muon optimiser)."""

    def __init__(self, weight, lr, momentum=0.9):
        self.weight, self.lr, self.momentum = weight, lr, momentum
        self.buf = torch.zeros_like(weight)

    def step(self, grad):
        self.buf.mul_(self.momentum).add_(grad)
        m, n = grad.shape
        o = q.orthogonalize(grad.add(self.buf, alpha=self.momentum))
        self.weight.add_(o, alpha=-self.lr * max(1.0, m / n) ** 0.5)


def main(steps=60, dtype="fp32", seed=0, show=True, dropout=0.0):
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(seed)
    net = conv_stack(g)
    images = torch.randn(IMAGES, 8, SIDE, SIDE, generator=g, device="cuda")
    features = net.forward(images).flatten(1)
    Cs = features.shape[1]
    labels = (features @ torch.randn(Cs, CLASSES, generator=g, device="cuda")).argmax(1)
    labels[::50] = -100  # some images have no label

    w1 = (torch.randn(HIDDEN, Cs, generator=g, device="cuda") * (2.0 / Cs) ** 0.5).to(dt)
    w2 = (torch.randn(CLASSES, HIDDEN, generator=g, device="cuda") * 0.01).to(dt)
    b1, b2 = torch.zeros(HIDDEN, device="cuda"), torch.zeros(CLASSES, device="cuda")
    u1, u2 = Update(w1, 0.02), Update(w2, 0.02)
    history = []
    for step in range(steps):
        x = net.forward(images).flatten(1).to(dt)
        h, z = q.dense_forward(x, w1, b1, act="relu", pre=True)
        if dropout:  # (what is dropped follows from seed and step: nothing is kept for the way back)
            h = q.dropout_forward(h, dropout, seed, step, out=h)
        loss, _, dh, dw2, db2 = q.xent_grad(h, w2, labels, b2)
        if dropout:
            dh = q.dropout_backward(dh, dropout, seed, step, out=dh)
        _, dw1, db1 = q.dense_backward(dh, x, w1, z, "relu", need_dx=False)
        u1.step(dw1)
        u2.step(dw2)
        b1.add_(db1, alpha=-0.1)
        b2.add_(db2, alpha=-0.1)
        history.append(loss.sum() / (labels >= 0).sum())
        if show and step % 10 == 0:
            print(f"step {step:3d}  loss {float(history[-1]):.4f}")

    # the last step: the fine-tuned layers quantized as well
    def quantize(w, csp, K):
        w = w.float().contiguous()
        init = torch.stack([w[torch.randperm(w.shape[0], generator=g, device="cuda")[:K] % w.shape[0],
                              m * csp:(m + 1) * csp] for m in range(w.shape[1] // csp)])
        return q.pq_quantize_fc(w, csp, K, init.contiguous(), 10)

    (D1, c1), (D2, c2) = quantize(w1, 4, 128), quantize(w2, 4, min(CLASSES, 32))
    h = q.fc_forward(features, D1, c1, b1, relu=True)
    logits = q.fc_forward(h, D2, c2, b2)
    keep = labels >= 0
    dense_h = q.dense_forward(features.to(dt), w1, b1, act="relu")
    dense_logits = q.dense_forward(dense_h, w2, b2).float()
    (c1, s1), (c2, s2) = q.int8_quantize(w1), q.int8_quantize(w2)
    int8_h = q.int8_dense_forward(features.to(dt), c1, s1, b1, act="relu")
    int8_logits = q.int8_dense_forward(int8_h, c2, s2, b2).float()
    right = [float((v.argmax(1)[keep] == labels[keep]).float().mean()) for v in (dense_logits, logits, int8_logits)]
    losses = [float(v) for v in history]
    if show:
        print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; right on the training images: dense "
              f"{right[0]:.1%}, quantized {right[1]:.1%}, in 8 bits {right[2]:.1%}")
    return losses, right


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--dtype", choices=["fp32", "bf16"], default="fp32")
    p.add_argument("--dropout", type=float, default=0.0)
    a = p.parse_args()
    main(a.steps, a.dtype, dropout=a.dropout)
