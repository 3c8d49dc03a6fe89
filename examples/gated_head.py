"""Fine-tune a gated head on a frozen ResNet-50's last feature map with 8-bit checkpoints, then serve it token by token.

    python examples/gated_head.py [--images 8] [--steps 20]

The tokens are the pixels of the backbone's [N, 7, 7, 2048] output, projected to C channels by a Linear-BN block in 8 bits (its input is
what would take the most memory to keep: 2048 channels a token).  The head learns to reproduce a random teacher head.  What the trained layers
keep of the forward pass for the backward one are codes and scales."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2305_11624_amd import quant as Q  # noqa: E402
from paper_2305_11624_amd.resnet50 import ResNet50  # noqa: E402


def head(M, C, F, train):
    return Q.Linear(M, 2048, C, train=train, need_dx=False), Q.GatedBlock(M, C, F, train=train)


def pack(layers, weights):
    layers[0].pack_weight(weights[0])
    layers[1].pack_weights(*weights[1:])


def forward(layers, x):
    return layers[1].forward(layers[0].forward(x))


def main(images=8, steps=20, C=256, F=512, lr=0.015):
    gen = torch.Generator(device="cuda").manual_seed(0)

    def weights():
        sizes = (C, 2048), (2 * F, C), (C, F)
        return [torch.randn(*s, generator=gen, device="cuda") * s[1] ** -0.5 for s in sizes]   # fp32 masters

    def bf16(ws):
        return [w.bfloat16() for w in ws]

    net = ResNet50(images, 224, mode="tune", group_units=True)
    x = net.forward(torch.randn(images, 224, 224, 3, generator=gen, device="cuda").bfloat16()).view(-1, 2048)
    x = (x.float() / x.float().std()).bfloat16()
    M = x.shape[0]
    teacher, student = weights(), weights()
    layers = head(M, C, F, train=True)
    pack(layers, bf16(teacher))
    target = forward(layers, x).float().clone()
    losses = []
    for _ in range(steps):
        pack(layers, bf16(student))
        out = forward(layers, x).float()
        diff = out - target
        losses.append(float(diff.square().mean()))
        dout = (diff * (2 / M)).bfloat16()
        dh, dW_up, dW_down = layers[1].backward(dout)
        _, dW_in, _ = layers[0].backward(dh)      # (the backbone is frozen: no gradient of x)
        for w, g in zip(student, (dW_in, dW_up, dW_down)):
            g = g.float()
            w -= lr * w.norm() / g.norm() * g      # a step in proportion to the weight's own size
    kept = sum(l.saved_bytes() for l in layers)
    whole = 2 * M * (2048 + C + 3 * F)
    print("%d tokens: loss %.4f -> %.4f in %d steps; kept for backward: codes and scales %.2f MB, the same rows in bf16 %.2f MB"
          % (M, losses[0], losses[-1], steps, kept / 1e6, whole / 1e6))
    one = head(1, C, F, train=False)
    pack(one, bf16(student))
    pack(layers, bf16(student))
    every = forward(layers, x)
    worst = max(float((forward(one, x[i:i + 1]).float() - every[i:i + 1].float()).abs().max()) for i in (0, M // 2, M - 1))
    print("one token at a time: at most %.2g from the batch" % worst)
    return losses, worst, kept, whole


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--images", type=int, default=8)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    main(a.images, a.steps)
