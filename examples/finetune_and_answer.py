"""Fine-tunes a small network on a whole image and answers with 8-bit fully connected layers.

The network scans an image densely (every window at once).  A training step computes the
gradient over all windows in one call, clips it by its norm over all tensors and moves the
weights.  Then the network's fully connected head, its last two layers, is coded in 8 bits
with a scale for each output channel, and the maps of the layers before it go through the
head window by window as 8-bit tokens.

    python examples/finetune_and_answer.py [steps]
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1508_06904_amd import dss, workloads as wl  # noqa: E402

BODY = [("conv", 3, 16, 5, 5, "relu"), ("pool", 2, 2), ("conv", 16, 64, 3, 3, "relu"), ("pool", 2, 2),
        ("conv", 64, 256, 4, 4, "relu")]
HEAD = [("conv", 256, 128, 1, 1, "relu"), ("conv", 128, 3, 1, 1, "none")]


def train_step(layers, x, target, rate, max_norm):
    """One step of gradient descent on the mean squared error over all windows: (loss, gradient norm)."""
    plan = dss.Plan(layers, 2, x.shape[0])
    diff = plan.eval_dense(x) - target
    gw, gb, _ = plan.backward(x, diff * (2.0 / diff.numel()), with_signal_grad=False)
    weights, biases = plan.split_grads(gw, gb)
    grads = weights + biases
    norm, _ = dss.clip_grads(grads, max_norm, out=grads)
    convs = [l for l in layers if l["kind"] == "conv"]
    for l, w, b in zip(convs, weights, biases):
        l["weight"] = l["weight"] - rate * w.cpu().numpy()
        l["bias"] = l["bias"] - rate * b.cpu().numpy()
    return float((diff * diff).mean()), float(norm)


def answer(layers, x):
    """The network's dense output with its head in 8 bits: [3][H'][W']."""
    n = len(HEAD)
    maps = dss.Plan(layers[:-n], 2, x.shape[0]).eval_dense(x)
    shape, y = maps.shape[1:], maps.flatten(1)
    for l in layers[-n:]:
        w, scales = dss.quantize_tokens(torch.from_numpy(l["weight"].reshape(l["cout"], l["cin"])).cuda())
        y = dss.linear_i8(y.t(), w, scales, bias=torch.from_numpy(l["bias"]).cuda(), act=l["act"], planar=True)
    return y.unflatten(1, shape)


def main(steps=8, size=150):
    rng = np.random.default_rng(0)
    layers = wl.init_layers(BODY + HEAD, rng)
    x = torch.from_numpy(wl.blob_image(rng, 3, size, size, 8)).cuda()
    with torch.no_grad():
        out = dss.Plan(layers, 2, 3).eval_dense(x)
        # what to learn: the smoothed colours at each window's centre
        margin = (size - out.shape[1]) // 2
        target = torch.nn.functional.avg_pool2d(x[None], 9, 1, 4)[0, :, margin:margin + out.shape[1],
                                                                  margin:margin + out.shape[2]].contiguous()
    history = []
    for step in range(steps):
        loss, norm = train_step(layers, x, target, rate=0.05, max_norm=1.0)
        history.append(loss)
        print("step %d: loss %.4f, gradient norm %.3f%s" % (step, loss, norm, " (clipped to 1)" if norm > 1 else ""))
    full = dss.Plan(layers, 2, 3).eval_dense(x)
    coded = answer(layers, x)
    off = float((coded - full).norm() / full.norm())
    print("head in 8 bits: %d windows, %.2f %% off the binary32 network" % (full[0].numel(), 100 * off))
    return history, off


if __name__ == "__main__":
    main(*map(int, sys.argv[1:2]))
