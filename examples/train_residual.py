"""A data-parallel training step, end to end: residual blocks on channels-last images whose layers, activations and
gradients come from paper_2506_17974_b200.training, and whose weight gradients go through one LQ-SGD round per step.

    python examples/train_residual.py [--steps 30] [--workers 4] [--channels 64] [--blocks 2] [--rank 2] [--bits 4]

The network: 3x3 patches of an image -> linear stem -> blocks of  h + W2 gelu(W1 silu(norm(h)))  -> mean over the pixels ->
linear classifier.  Between the passes it keeps activations in 8 bits: the normalised one is packed once by the group norm
and handed to the linear layer that reads it.  Every simulated worker runs its own batch; the round averages the workers'
compressed gradients and updates the float32 weights in its last pass.  The data are drawn (ten fixed patterns, each
with a colour of its own, plus noise), so the loss has to fall."""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_17974_b200 import binding, training as tr  # noqa: E402

CLASSES = 10


class ResidualNet:
    """Weights in one list of float32 tensors, matrices out x in, in the order the round's layer table has."""

    def __init__(self, channels: int, blocks: int, groups: int, device: str, seed: int = 0):
        g = torch.Generator().manual_seed(seed)
        self.groups, self.blocks, c, hid = groups, blocks, channels, 4 * channels

        def matrix(out, inp, scale=1.0):
            return (torch.randn(out, inp, generator=g) * scale * inp ** -0.5).to(device)

        self.weights = [matrix(c, 27), torch.zeros(c, device=device)]
        for _ in range(blocks):
            self.weights += [torch.ones(c, device=device), torch.zeros(c, device=device), matrix(hid, c),
                             torch.zeros(hid, device=device), matrix(c, hid, 0.5), torch.zeros(c, device=device)]
        self.weights += [matrix(CLASSES, c), torch.zeros(CLASSES, device=device)]
        for w in self.weights:
            w.requires_grad_(True)

    def layers(self):
        return [(w.shape[0], w.shape[1] if w.dim() == 2 else 1) for w in self.weights]

    def forward(self, images: torch.Tensor) -> torch.Tensor:
        n, _, height, width = images.shape
        patches = F.unfold(images, 3, padding=1).transpose(1, 2).reshape(n * height * width, 27).contiguous()
        w = iter(self.weights)
        h = tr.linear_layer(patches, next(w), next(w))
        c = h.shape[1]
        for _ in range(self.blocks):
            kept = []
            a = tr.norm_layer(h.view(n, height * width, c), next(w), next(w), self.groups, act="silu", keep=kept)
            a = tr.linear_layer(a.view(-1, c), next(w), next(w), act="gelu", x8=kept[0])
            h = tr.linear_layer(a, next(w), next(w), residual=h)
        pooled = h.view(n, height * width, c).float().mean(1).to(h.dtype)
        return tr.linear_layer(pooled, next(w), next(w))


def train(steps: int = 30, workers: int = 4, channels: int = 64, blocks: int = 2, rank: int = 2, bits: int = 4, batch: int = 32,
          size: int = 8, lr: float = 0.1, device: str = "cuda:0", seed: int = 0):
    """Runs the steps and returns the mean loss over the workers at each of them."""
    net = ResidualNet(channels, blocks, groups=8, device=device, seed=seed)
    comp = binding.LQSGD(net.layers(), rank, bits, workers=workers, seed=seed, device=device)
    g = torch.Generator(device=device).manual_seed(seed)
    patterns = torch.randn(CLASSES, 3, size, size, generator=g, device=device) + torch.randn(CLASSES, 3, 1, 1, generator=g, device=device)
    losses = torch.zeros(steps, device=device)
    for step in range(steps):
        grads = []
        for _ in range(workers):
            label = torch.randint(CLASSES, (batch,), generator=g, device=device)
            images = patterns[label] + 0.5 * torch.randn(batch, 3, size, size, generator=g, device=device)
            loss = F.cross_entropy(net.forward(images.bfloat16()).float(), label)
            grads.append(torch.autograd.grad(loss, net.weights))
            losses[step] += loss.detach() / workers
        with torch.no_grad():
            comp.step_update(grads, None, net.weights, lr)
    if any(comp.status()) or tr.status(device):
        raise RuntimeError(f"a round or a layer reported a status: {comp.status()}, {tr.status(device)}")
    raw = 4 * sum(w.numel() for w in net.weights)
    return losses.tolist(), raw, comp.payload_nbytes


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("steps", 30), ("workers", 4), ("channels", 64), ("blocks", 2), ("rank", 2), ("bits", 4), ("batch", 32)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--lr", type=float, default=0.1)
    a = ap.parse_args()
    losses, raw, sent = train(a.steps, a.workers, a.channels, a.blocks, a.rank, a.bits, a.batch, lr=a.lr)
    for step in sorted({0, *range(0, a.steps, max(1, a.steps // 10)), a.steps - 1}):
        print(f"step {step:4d}  loss {losses[step]:.4f}")
    print(f"per worker and step: {raw} bytes of gradients, {sent} bytes sent")


if __name__ == "__main__":
    main()
