"""A learned reconstruction, trained through the projector, whose activations are kept in 8 bits.

    python examples/train_patch_network.py [--reduction 8] [--items 2] [--patch 8] [--hidden 512] [--blocks 2] [--rounds 2] [--steps 30]

Unrolled: every round takes a gradient step on |A x - y|^2 (`Projector` both ways, float32) and passes the volume through its own
stack of feed-forward blocks on patches (`activations.feed_forward8`, bfloat16 products, 8 bits kept).  The loss is the distance to
the phantom; float32 copies of the weights are what the optimizer works on.  Scans: the 512^3 cone-beam case, reduced.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2307_05801_amd import Projector  # noqa: E402
from paper_2307_05801_amd import activations as A  # noqa: E402
from synthetic import configs, phantoms  # noqa: E402


class Block(torch.nn.Module):
    """A feed-forward block on float32 weights, rounded to bfloat16 for each use."""

    def __init__(self, columns: int, hidden: int, device):
        super().__init__()
        self.norm = torch.nn.Parameter(torch.ones(columns, device=device))
        self.up = torch.nn.Parameter(torch.randn(2 * hidden, columns, device=device) / math.sqrt(columns))
        self.down = torch.nn.Parameter(torch.zeros(columns, hidden, device=device))          # at first the block changes nothing

    def forward(self, x, residual):
        return A.feed_forward8(x, self.norm, self.up.bfloat16(), self.down.bfloat16(), residual=residual)


class UnrolledNetwork(torch.nn.Module):
    def __init__(self, projector: Projector, patch: int, hidden: int, blocks: int, rounds: int, scale: float):
        super().__init__()
        self.projector, self.patch, self.scale = projector, patch, scale
        device = projector.geometry.device
        self.rounds = torch.nn.ModuleList(torch.nn.ModuleList(Block(patch ** 3, hidden, device) for _ in range(blocks)) for _ in range(rounds))
        self.step = torch.nn.Parameter(torch.full((rounds,), 0.5, device=device))
        # steps in units of what A^T A does to a constant volume
        one = torch.ones(projector.geometry.vol_shape, device=device)
        self.norm = float(projector.backproject(projector(one)).mean())

    def to_patches(self, x):
        p, (n, nz, ny, nx) = self.patch, x.shape
        return x.reshape(n, nz // p, p, ny // p, p, nx // p, p).permute(0, 1, 3, 5, 2, 4, 6).reshape(-1, p ** 3)

    def to_volume(self, rows, shape):
        p, (n, nz, ny, nx) = self.patch, shape
        return rows.reshape(n, nz // p, ny // p, nx // p, p, p, p).permute(0, 1, 4, 2, 5, 3, 6).reshape(shape)

    def forward(self, y):
        x = self.projector.backproject(y) / self.norm
        for step, blocks in zip(self.step, self.rounds):
            with A.keep_in_8_bits():                   # autograd keeps a volume here, for the gradient of `step`
                x = x - step / self.norm * self.projector.backproject(self.projector(x.contiguous()) - y)
            patches = self.to_patches(x / self.scale).bfloat16()
            rows, total = patches, None
            for block in blocks:
                rows, total = block(rows, total)
            # the volume itself stays float32: what the blocks add is theirs
            x = x + self.scale * self.to_volume(rows.float() + (total - patches).float(), x.shape)
        return x


def train(reduction=8, items=2, patch=8, hidden=512, blocks=2, rounds=2, steps=30, rate=5e-4, report=print):
    """The losses of `steps` steps."""
    torch.manual_seed(0)
    cfg = configs.reduced(configs.config(3), reduction)
    projector = Projector(cfg)
    truth = torch.stack([torch.as_tensor(phantoms.standard_volume(3, cfg, i), dtype=torch.float32) for i in range(items)]).cuda()
    y = projector(truth)
    scale = float(truth.std())
    network = UnrolledNetwork(projector, patch, hidden, blocks, rounds, scale)
    optimizer = torch.optim.Adam(network.parameters(), lr=rate)
    losses = []
    for step in range(steps):
        optimizer.zero_grad()
        torch.cuda.reset_peak_memory_stats()
        loss = ((network(y) - truth) / scale).square().mean()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
        if step % 5 == 0 or step == steps - 1:
            report(f"step {step}: loss {losses[-1]:.5f}, peak memory {torch.cuda.max_memory_allocated() / 2 ** 20:.0f} MiB")
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    for name, value in (("reduction", 8), ("items", 2), ("patch", 8), ("hidden", 512), ("blocks", 2), ("rounds", 2), ("steps", 30)):
        parser.add_argument("--" + name, type=int, default=value)
    train(**vars(parser.parse_args()))
