"""A learned reconstruction, trained through the projector, whose activations are kept in 8 bits.

    python examples/train_patch_network.py [--reduction 8] [--items 2] [--patch 8] [--hidden 512] [--blocks 2] [--rounds 2] [--steps 30] [--heads 0]

Unrolled: every round takes a gradient step on |A x - y|^2 (`Projector` both ways, float32) and passes the volume through its own
stack of feed-forward blocks on patches (`activations.feed_forward8`, bfloat16 products, 8 bits kept), with --heads after attention over all of
an item's patches (`networks.group_norm` and `networks.attention`, with a learned number for every bucket of relative positions).  The loss is the distance to
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
from paper_2307_05801_amd import networks as N  # noqa: E402
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


class Attention(torch.nn.Module):
    """What attention over the patches of a grid adds to them: float32 weights, rounded to bfloat16 for each use."""

    def __init__(self, columns: int, heads: int, grid, device):
        super().__init__()
        near, codes = 2, 5                                     # distances 0, 1, 2 - 3, 4 - 7, 8 and more, either way on each axis
        self.heads = heads
        self.norm = N.GroupNorm(1, columns, device=device)
        self.inputs = torch.nn.Parameter(torch.randn(3 * columns, columns, device=device) / math.sqrt(columns))
        self.output = torch.nn.Parameter(torch.zeros(columns, columns, device=device))           # at first nothing is added
        self.table = torch.nn.Parameter(torch.zeros(heads, (2 * codes - 1) ** len(grid), device=device))
        positions, buckets = N.relative_buckets(grid, near, codes, device=device)
        self.register_buffer("positions", positions)
        self.register_buffer("buckets", buckets)

    def forward(self, x):
        q, k, v = torch.nn.functional.linear(self.norm(x), self.inputs.bfloat16()).unflatten(2, (3, self.heads, -1)).unbind(2)
        o = N.attention(q, k, v, table=self.table, buckets=self.buckets, positions=self.positions)
        return torch.nn.functional.linear(o.flatten(2), self.output.bfloat16())


class UnrolledNetwork(torch.nn.Module):
    def __init__(self, projector: Projector, patch: int, hidden: int, blocks: int, rounds: int, scale: float, heads: int = 0):
        super().__init__()
        self.projector, self.patch, self.scale = projector, patch, scale
        device = projector.geometry.device
        self.rounds = torch.nn.ModuleList(torch.nn.ModuleList(Block(patch ** 3, hidden, device) for _ in range(blocks)) for _ in range(rounds))
        self.step = torch.nn.Parameter(torch.full((rounds,), 0.5, device=device))
        grid = tuple(n // patch for n in projector.geometry.vol_shape)
        self.attention = torch.nn.ModuleList(Attention(patch ** 3, heads, grid, device) for _ in range(rounds)) if heads else [None] * rounds
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
        for step, attention, blocks in zip(self.step, self.attention, self.rounds):
            with A.keep_in_8_bits():                   # autograd keeps a volume here, for the gradient of `step`
                x = x - step / self.norm * self.projector.backproject(self.projector(x.contiguous()) - y)
            patches = self.to_patches(x / self.scale).bfloat16()
            rows, total = patches, None
            if attention is not None:
                rows = patches + attention(patches.unflatten(0, (len(x), -1))).flatten(0, 1)
            for block in blocks:
                rows, total = block(rows, total)
            # the volume itself stays float32: what the blocks add is theirs
            x = x + self.scale * self.to_volume(rows.float() + (total - patches).float(), x.shape)
        return x


def train(reduction=8, items=2, patch=8, hidden=512, blocks=2, rounds=2, steps=30, rate=5e-4, report=print, heads=0):
    """The losses of `steps` steps."""
    torch.manual_seed(0)
    cfg = configs.reduced(configs.config(3), reduction)
    projector = Projector(cfg)
    truth = torch.stack([torch.as_tensor(phantoms.standard_volume(3, cfg, i), dtype=torch.float32) for i in range(items)]).cuda()
    y = projector(truth)
    scale = float(truth.std())
    network = UnrolledNetwork(projector, patch, hidden, blocks, rounds, scale, heads)
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
    for name, value in (("reduction", 8), ("items", 2), ("patch", 8), ("hidden", 512), ("blocks", 2), ("rounds", 2), ("steps", 30), ("heads", 0)):
        parser.add_argument("--" + name, type=int, default=value)
    train(**vars(parser.parse_args()))
