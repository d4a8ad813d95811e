"""Attention and group norm from their definitions, in 64 bits on the CPU, and how far a kernel may be off.

As in activations_reference.py a rounding counts half a step and a sum of n terms in 32 bits n * 2^-24 (no fewer than 64) times the sum
of their magnitudes.
"""
import torch

from activations_reference import half_step, sum_error

HALF = half_step(torch.bfloat16)


def bias_of(table, buckets, query_positions, key_positions):
    """[heads, queries, keys] of float64."""
    d = key_positions.long()[None, :] - query_positions.long()[:, None] + buckets.numel() // 2
    b = buckets.long()[d.clamp(0, buckets.numel() - 1)].clamp(0, table.shape[1] - 1)
    return table.double()[:, b], b


def attention(q, k, v, mask=None, bias=None, scale=None):
    """(o, x, p): o [batch, queries, heads, width], scores and probabilities [batch, heads, queries, keys], float64."""
    group = q.shape[2] // k.shape[2]
    q, k, v = (t.double().transpose(1, 2) for t in (q, k, v))
    if mask is not None:                                           # what is left out does not matter whatever it holds
        k, v = (torch.where(mask[:, None, :, None], t, 0.0) for t in (k, v))
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    x = q @ k.transpose(2, 3) * (q.shape[3] ** -0.5 if scale is None else scale)
    if bias is not None:
        x = x + bias
    if mask is not None:
        x = torch.where(mask[:, None, None, :], x, -torch.inf)
    if x.shape[3] == 0:
        return torch.zeros_like(q).transpose(1, 2), x, x
    most = x.amax(3, keepdim=True)
    e = torch.exp(x - torch.where(most == -torch.inf, 0.0, most))
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    return (p @ v).transpose(1, 2), x, p


class Attention:
    """The values and bounds of one call: o, grad_q, grad_k, grad_v, grad_table and the same names + "_off"."""

    def __init__(self, q, k, v, grad, mask=None, table=None, buckets=None, positions=None, scale=None, fine=True):
        batch, queries, heads, width = q.shape
        keys, kv_heads = k.shape[1], k.shape[2]
        group, scale = heads // kv_heads, width ** -0.5 if scale is None else scale
        bias = index = None
        if table is not None:
            qp, kp = positions if isinstance(positions, tuple) else (positions, positions)
            qp, kp = torch.arange(queries) if qp is None else qp, torch.arange(keys) if kp is None else kp
            bias, index = bias_of(table, buckets, qp, kp)
        self.o, x, p = attention(q, k, v, mask, bias, scale)
        if mask is not None:
            k, v = (torch.where(mask[:, :, None, None], t.double(), 0.0) for t in (k, v))
        wide = [t.double().transpose(1, 2) for t in (q, k, v, grad)]
        q, g = wide[0], wide[3]
        k, v = (t.repeat_interleave(group, 1) for t in wide[1:3])
        dp = g @ v.transpose(2, 3)
        delta = (p * dp).sum(3, keepdim=True)
        ds = p * (dp - delta)

        def back(t, shared=False):
            if shared:
                t = t.unflatten(1, (kv_heads, group)).sum(2)
            return t.transpose(1, 2)

        self.grad_q, self.grad_k = back(ds @ k) * scale, back(ds.transpose(2, 3) @ q, True) * scale
        self.grad_v = back(p.transpose(2, 3) @ g, True)

        # Scores: the product's sum, the scaling, the bias, the difference to the largest and the logarithm of the sum, each a rounding of 32 bits; the
        # exponential is good to 2^-22 of itself.  e: the relative error of a probability, that of the sum included.
        finite = torch.where(torch.isfinite(x), x.abs(), 0.0)
        off_x = scale * sum_error(width) * (q.abs() @ k.abs().transpose(2, 3)) + 8 * 2.0 ** -24 * (finite + finite.amax(3, keepdim=True) if keys else finite)
        if bias is not None:
            off_x = off_x + 4 * 2.0 ** -24 * torch.where(torch.isfinite(bias), bias.abs(), 0.0)
        e = off_x + ((p * off_x).sum(3, keepdim=True)) + sum_error(keys) + 2.0 ** -22
        off_p = p * e
        held = 2.0 ** -16 if fine else HALF                        # of a probability in the product, of o's own rounding
        off_o = (off_p + held * p) @ v.abs() + sum_error(keys) * (p @ v.abs())
        self.o_off = back(off_o) + HALF * self.o.abs()
        self.grad_v_off = back((off_p + HALF * p + sum_error(queries) * p).transpose(2, 3) @ g.abs(), True) + HALF * self.grad_v.abs()
        size = g.abs() @ v.abs().transpose(2, 3)
        off_delta = (g.abs() * (off_o + (2.0 ** -19 if fine else HALF) * back(self.o).abs())).sum(3, keepdim=True) + sum_error(width) * (p * size).sum(3, keepdim=True)
        off_ds = off_p * (dp - delta).abs() + p * (sum_error(width) * size + off_delta)
        self.grad_q_off = back((off_ds + (HALF + sum_error(keys)) * ds.abs()) @ k.abs()) * scale + HALF * self.grad_q.abs()
        self.grad_k_off = back((off_ds + (HALF + sum_error(queries)) * ds.abs()).transpose(2, 3) @ q.abs(), True) * scale + HALF * self.grad_k.abs()
        if table is not None:
            def by_bucket(t):
                return torch.zeros(table.shape, dtype=torch.float64).index_add_(1, index.flatten(), t.sum(0).flatten(1))
            self.grad_table = by_bucket(ds)
            # sums of a bucket's pairs: within a block in 32 bits, blocks in 64
            self.grad_table_off = by_bucket(off_ds + sum_error(queries + keys) * ds.abs()) + half_step(table.dtype) * self.grad_table.abs()
