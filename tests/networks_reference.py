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


def rounding(t, dtype):
    """How far rounding float64 t to dtype may put it off: half a step, which below float16's least normal number, 2^-14, is 2^-25 whatever the value
    (steps there are 2^-24; the other types' are below 2^-126)."""
    return half_step(dtype) * t.abs() + (2.0 ** -25 if dtype is torch.float16 else 0.0)


def _slope(u, activation):
    s = torch.sigmoid(u)
    return s * (1 + u * (1 - s)) if activation == "silu" else (u > 0).double() if activation == "relu" else torch.ones_like(u)


class GroupNorm:
    """The values and bounds of one call: y, grad_x, grad_weight, grad_bias and the same names + "_off"; x [batch, ..., channels].

    A value's difference to the mean is off by the roundings of both, half a unit each, of the largest value's size, and the mean by what joining pieces adds: 2^-22 of the
    largest in all.  The variance's relative error is twice that of the differences, over the deviation, and the roundings of the sums (pieces of eight, a
    thread's few hundred, a block's).  sigmoid is good to (3 + |u|) 2^-24 or so, and its slope's slope is at most 1/2."""

    def __init__(self, x, groups, weight=None, bias=None, activation=None, eps=1e-5, grad=None):
        shape, dtype = x.shape, x.dtype
        batch, channels = shape[0], shape[-1]
        size, unit = channels // groups, 2.0 ** -24
        x = x.double().reshape(batch, -1, groups, size)
        voxels = x.shape[1]
        w, b = (torch.full((channels,), d, dtype=torch.float64) if t is None else t.double() for t, d in ((weight, 1.0), (bias, 0.0)))
        w, b = w.view(groups, size), b.view(groups, size)
        if voxels == 0 or batch == 0:
            self.y = self.grad_x = self.y_off = self.grad_x_off = torch.zeros(shape, dtype=torch.float64)
            self.grad_weight = self.grad_bias = self.grad_weight_off = self.grad_bias_off = torch.zeros(channels, dtype=torch.float64)
            return
        mean = x.mean((1, 3), keepdim=True)
        rstd = 1 / torch.sqrt((x - mean).square().mean((1, 3), keepdim=True) + eps)
        h = (x - mean) * rstd
        u = h * w + b
        s = torch.sigmoid(u)
        y = u * s if activation == "silu" else torch.relu(u) if activation == "relu" else u
        off_d = 4 * unit * x.abs().amax((1, 3), keepdim=True)
        off_r = off_d * rstd + sum_error(min(voxels, 512))
        off_h = off_d * rstd + h.abs() * (off_r + 4 * unit)
        off_u = w.abs() * off_h + 4 * unit * ((h * w).abs() + b.abs())
        near = (8 + u.abs()) * unit if activation == "silu" else 0.0
        self.y, self.y_off = y.reshape(shape), (1.1 * off_u + near * y.abs() + rounding(y, dtype)).reshape(shape)
        if grad is None:
            return
        g = grad.double().reshape(x.shape)
        du = g * _slope(u, activation)
        bend = 0.5 * off_u + near if activation == "silu" else (u.abs() <= off_u).double() if activation == "relu" else 0.0     # either side of relu's bend
        off_du = g.abs() * bend + 2 * unit * du.abs()
        parameter = dtype if weight is None and bias is None else (weight if weight is not None else bias).dtype
        many = sum_error(min(batch * voxels, 2048))
        one, two = du.sum((0, 1)), (du * h).sum((0, 1))
        off_one = (off_du + many * du.abs()).sum((0, 1))
        off_two = (off_du * h.abs() + du.abs() * off_h + many * (du * h).abs()).sum((0, 1))
        self.grad_bias, self.grad_bias_off = one.flatten(), (off_one + rounding(one, parameter)).flatten()
        self.grad_weight, self.grad_weight_off = two.flatten(), (off_two + rounding(two, parameter)).flatten()
        d = du * w
        first, second = d.mean((1, 3), keepdim=True), (d * h).mean((1, 3), keepdim=True)
        off_first = ((off_du + many * du.abs()) * w.abs()).mean((1, 3), keepdim=True)
        off_second = ((off_du * h.abs() + du.abs() * off_h + many * (du * h).abs()) * w.abs()).mean((1, 3), keepdim=True)
        grad_x = rstd * (d - first - h * second)
        size_ = d.abs() + first.abs() + (h * second).abs()
        off = rstd * (off_du * w.abs() + off_first + h.abs() * off_second + off_h * second.abs() + (8 * unit + off_r) * size_)
        self.grad_x, self.grad_x_off = grad_x.reshape(shape), (off + rounding(grad_x, dtype)).reshape(shape)
