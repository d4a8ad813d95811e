"""Operators for networks trained through the projector, beside those in 8 bits (`activations`): attention over patches, and group norm.

"PyTorch Interfaces and CT Parameters" puts the projector into a network's training loop.  Such a network cuts a volume into patches, the rows of
its blocks, or keeps voxels with their channels last:

    positions, buckets = relative_buckets((16, 16, 16), near=4, codes=6)             # places of a volume's patches, once
    o = attention(q, k, v, table=table, positions=positions, buckets=buckets)        # q, k, v: [batch, patches, heads, width]
    y = group_norm(x, 8, weight, bias, activation="silu")                            # x: [batch, nz, ny, nx, channels]
    norm = GroupNorm(8, 64, activation="silu"); y = norm(x)                          # the same as a module

Both are differentiable (backward; in forward mode they raise), run in libleap_hip.so on the current HIP stream, and take memory from PyTorch alone.  Tensors are on one GPU; the values of
a row (the last dimension) are neighbours (else ValueError: `.contiguous()` them).  The same call gives the same bits.
As with any operator, do not capture a backward pass into a graph while an eager graph of the same leaves is alive.
"""
from __future__ import annotations

import math
import struct

import torch

from . import binding as B
from .activations import _TYPES, _address, _call, _on_gpu, _records

BF16 = torch.bfloat16


def _bytes(t):
    """t's memory as autograd is to keep it: as bytes, which hooks that pack what is saved (activations.keep_in_8_bits) leave as they are.  Detached first: a
    view would hold its base, and an output that its graph.  Rows of one value may have any last stride (.contiguous() leaves it); as bytes they need one of 1."""
    if t is None:
        return None
    t = t.detach()
    return (t if t.stride(-1) == 1 else t.as_strided(t.shape, (*t.stride()[:-1], 1))).view(torch.uint8)


def _library():
    return B._activations or B.load_activations()


def _work(n: int, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


# ---- attention ----------------------------------------------------------------------------------------------------------

_DESC = struct.Struct("<18q5Qif")                             # leap_attention_desc


def _heads(t: torch.Tensor, what: str, device=None):
    """Checks a tensor [batch, rows, heads, width]."""
    _on_gpu(t, what, device)
    if t.dtype is not BF16 or t.dim() != 4 or not 1 <= t.shape[3] <= B.LEAP_ATTENTION_WIDEST:
        raise ValueError(f"{what} must be bfloat16 [batch, rows, heads, width], width at most {B.LEAP_ATTENTION_WIDEST}, got {t.dtype} {tuple(t.shape)}")
    if t.is_neg():
        raise ValueError(f"{what} is a negated view, whose memory holds other values; call .resolve_neg()")
    if t.stride(3) != 1 and t.shape[3] > 1:
        raise ValueError(f"{what}: the values of a row must be neighbours; call .contiguous()")


def _integers(t: torch.Tensor, n: int, device, what: str):
    _on_gpu(t, what, device)
    if t.dtype is not torch.int32 or t.dim() != 1 or not t.is_contiguous() or (n is not None and t.shape[0] != n) or t.is_neg():
        raise ValueError(f"{what} must be contiguous int32 [{'n' if n is None else n}] and no negated view, got {t.dtype} {tuple(t.shape)}")


def _description(q, k, v, mask, table, buckets, positions, scale):
    """leap_attention_desc of checked arguments, as bytes."""
    batch, queries, heads, width = q.shape
    _, keys, kv_heads, _ = k.shape
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    places = (None, None) if positions is None else positions
    return _DESC.pack(batch, queries, keys, heads, kv_heads, width, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                      0 if mask is None else mask.stride(0), 0 if table is None else buckets.shape[0], 0 if table is None else table.shape[1],
                      _address(mask) or 0, _address(table) or 0, _address(buckets) or 0, _address(places[0]) or 0, _address(places[1]) or 0,
                      0 if table is None else _TYPES[table.dtype], scale)


def _attend(q, k, v, mask, table, buckets, positions, scale, keep):
    """(o, the memory of its statistics and of what its rounding leaves)"""
    batch, queries, heads, width = q.shape
    device = q.device
    desc = _description(q, k, v, mask, table, buckets, positions, scale)
    o = torch.empty(q.shape, dtype=BF16, device=device)
    kept = stats = rest = None
    if keep:
        kept = torch.empty(batch * heads * queries * (8 + 2 * width), dtype=torch.uint8, device=device)
        stats = kept.data_ptr()
        rest = stats + batch * heads * queries * 8
    work = _work(_library().leap_attention_work(desc), device)
    _call("leap_attention", device, desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), stats, rest, _address(work))
    return o, kept


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, table, mask, buckets, places, scale):
        o, kept = _attend(q, k, v, mask, table, buckets, places, scale, True)
        # the probabilities are formed again from what made the statistics: nothing of it is packed
        ctx.save_for_backward(_bytes(q), _bytes(k), _bytes(v), _bytes(o), _bytes(table), kept, mask, buckets, *(places or (None, None)))
        ctx.scale, ctx.table_type = scale, None if table is None else table.dtype
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        q, k, v, o, table, kept, mask, buckets, *places = ctx.saved_tensors
        q, k, v, o = q.view(BF16), k.view(BF16), v.view(BF16), o.view(BF16)
        table = None if table is None else table.view(ctx.table_type)
        need_q, need_k, need_v, need_table = ctx.needs_input_grad[:4]
        device = q.device
        if grad.stride(3) != 1 or grad.is_neg():
            grad = grad.resolve_neg().contiguous()
        desc = _description(q, k, v, mask, table, buckets, places, ctx.scale)
        grad_q = torch.empty(q.shape, dtype=BF16, device=device) if need_q else None
        grad_k = torch.empty(k.shape, dtype=BF16, device=device) if need_k else None
        grad_v = torch.empty(v.shape, dtype=BF16, device=device) if need_v else None
        grad_table = torch.empty(table.shape, dtype=torch.float32, device=device) if need_table else None
        work = _work(_library().leap_attention_backward_work(desc, need_table), device)
        stats = kept.data_ptr()
        _call("leap_attention_backward", device, desc, grad.data_ptr(), *grad.stride()[:3], q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
              stats, stats + q.shape[0] * q.shape[1] * q.shape[2] * 8, _address(grad_q), _address(grad_k), _address(grad_v), _address(grad_table), _address(work))
        return grad_q, grad_k, grad_v, grad_table.to(ctx.table_type) if need_table else None, None, None, None, None


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, mask: torch.Tensor = None, table: torch.Tensor = None,
              buckets: torch.Tensor = None, positions=None, scale: float = None) -> torch.Tensor:
    """softmax(scale q k^T + bias) v over each item's keys, differentiable in q, k, v and table; bfloat16 [batch, queries, heads, width].

    q: bfloat16 [batch, queries, heads, width], width at most 128; k, v: [batch, keys, kv_heads, width], heads a multiple of kv_heads, whose keys and
    values neighbouring heads share.  mask: bool [batch, keys], True for keys that count (padded batches, patches outside the field of view); what is left out does
    not matter whatever it holds, and a query without keys has zeros.  scale: width ** -0.5 if not given.

    table: a learned number [heads, buckets] (float32, bfloat16, float16; at most 4096 buckets) for every head and bucket of relative positions, added to the scaled
    product.  positions: int32 [rows] of queries and keys alike, or a pair of them (None: 0, 1, 2, ...), within +-2^30; buckets: int32 [n], the bucket of
    key's position - query's position at index n // 2 + that, n at most 2^24 and 2^30 / heads; differences beyond its ends take the ends'.  relative_buckets makes both for a grid of
    patches.  -inf in the table leaves pairs out.

    Scores, the softmax and sums are 32 bits; probabilities and the gradients of scores are rounded to bfloat16 for the products that sum over them, but for
    the forward pass that a backward pass follows: there probabilities have 16 bits, with a table 24 (so o's last bits differ from those without one).  Kept for the
    backward pass: q, k, v and o, as they are also within keep_in_8_bits (the probabilities are formed again from what made them), 2 bytes more a value of
    o, and two floats a query and head."""
    _heads(q, "q")
    device = q.device
    _heads(k, "k", device)
    _heads(v, "v", device)
    batch, queries, heads, width = q.shape
    keys, kv_heads = k.shape[1], k.shape[2]
    if k.shape[0] != batch or k.shape[3] != width or v.shape != k.shape or kv_heads < 1 or heads < 1 or heads % kv_heads:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not fit: one batch and width, heads a multiple of k's and v's")
    if mask is not None:
        _on_gpu(mask, "mask", device)
        if mask.dtype is not torch.bool or mask.shape != (batch, keys):
            raise ValueError(f"mask must be bool {(batch, keys)}, got {mask.dtype} {tuple(mask.shape)}")
        if mask.stride(1) != 1 and keys > 1:
            raise ValueError("mask: the values of a row must be neighbours; call .contiguous()")
    if table is None:
        if buckets is not None or positions is not None:
            raise ValueError("buckets and positions are a table's")
    else:
        _on_gpu(table, "table", device)
        if table.dtype not in _TYPES or table.dim() != 2 or table.shape[0] != heads or not 1 <= table.shape[1] <= B.LEAP_ATTENTION_BUCKETS:
            raise ValueError(f"table must be [{heads}, buckets] of float32, bfloat16 or float16 with 1 to {B.LEAP_ATTENTION_BUCKETS} buckets, "
                             f"got {table.dtype} {tuple(table.shape)}")
        if not table.is_contiguous() or table.is_neg():
            raise ValueError("table must be contiguous")
        if buckets is None:
            raise ValueError("a table needs the buckets of differences of positions")
        _integers(buckets, None, device, "buckets")
        if buckets.shape[0] < 1:
            raise ValueError("buckets must not be empty")
        if positions is not None:
            positions = (positions, positions) if isinstance(positions, torch.Tensor) else tuple(positions)
            if len(positions) != 2:
                raise ValueError("positions: one tensor, or one of queries and one of keys")
            for t, n, what in ((positions[0], queries, "queries"), (positions[1], keys, "keys")):
                if t is not None:
                    _integers(t, n, device, f"positions of {what}")
    scale = width ** -0.5 if scale is None else float(scale)
    if not 0.0 < scale < 1e30:
        raise ValueError(f"scale must be positive, got {scale}")
    if _records(q, k, v, table):
        return _Attention.apply(q, k, v, table, mask, buckets, positions, scale)
    return _attend(q, k, v, mask, table, buckets, positions, scale, False)[0]


def relative_buckets(shape, near: int, codes: int, device="cuda:0"):
    """(positions, buckets), int32, for attention over the patches of a grid, in the order of its memory: shape (n,), (ny, nx), (nz, ny, nx).

    On an axis a distance d below `near` has the code d, those from near on one more for each doubling (near .. 2 near - 1: near, then near + 1, ...), and
    `codes` - 1 is the last; the two directions differ.  A bucket counts the axes' codes through, the last axis fastest: (2 codes - 1) ** axes in all.  At most 4096
    buckets and 2^24 differences ((2 nz - 1) (2 ny - 1) (2 nx - 1)), which is what attention takes."""
    sizes = tuple(int(n) for n in shape)
    if not sizes or any(n < 1 for n in sizes) or not 1 <= near <= codes:
        raise ValueError("a grid has axes of at least one patch, and 1 <= near <= codes")
    many = 2 * codes - 1
    if many ** len(sizes) > B.LEAP_ATTENTION_BUCKETS or math.prod(2 * n - 1 for n in sizes) > B.LEAP_ATTENTION_OFFSETS:
        raise ValueError(f"at most {B.LEAP_ATTENTION_BUCKETS} buckets and {B.LEAP_ATTENTION_OFFSETS} differences, got {many ** len(sizes)} and "
                         f"{math.prod(2 * n - 1 for n in sizes)}")
    positions, buckets = torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for n in sizes:
        code = [min(d if d < near else near + (d // near).bit_length() - 1, codes - 1) for d in range(n)]
        axis = torch.tensor([-c for c in code[:0:-1]] + code, dtype=torch.int32) + codes - 1
        positions = (positions[:, None] * (2 * n - 1) + torch.arange(n, dtype=torch.int32)).flatten()
        buckets = (buckets[:, None] * many + axis).flatten()
    return positions.to(device), buckets.to(device)


# ---- group norm ---------------------------------------------------------------------------------------------------------

_ACTIVATIONS = {None: B.LEAP_LINEAR, "relu": B.LEAP_RELU, "silu": B.LEAP_SILU}


def _voxels(t: torch.Tensor, what: str):
    """(voxels, distance of items, of voxels) of [batch, ..., channels]; ValueError where an item's voxels are not evenly spaced."""
    dims, strides, cols = t.shape, t.stride(), t.shape[-1]
    if t.is_neg():
        raise ValueError(f"{what} is a negated view, whose memory holds other values; call .resolve_neg()")
    if t.is_contiguous():
        voxels = math.prod(dims[1:-1])
        return voxels, voxels * cols, cols
    if strides[-1] == 1 or cols == 1:
        voxels, step = 1, None
        for n, s in zip(reversed(dims[1:-1]), reversed(strides[1:-1])):
            if n == 0:
                return 0, 0, cols
            if n > 1:
                if step is None:
                    step = s
                elif s != step * voxels:
                    break
                voxels *= n
        else:
            if step is None or step >= cols:
                return voxels, strides[0], cols if step is None else step
    raise ValueError(f"{what}: the channels of a voxel must be neighbours and an item's voxels evenly spaced; call .contiguous()")


def _norm_parameter(w, x, what: str):
    if w is not None:
        _on_gpu(w, what, x.device)
        if w.shape != (x.shape[-1],) or not w.is_contiguous() or w.is_neg() or (w.dtype is not torch.float32 and w.dtype is not x.dtype):
            raise ValueError(f"{what} must be contiguous [{x.shape[-1]}], float32 or {x.dtype}")


def _norm_forward(x, groups, weight, bias, activation, eps, keep):
    """(y, statistics)"""
    device, batch, channels = x.device, x.shape[0], x.shape[-1]
    voxels, item, row = _voxels(x, "x")
    y = torch.empty(x.shape, dtype=x.dtype, device=device)
    stats = torch.empty((batch, groups, 2), dtype=torch.float32, device=device) if keep else None
    work = _work(_library().leap_group_norm_work(batch, voxels, channels, groups), device)
    parameter = weight if weight is not None else bias
    _call("leap_group_norm", device, x.data_ptr(), _TYPES[x.dtype], item, row, _address(weight), _address(bias),
          B.LEAP_F32 if parameter is None else _TYPES[parameter.dtype], batch, voxels, channels, groups, eps, activation, y.data_ptr(), _address(stats), _address(work))
    return y, stats


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, activation, eps):
        y, stats = _norm_forward(x, groups, weight, bias, activation, eps, True)
        ctx.save_for_backward(x, weight, bias, _bytes(stats))          # hooks may pack x
        ctx.groups, ctx.activation = groups, activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, weight, bias, stats = ctx.saved_tensors
        need_x, need_weight, need_bias = ctx.needs_input_grad[:3]
        device, batch, channels = x.device, x.shape[0], x.shape[-1]
        try:
            _, grad_item, grad_row = _voxels(grad, "grad")
        except ValueError:
            grad = grad.resolve_neg().contiguous()
            _, grad_item, grad_row = _voxels(grad, "grad")
        voxels, item, row = _voxels(x, "x")
        grad_x = torch.empty(x.shape, dtype=x.dtype, device=device) if need_x else None
        grad_weight = torch.empty_like(weight) if need_weight else None
        grad_bias = torch.empty_like(bias) if need_bias else None
        work = _work(_library().leap_group_norm_backward_work(batch, voxels, channels, ctx.groups), device)
        parameter = weight if weight is not None else bias
        _call("leap_group_norm_backward", device, grad.data_ptr(), grad_item, grad_row, x.data_ptr(), _TYPES[x.dtype], item, row, _address(weight), _address(bias),
              B.LEAP_F32 if parameter is None else _TYPES[parameter.dtype], stats.data_ptr(), batch, voxels, channels, ctx.groups, ctx.activation, _address(grad_x),
              _address(grad_weight), _address(grad_bias), work.data_ptr())
        return grad_x, grad_weight, grad_bias, None, None, None


def group_norm(x: torch.Tensor, groups: int, weight: torch.Tensor = None, bias: torch.Tensor = None, activation: str = None, eps: float = 1e-5) -> torch.Tensor:
    """activation((x - mean) * rstd * weight + bias), differentiable in x, weight and bias; mean and rstd = 1 / sqrt(variance + eps) over an item's voxels and a
    group's channels.

    x: float32, bfloat16 or float16 [batch, ..., channels], channels last (a torch tensor in a channels-last memory format: x.movedim(1, -1)); groups divide the
    channels, each of neighbouring ones; weight, bias: [channels], x's type or float32, both of one type; activation: None, "relu" or "silu" (u * sigmoid(u)).
    Kept for the backward pass: x, which may be packed (activations.keep_in_8_bits: the gradients are then those of the values held), and two floats a group."""
    _on_gpu(x, "x")
    if x.dtype not in _TYPES or x.dim() < 2 or x.shape[-1] < 1:
        raise ValueError(f"x must be float32, bfloat16 or float16 [batch, ..., channels], got {x.dtype} {tuple(x.shape)}")
    if groups < 1 or x.shape[-1] % groups:
        raise ValueError(f"{groups} groups do not divide {x.shape[-1]} channels")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be None, 'relu' or 'silu', not {activation!r}")
    if not eps >= 0.0:
        raise ValueError(f"eps must not be negative, got {eps}")
    _norm_parameter(weight, x, "weight")
    _norm_parameter(bias, x, "bias")
    if weight is not None and bias is not None and weight.dtype is not bias.dtype:
        raise ValueError(f"weight and bias must be of one type, got {weight.dtype} and {bias.dtype}")
    if _records(x, weight, bias):
        return _GroupNorm.apply(x, weight, bias, groups, _ACTIVATIONS[activation], eps)
    return _norm_forward(x, groups, weight, bias, _ACTIVATIONS[activation], eps, False)[0]


class GroupNorm(torch.nn.Module):
    """group_norm with a weight and a bias of its own (float32)."""

    def __init__(self, groups: int, channels: int, activation: str = None, eps: float = 1e-5, device="cuda:0"):
        super().__init__()
        if groups < 1 or channels % groups:
            raise ValueError(f"{groups} groups do not divide {channels} channels")
        self.groups, self.activation, self.eps = groups, activation, eps
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(channels, device=device))

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return group_norm(x, self.groups, self.weight, self.bias, self.activation, self.eps)
