"""Operators for networks trained through the projector, with what the backward pass needs kept in 8 bits.

"PyTorch Interfaces and CT Parameters" puts the projector into a network's training loop, and every unrolled iteration keeps
volume-sized activations until its backward pass.  Here they are kept, and worked on, as 8-bit floats whose groups of 32
neighbours share a power of two: 1 + 1/32 bytes a value (include/leap_activations.h defines the format and the operators).

    packed = pack8(x); x_again = packed.unpack(torch.float32)          # any tensor, to 8 bits and back
    with keep_in_8_bits(): loss = network(volume)                      # what autograd saves inside is kept packed
    y, x = feed_forward8(y, norm_weight, up, down, residual=x)         # a block that keeps 8 bits only; differentiable
    block = FeedForward8(512, 1024); y, x = block(y, x)                # the same as a module

and its parts, forward and backward, for blocks of another make: rms_norm8, linear8, gated_linear8 and their *_backward.  The parts record no
gradients and refuse tensors that want one while autograd records: call them within torch.no_grad() or an autograd.Function.
A row is whatever the last dimension holds: a voxel's channels, a patch of a volume.

All run in libleap_hip.so on the current HIP stream; PyTorch supplies memory.  Tensors are on one GPU; the values of a row
are neighbours and the rows evenly spaced (else ValueError: `.contiguous()` them).  A rounding to 8 bits has the gradient 1.
As with any operator, do not capture a backward pass into a graph while an eager graph of the same leaves is alive.
"""
from __future__ import annotations

import torch

from . import binding as B
from .projector import _current_stream

GROUP = 32
_TYPES = {torch.float32: B.LEAP_F32, torch.bfloat16: B.LEAP_BF16, torch.float16: B.LEAP_F16}
_CODES = torch.float8_e4m3fn
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


class Packed8:
    """A tensor held in 8 bits: codes (float8_e4m3fn, its shape) and scales (uint8, one for each 32 values of a row: the
    power of two + 127)."""

    __slots__ = ("codes", "scales")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        if codes.dtype is not _CODES or scales.dtype is not torch.uint8:
            raise ValueError("codes are float8_e4m3fn, scales uint8")
        if codes.dim() < 1 or scales.shape != codes.shape[:-1] + (-(-codes.shape[-1] // GROUP),):
            raise ValueError(f"scales of shape {tuple(scales.shape)} do not fit codes of shape {tuple(codes.shape)}")
        if not codes.is_contiguous() or not scales.is_contiguous() or codes.device != scales.device:
            raise ValueError("codes and scales must be contiguous, on one device")
        self.codes, self.scales = codes, scales

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    def unpack(self, dtype: torch.dtype = torch.bfloat16, finite: bool = False) -> torch.Tensor:
        return unpack8(self, dtype, finite)

    def __repr__(self):
        return f"Packed8(shape={tuple(self.shape)}, device={self.device})"


class FineGradient:
    """A gradient as the sum of two tensors of bfloat16, to 2^-17 of a value: `rounded`, and `rest`, what the rounding leaves.  gate8_backward and
    linear_gate8_backward make it, linear8_backward takes it; float() and its like give a tensor."""

    __slots__ = ("memory", "shape")

    def __init__(self, shape, device):
        self.shape = torch.Size(shape)
        # both parts of a row side by side, each up to a multiple of 16 bytes (include/leap_activations.h)
        self.memory = torch.empty((*shape[:-1], 2, -(-shape[-1] // 8) * 8), dtype=torch.bfloat16, device=device)

    @property
    def device(self):
        return self.memory.device

    @property
    def rounded(self) -> torch.Tensor:
        return self.memory[..., 0, :self.shape[-1]]

    @property
    def rest(self) -> torch.Tensor:
        return self.memory[..., 1, :self.shape[-1]]

    def float(self) -> torch.Tensor:
        return self.rounded.float() + self.rest.float()

    def double(self) -> torch.Tensor:
        return self.float().double()

    def cpu(self) -> torch.Tensor:
        return self.float().cpu()

    def detach(self):
        return self                                           # it has no graph

    def __repr__(self):
        return f"FineGradient(shape={tuple(self.shape)}, device={self.device})"


def _not_recorded(*tensors) -> None:
    """The results have no graph: silently without one they would train with a part of the gradient."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("this operator records no gradient, and an argument requires one: use feed_forward8, call it within torch.no_grad() or an "
                                 "autograd.Function (with the *_backward operators), or hand it .detach()ed tensors")


def _type_of(t: torch.Tensor, what: str) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16, not {t.dtype}")
    return kind


def _on_gpu(t: torch.Tensor, what: str, device=None) -> None:
    if not t.is_cuda:
        raise ValueError(f"{what} must be on a GPU")
    if device is not None and t.device != device:
        raise ValueError(f"{what} must be on {device}")


def _rows(t: torch.Tensor, what: str):
    """(rows, columns, distance between rows) of a tensor whose last dimension is a row."""
    dims = t.shape
    if len(dims) == 0 or dims[-1] < 1:
        raise ValueError(f"{what} must have rows of at least one value")
    if t.is_neg():
        raise ValueError(f"{what} is a negated view, whose memory holds other values; call .resolve_neg()")
    cols = dims[-1]
    if t.is_contiguous():
        return t.numel() // cols, cols, cols
    strides = t.stride()
    if strides[-1] == 1 or cols == 1:
        rows, step = 1, None
        for n, s in zip(reversed(dims[:-1]), reversed(strides[:-1])):
            if n == 0:
                return 0, cols, cols
            if n == 1:
                continue
            if step is None:
                step = s
            elif s != step * rows:
                break
            rows *= n
        else:
            if step is None or step >= cols:
                return rows, cols, cols if step is None else step
    raise ValueError(f"{what}: the values of a row must be neighbours and the rows evenly spaced; call .contiguous()")


def _weight(w: torch.Tensor, cols: int, device, what: str = "weight"):
    """(rows, distance between them) of a bfloat16 weight [rows, cols]."""
    _on_gpu(w, what, device)
    if w.dtype is not torch.bfloat16 or w.dim() != 2 or w.shape[1] != cols or w.shape[0] < 1:
        raise ValueError(f"{what} must be bfloat16 [outputs, {cols}], got {w.dtype} {tuple(w.shape)}")
    rows, _, stride = _rows(w, what)
    return rows, stride


def _gradient(g: torch.Tensor, shape, device, types, what: str):
    _on_gpu(g, what, device)
    if g.shape != shape or g.dtype not in types:
        raise ValueError(f"{what} must be {' or '.join(str(t) for t in types)} {tuple(shape)}, got {g.dtype} {tuple(g.shape)}")
    return _rows(g, what)


def _call(name: str, device, *arguments) -> None:
    """The library's function on `device`, on its current stream."""
    lib = B._activations or B.load_activations()
    index = device.index
    if _current_device() == index:
        status = getattr(lib, name)(*arguments, _current_stream(index))
    else:
        with torch.cuda.device(index):
            status = getattr(lib, name)(*arguments, _current_stream(index))
    if status != B.LEAP_OK:
        B._check(lib, status)


def _empty_packed(shape, device) -> Packed8:
    p = Packed8.__new__(Packed8)
    p.codes = torch.empty(shape, dtype=_CODES, device=device)
    p.scales = torch.empty((*shape[:-1], -(-shape[-1] // GROUP)), dtype=torch.uint8, device=device)
    return p


_PLAIN = (torch.Tensor, torch.nn.Parameter)


def _like(t: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
    """A plain tensor without gaps of t's shape and device (empty_like takes 0.4 us less than empty, but keeps gaps and subclasses)."""
    if type(t) in _PLAIN and t.is_contiguous():
        return torch.empty_like(t, dtype=dtype)
    return torch.empty(t.shape, dtype=dtype, device=t.device)


def _packed_like(t: torch.Tensor) -> Packed8:
    p = Packed8.__new__(Packed8)
    p.codes = _like(t, _CODES)
    p.scales = torch.empty((*t.shape[:-1], -(-t.shape[-1] // GROUP)), dtype=torch.uint8, device=t.device)
    return p


def _work(name: str, device, *sizes):
    """Workspace of so many bytes as the library asks for, or None."""
    lib = B._activations or B.load_activations()
    n = getattr(lib, name)(*sizes)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _address(t):
    return None if t is None else t.data_ptr()


# ---- packing ------------------------------------------------------------------------------------------------------------


def pack8(x: torch.Tensor) -> Packed8:
    """x (float32, bfloat16, float16; [..., columns]) in 8 bits."""
    _not_recorded(x)
    _on_gpu(x, "x")
    kind = _type_of(x, "x")
    rows, cols, stride = _rows(x, "x")
    p = _packed_like(x)
    _call("leap_pack8", x.device, x.data_ptr(), kind, stride, rows, cols, p.codes.data_ptr(), p.scales.data_ptr())
    return p


def unpack8(packed: Packed8, dtype: torch.dtype = torch.bfloat16, finite: bool = False) -> torch.Tensor:
    """The values held; bfloat16 and float32 hold them exactly (but for 2^128, to which float32's largest numbers round and which is
    infinity there), float16 those between 2^-14 and 65504.  finite: what is beyond the type's largest number becomes that instead of an infinity."""
    kind = _TYPES.get(dtype)
    if kind is None:
        raise ValueError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
    codes = packed.codes
    _on_gpu(codes, "packed")
    rows, cols, _ = _rows(codes, "packed")
    out = _like(codes, dtype)
    _call("leap_unpack8_finite" if finite else "leap_unpack8", codes.device, codes.data_ptr(), packed.scales.data_ptr(), rows, cols, out.data_ptr(), kind)
    return out


_LONGEST = 1 << 20                                            # columns that the library takes
_PIECE = 1 << 15                                              # a row that the values of longer ones are cut into: whole groups


def _pack_flat(t: torch.Tensor):
    """The values of a tensor without gaps, whatever its shape, in rows of _PIECE and a last shorter one: [Packed8, ...]."""
    flat = t.view(-1)
    whole = flat.numel() // _PIECE * _PIECE
    return [pack8(part) for part in (flat[:whole].view(-1, _PIECE), flat[whole:]) if part.numel()]


def _unpack_flat(parts, shape, dtype: torch.dtype) -> torch.Tensor:
    out = torch.empty(shape, dtype=dtype, device=parts[0].device)
    to = out.data_ptr()
    for p in parts:
        rows, cols, _ = _rows(p.codes, "packed")
        _call("leap_unpack8_finite", p.device, p.codes.data_ptr(), p.scales.data_ptr(), rows, cols, to, _TYPES[dtype])
        to += rows * cols * dtype.itemsize
    return out


class keep_in_8_bits(torch.autograd.graph.saved_tensors_hooks):
    """Inside this context what autograd saves for the backward pass is kept packed: plain tensors on a GPU of float32, bfloat16 or
    float16 with at least `min_values` values and evenly spaced rows (no gaps, where they have more than 2^20 columns).  Leaves that want
    a gradient (weights) and everything else are kept as they are; a weight's cast or slice is no leaf: keep its use outside.  The
    gradients are those of the values held (3 mantissa bits).  What is finite stays so (a mask's lowest number too); infinities come back as NaN: operations that save a tensor masked with
    them (logsumexp of -inf) belong outside."""

    def __init__(self, min_values: int = 1 << 16):
        # What is kept as it is is kept detached: an output that its own operation saves would hold its graph, and that the output.
        # Autograd takes it back into the graph by itself, but leaves it to the hooks to notice that it was changed in place.
        def as_it_is(t):
            return t.detach(), t._version

        def pack(t):
            if (not t.is_cuda or t.dtype not in _TYPES or type(t) not in _PLAIN or t.layout is not torch.strided or t.is_nested or t.numel() < min_values
                    or (t.is_leaf and t.requires_grad)):
                return as_it_is(t)
            try:
                cols = _rows(t, "tensor")[1]
            except ValueError:
                return as_it_is(t)
            if cols <= _LONGEST:
                return pack8(t.detach()), t.dtype
            return (_pack_flat(t.detach()), (t.shape, t.dtype)) if t.is_contiguous() else as_it_is(t)

        def unpack(kept):
            held, known = kept
            if isinstance(held, Packed8):
                return held.unpack(known, finite=True)
            if isinstance(held, list):
                return _unpack_flat(held, *known)
            if held._version != known:
                raise RuntimeError(f"a tensor kept for the backward pass, {held.dtype} {tuple(held.shape)}, was changed in place (version {held._version}, "
                                   f"kept at {known})")
            return held

        super().__init__(pack, unpack)


# ---- the norm -----------------------------------------------------------------------------------------------------------


def rms_norm8(x: torch.Tensor, weight: torch.Tensor, residual: torch.Tensor = None, eps: float = 1e-6, keep: bool = True):
    """(sum, normed, kept, rstd): sum = x + residual (x itself without one), normed = packed sum * rstd * weight with rstd =
    1 / sqrt(mean(sum^2) + eps) over the row; kept = packed sum and rstd (float32) are for rms_norm8_backward (None with
    keep=False).  residual: x's type and shape; weight: [columns], x's type or float32."""
    _not_recorded(x, weight, residual)
    _on_gpu(x, "x")
    device, kind = x.device, _type_of(x, "x")
    rows, cols, stride = _rows(x, "x")
    if residual is not None:
        _, _, residual_stride = _gradient(residual, x.shape, device, (x.dtype,), "residual")
    _norm_weight(weight, x, cols)
    normed = _packed_like(x)
    total = x if residual is None else _like(x, x.dtype)
    kept = rstd = None
    if keep:
        kept = Packed8.__new__(Packed8)
        kept.codes, kept.scales = torch.empty_like(normed.codes), torch.empty_like(normed.scales)
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=device)
    _call("leap_rms_norm8", device, x.data_ptr(), stride, _address(residual), residual_stride if residual is not None else 0, kind,
          weight.data_ptr(), _TYPES[weight.dtype], rows, cols, eps, None if residual is None else total.data_ptr(), normed.codes.data_ptr(),
          normed.scales.data_ptr(), kept.codes.data_ptr() if keep else None, kept.scales.data_ptr() if keep else None, _address(rstd))
    return total, normed, kept, rstd


def _norm_weight(weight: torch.Tensor, x, cols: int) -> None:
    _on_gpu(weight, "weight", x.device)
    if weight.shape != (cols,) or not weight.is_contiguous() or weight.is_neg() or (weight.dtype is not torch.float32 and weight.dtype is not x.dtype):
        raise ValueError(f"weight must be contiguous [{cols}], float32 or {x.dtype}")


def rms_norm8_backward(grad: torch.Tensor, kept: Packed8, rstd: torch.Tensor, weight: torch.Tensor, grad_sum: torch.Tensor = None,
                       dtype: torch.dtype = None, need_weight: bool = True):
    """(grad_x, grad_weight or None if not needed) from the gradient of `normed` and, where there is one, of `sum`.  grad_x is the residual's gradient
    too, of type `dtype` (grad's if not given); grad: that type or float32."""
    _not_recorded(grad, grad_sum)
    dtype = grad.dtype if dtype is None else dtype
    if dtype not in _TYPES:
        raise ValueError(f"gradients are float32, bfloat16 or float16, not {dtype}")
    device = kept.device
    _on_gpu(kept.codes, "kept")
    rows, cols, stride = _gradient(grad, kept.shape, device, (dtype, torch.float32), "grad")
    sum_stride = 0 if grad_sum is None else _gradient(grad_sum, kept.shape, device, (dtype,), "grad_sum")[2]
    grad_x = _like(kept.codes, dtype)
    _norm_weight(weight, grad_x, cols)
    _on_gpu(rstd, "rstd", device)
    if rstd.shape != kept.shape[:-1] or rstd.dtype is not torch.float32 or not rstd.is_contiguous():
        raise ValueError(f"rstd must be contiguous float32 {tuple(kept.shape[:-1])}")
    grad_weight = work = None
    if need_weight:
        grad_weight = _like(weight, weight.dtype)
        lib = B._activations or B.load_activations()
        work = torch.empty(lib.leap_rms_norm8_work(rows, cols), dtype=torch.float32, device=device)
    _call("leap_rms_norm8_backward", device, grad.data_ptr(), _TYPES[grad.dtype], stride, _address(grad_sum), sum_stride, _TYPES[dtype],
          kept.codes.data_ptr(), kept.scales.data_ptr(), rstd.data_ptr(), weight.data_ptr(), _TYPES[weight.dtype], rows, cols,
          grad_x.data_ptr(), _address(grad_weight), _address(work))
    return grad_x, grad_weight


# ---- products -----------------------------------------------------------------------------------------------------------


def _packed_rows(x: Packed8, what: str = "x"):
    _on_gpu(x.codes, what)
    return _rows(x.codes, what)[:2]


def linear8(x: Packed8, weight: torch.Tensor) -> torch.Tensor:
    """x W^T, bfloat16 [..., outputs], from packed rows and a bfloat16 weight [outputs, columns]."""
    _not_recorded(weight)
    rows, cols = _packed_rows(x)
    out, w_stride = _weight(weight, cols, x.device)
    y = torch.empty(x.shape[:-1] + (out,), dtype=torch.bfloat16, device=x.device)
    work = _work("leap_linear8_work", x.device, x.codes.data_ptr(), rows, cols, weight.data_ptr(), w_stride, out)
    _call("leap_linear8", x.device, x.codes.data_ptr(), x.scales.data_ptr(), rows, cols, weight.data_ptr(), w_stride, out, y.data_ptr(), _address(work))
    return y


def linear8_backward(grad, x: Packed8, weight: torch.Tensor, need_x: bool = True, need_weight: bool = True,
                     dtype: torch.dtype = torch.bfloat16):
    """(grad_x, grad_weight): dy W (bfloat16, or float32 by `dtype`) and dy^T x (bfloat16); None for one that is not needed.
    grad: bfloat16, or a FineGradient, whose products take twice as long."""
    fine = type(grad) is FineGradient
    if not fine:
        _not_recorded(grad)
    rows, cols = _packed_rows(x)
    out, w_stride = _weight(weight, cols, x.device)
    if fine:
        if grad.shape != x.shape[:-1] + (out,) or grad.device != x.device:
            raise ValueError(f"grad {tuple(grad.shape)} is not of this x {tuple(x.shape)} and weight {tuple(weight.shape)}, or on another device")
    else:
        _, _, stride = _gradient(grad, x.shape[:-1] + (out,), x.device, (torch.bfloat16,), "grad")
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("grad_x is bfloat16 or float32")
    grad_x = _like(x.codes, dtype) if need_x else None
    grad_weight = _like(weight, torch.bfloat16) if need_weight else None
    name, dy = ("leap_linear8_backward_fine", ()) if fine else ("leap_linear8_backward", (stride,))
    address = grad.memory.data_ptr() if fine else grad.data_ptr()
    work = _work(name + "_work", x.device, *(() if fine else (address, stride)), x.codes.data_ptr(), rows, cols, weight.data_ptr(), w_stride, out)
    _call(name, x.device, address, *dy, x.codes.data_ptr(), x.scales.data_ptr(), rows, cols, weight.data_ptr(),
          w_stride, out, _address(grad_x), _TYPES[dtype], _address(grad_weight), _address(work))
    return grad_x, grad_weight


def _halves(weight: torch.Tensor, cols: int, device, what: str = "weight"):
    out, w_stride = _weight(weight, cols, device, what)
    if out % 2:
        raise ValueError(f"{what} must have twice as many rows as there are gated outputs, the gate's first; got {out}")
    return out // 2, w_stride


def gated_linear8(x: Packed8, weight: torch.Tensor, keep: bool = True):
    """(gated, kept): with u = x W^T = (g, p), W bfloat16 [2 * outputs, columns], gated = packed g * sigmoid(g) * p [...,
    outputs] and kept = packed u [..., 2, outputs] for the backward pass (None with keep=False).  u is 32 bits and never stored."""
    _not_recorded(weight)
    rows, cols = _packed_rows(x)
    out, w_stride = _halves(weight, cols, x.device)
    gated = _empty_packed(x.shape[:-1] + (out,), x.device)
    kept = _empty_packed(x.shape[:-1] + (2, out), x.device) if keep else None
    work = _work("leap_linear8_work", x.device, x.codes.data_ptr(), rows, cols, weight.data_ptr(), w_stride, 2 * out)
    _call("leap_gated_linear8", x.device, x.codes.data_ptr(), x.scales.data_ptr(), rows, cols, weight.data_ptr(), w_stride, out,
          gated.codes.data_ptr(), gated.scales.data_ptr(), kept.codes.data_ptr() if keep else None, kept.scales.data_ptr() if keep else None,
          _address(work))
    return gated, kept


def _kept_halves(kept: Packed8):
    _on_gpu(kept.codes, "kept")
    shape = kept.shape
    if len(shape) < 2 or shape[-2] != 2:
        raise ValueError(f"kept must be [..., 2, outputs], got {tuple(shape)}")
    return shape[:-2], shape[-1]


def _empty_du(shape, device, fine: bool):
    """(du, its address) to be written."""
    du = FineGradient(shape, device) if fine else torch.empty(shape, dtype=torch.bfloat16, device=device)
    return du, (du.memory if fine else du).data_ptr()


def gate8_backward(grad: torch.Tensor, kept: Packed8, fine: bool = True):
    """du [..., 2 * outputs], the gradient of gated_linear8's u, from that of `gated`: a FineGradient, or with fine=False rounded to bfloat16."""
    _not_recorded(grad)
    lead, out = _kept_halves(kept)
    rows, _, stride = _gradient(grad, lead + (out,), kept.device, (torch.bfloat16,), "grad")
    du, address = _empty_du(lead + (2 * out,), kept.device, fine)
    _call("leap_gate8_backward_fine" if fine else "leap_gate8_backward", kept.device, grad.data_ptr(), stride, kept.codes.data_ptr(), kept.scales.data_ptr(),
          rows, out, address)
    return du


def linear_gate8_backward(grad: torch.Tensor, weight: torch.Tensor, kept: Packed8, fine: bool = True):
    """gate8_backward of grad W, which stays in 32 bits: du from the gradient of the product linear8(gated, weight)."""
    _not_recorded(grad)
    lead, out = _kept_halves(kept)
    following, w_stride = _weight(weight, out, kept.device)
    rows, _, stride = _gradient(grad, lead + (following,), kept.device, (torch.bfloat16,), "grad")
    du, address = _empty_du(lead + (2 * out,), kept.device, fine)
    work = _work("leap_linear_gate8_work", kept.device, grad.data_ptr(), stride, weight.data_ptr(), w_stride, following, rows, out)
    _call("leap_linear_gate8_backward_fine" if fine else "leap_linear_gate8_backward", kept.device, grad.data_ptr(), stride, weight.data_ptr(), w_stride,
          following, kept.codes.data_ptr(), kept.scales.data_ptr(), rows, out, address, _address(work))
    return du


def gated_linear8_backward(grad: torch.Tensor, kept: Packed8, x: Packed8, weight: torch.Tensor, need_x: bool = True, need_weight: bool = True,
                           fine: bool = True):
    """(grad_x, grad_weight) of gated_linear8 from the gradient of `gated` (bfloat16).  In between is du, the gradient of u, a FineGradient, so that
    the results' rounding is the only one (0.0017 of their norm); with fine=False it is bfloat16 (0.0024), which the products take in half the time."""
    _not_recorded(grad)
    if kept.shape[:-2] != x.shape[:-1]:
        raise ValueError(f"kept {tuple(kept.shape)} is not of this x {tuple(x.shape)}")
    lead, out = _kept_halves(kept)
    rows, cols = _packed_rows(x)
    halves, w_stride = _halves(weight, cols, x.device)
    if halves != out or kept.device != x.device:
        raise ValueError(f"kept {tuple(kept.shape)} is not of this weight {tuple(weight.shape)}, or on another device")
    stride = _gradient(grad, lead + (out,), x.device, (torch.bfloat16,), "grad")[2]
    grad_x = _like(x.codes, torch.bfloat16) if need_x else None
    grad_weight = _like(weight, torch.bfloat16) if need_weight else None
    name = "leap_gated_linear8_backward_fine" if fine else "leap_gated_linear8_backward"
    work = _work(name + "_work", x.device, x.codes.data_ptr(), rows, cols, weight.data_ptr(), w_stride, out)
    _call(name, x.device, grad.data_ptr(), stride, kept.codes.data_ptr(), kept.scales.data_ptr(), x.codes.data_ptr(), x.scales.data_ptr(),
          rows, cols, weight.data_ptr(), w_stride, out, _address(grad_x), B.LEAP_BF16, _address(grad_weight), _address(work))
    return grad_x, grad_weight


# ---- the block ----------------------------------------------------------------------------------------------------------


def _block_forward(x, residual, norm_weight, up, down, eps, keep):
    """(y, sum, kept, (rows, columns, hidden, outputs)); kept None where there is nothing to keep it for."""
    device = x.device
    rows, cols, stride = _rows(x, "x")
    residual_stride = 0 if residual is None else _gradient(residual, x.shape, device, (x.dtype,), "residual")[2]
    _norm_weight(norm_weight, x, cols)
    hidden, up_stride = _halves(up, cols, device, "up")
    out, down_stride = _weight(down, hidden, device, "down")
    total = None if residual is None else _like(x, x.dtype)
    y = torch.empty(x.shape[:-1] + (out,), dtype=x.dtype, device=device)
    weights = (up.data_ptr(), up_stride, hidden, down.data_ptr(), down_stride, out)
    name, kept = "leap_feed_forward8" if keep else "leap_feed_forward8_alone", None
    if keep:
        lib = B._activations or B.load_activations()
        kept = torch.empty(lib.leap_feed_forward8_kept(rows, cols, hidden), dtype=torch.uint8, device=device)
    work = _work(name + "_work", device, rows, cols, *weights)
    _call(name, device, x.data_ptr(), stride, _address(residual), residual_stride, norm_weight.data_ptr(), _TYPES[norm_weight.dtype], rows, cols, eps,
          *weights, _address(total), y.data_ptr(), *((kept.data_ptr(),) if keep else ()), _address(work))
    # without a residual a tensor apart from its input: autograd would take it for a view
    return y, x.view_as(x) if total is None else total, kept, (rows, cols, hidden, out)


class _FeedForward8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, norm_weight, up, down, eps, fine):
        y, total, kept, sizes = _block_forward(x, residual, norm_weight, up, down, eps, True)
        ctx.save_for_backward(norm_weight, up, down, kept)
        ctx.set_materialize_grads(False)
        ctx.added, ctx.shape, ctx.sizes, ctx.fine = residual is not None, x.shape, sizes, fine
        return y, total

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_y, grad_sum):
        if grad_y is None:
            return grad_sum, grad_sum if ctx.added else None, None, None, None, None, None
        norm_weight, up, down, kept = ctx.saved_tensors
        rows, cols, hidden, out = ctx.sizes
        need_x, need_r, need_norm, need_up, need_down = ctx.needs_input_grad[:5]
        device = kept.device
        # hooks on saved tensors may have laid the weights out anew
        up_stride, down_stride = _weight(up, cols, device, "up")[1], _weight(down, hidden, device, "down")[1]
        grad_y = grad_y.contiguous()
        grad_sum = None if grad_sum is None else grad_sum.contiguous()
        grad_x = torch.empty(ctx.shape, dtype=torch.bfloat16, device=device) if need_x or need_r or need_norm else None
        grad_norm = _like(norm_weight, norm_weight.dtype) if need_norm else None
        grad_up = _like(up, torch.bfloat16) if need_up else None
        grad_down = _like(down, torch.bfloat16) if need_down else None
        weights = (up.data_ptr(), up_stride, hidden, down.data_ptr(), down_stride, out)
        name = "leap_feed_forward8_backward_fine" if ctx.fine else "leap_feed_forward8_backward"
        work = _work(name + "_work", device, grad_y.data_ptr(), out, rows, cols, *weights)
        _call(name, device, grad_y.data_ptr(), out, _address(grad_sum), cols, norm_weight.data_ptr(), _TYPES[norm_weight.dtype],
              rows, cols, *weights, kept.data_ptr(), _address(grad_x), _address(grad_norm), _address(grad_up), _address(grad_down), _address(work))
        return grad_x if need_x else None, grad_x if need_r else None, grad_norm, grad_up, grad_down, None, None


def feed_forward8(x: torch.Tensor, norm_weight: torch.Tensor, up: torch.Tensor, down: torch.Tensor, residual: torch.Tensor = None,
                  eps: float = 1e-6, fine: bool = True):
    """(y, sum), differentiable: sum = x + residual and y = linear8(gated_linear8(rms_norm8(sum), up), down).  x, residual: bfloat16
    [..., columns]; up: [2 * hidden, columns], the gate's rows first; down: [outputs, hidden].  For a stack of blocks y and sum are the next one's
    x and residual.  Kept for the backward pass, if there is one to come: the norm's output, sum and the hidden rows (three times), all in 8 bits.
    fine=False: the gradient of up's product is rounded to bfloat16 on its way to the gradients of x, norm_weight and up, whose products then take half
    the time (gated_linear8_backward says how far off they are)."""
    _on_gpu(x, "x")
    if x.dtype is not torch.bfloat16:
        raise ValueError(f"x must be bfloat16, not {x.dtype}")
    tensors = (x, residual, norm_weight, up, down)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        return _FeedForward8.apply(*tensors, eps, fine)
    return _block_forward(*tensors, eps, False)[:2]


class FeedForward8(torch.nn.Module):
    """feed_forward8 with weights of its own (bfloat16): (x, residual) -> (y, sum)."""

    def __init__(self, columns: int, hidden: int, eps: float = 1e-6, device="cuda:0", fine: bool = True):
        super().__init__()
        self.eps, self.fine = eps, fine
        self.norm_weight = torch.nn.Parameter(torch.ones(columns, dtype=torch.bfloat16, device=device))
        self.up = torch.nn.Parameter((torch.randn(2 * hidden, columns, device=device) / columns ** 0.5).to(torch.bfloat16))
        self.down = torch.nn.Parameter((torch.randn(columns, hidden, device=device) / hidden ** 0.5).to(torch.bfloat16))

    def forward(self, x: torch.Tensor, residual: torch.Tensor = None):
        return feed_forward8(x, self.norm_weight, self.up, self.down, residual, self.eps, self.fine)
