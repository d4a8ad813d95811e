"""The operators on activations in 8 bits from their definitions, in 64 bits on the CPU, and how far a kernel may be off.

Roundings count half a step: half of torch.finfo(t).eps relative (2^-8 in bfloat16, 2^-11 in float16, 2^-24 in float32), 2^-4
for a code, and half of the smallest code's step below the normal codes.  A sum of n terms in 32 bits, whatever its order, is
off by at most n * 2^-24 times the sum of their magnitudes; no fewer than 64 terms are counted, for the few operations beside
the sum.
"""
import torch

GROUP = 32


def _code_values():
    v = torch.arange(127, dtype=torch.float64)                   # codes 0 .. 126: 0 .. 448
    e, m = torch.div(v, 8, rounding_mode="floor"), v % 8
    return torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7))


CODE_VALUES = _code_values()


def grouped(x):
    """[..., columns] as [..., groups, 32], zeros behind the end."""
    pad = -x.shape[-1] % GROUP
    return torch.nn.functional.pad(x, (0, pad)).reshape(*x.shape[:-1], -1, GROUP)


def scale_exponent(x):
    """e of each group of float64 x: the smallest integer >= -127 with amax <= 448 * 2^e."""
    amax = torch.where(torch.isfinite(grouped(x)), grouped(x).abs(), 0.0).amax(-1)
    e = torch.full_like(amax, -127.0)
    ok = amax > 0
    guess = torch.floor(torch.log2(amax[ok] / 448.0)) - 1
    for _ in range(3):                                           # a logarithm may be off by one
        guess = torch.where(amax[ok] > 448.0 * 2.0 ** guess, guess + 1, guess)
    e[ok] = guess.clamp(min=-127)
    return e


def pack(x):
    """(code bytes, scale bytes) of x, from the table of the codes' values: the nearest, the even one of two as near."""
    x = x.double()
    e = scale_exponent(x)
    y = grouped(x) / (2.0 ** e).unsqueeze(-1)
    y = y.reshape(*x.shape[:-1], -1)[..., :x.shape[-1]]
    a = y.abs().nan_to_num(nan=0.0, posinf=0.0)
    hi = torch.searchsorted(CODE_VALUES, a.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = (a - CODE_VALUES[lo]).abs(), (CODE_VALUES[hi] - a).abs()
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = torch.where(torch.isfinite(y), code, 127)
    sign = torch.where(torch.signbit(y), 128, 0)
    return (code + sign).to(torch.uint8), (e + 127).to(torch.uint8)


def values(codes, scales):
    """float64 values of code and scale bytes (uint8, CPU)."""
    c = codes.long()
    v = torch.cat([CODE_VALUES, torch.tensor([float("nan")], dtype=torch.float64)])[c % 128]
    v = torch.where(c >= 128, -v, v)
    power = (2.0 ** (scales.double() - 127)).repeat_interleave(GROUP, -1)[..., :codes.shape[-1]]
    return v * power


def held(p):
    """float64 values of a Packed8."""
    return values(p.codes.view(torch.uint8).cpu(), p.scales.cpu())


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def sum_error(n):
    return max(n, 64) * 2.0 ** -24


def assert_close(got, want, bound, what=""):
    """|got - want| <= bound elementwise; where `want` is not a number neither is `got`."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN in other places"
    off = torch.where(nan, 0.0, (got - want).abs() - bound)
    worst = off.argmax() if off.numel() else None
    assert not off.numel() or off.max() <= 0, f"{what}: {got.flatten()[worst]} for {want.flatten()[worst]}, bound {bound.flatten()[worst]}"


def assert_held(packed, want, error, what=""):
    """The values of a Packed8 against float64 `want`, itself known to within `error` in 32 bits: each is the nearest code of a
    number as near to it as that, on a scale that may be the next one where amax is as near to the border."""
    e = scale_exponent(want.abs() + error)
    step = (2.0 ** (e - 9)).repeat_interleave(GROUP, -1)[..., :want.shape[-1]]
    reach = want.abs() + error
    assert_close(held(packed), want, torch.maximum(reach * 2.0 ** -4, step / 2) + error, what)


def rms_norm(x, weight, residual, eps, dtype):
    """(sum, rstd, normed) of CPU tensors: sum as the type holds it, the rest float64."""
    s = x if residual is None else (x.float() + residual.float()).to(dtype)
    rstd = 1.0 / torch.sqrt(s.double().square().mean(-1) + eps)
    return s, rstd, s.double() * rstd.unsqueeze(-1) * weight.double()


def rms_norm_backward(grad, kept, rstd, weight, grad_sum):
    """(grad_x, its magnitude, grad_weight, its magnitude) from the values kept."""
    rstd = rstd.double().unsqueeze(-1)
    h, d = kept * rstd, grad.double() * weight.double()
    mean, size = (d * h).mean(-1, keepdim=True), (d * h).abs().mean(-1, keepdim=True)
    gs = torch.zeros_like(d) if grad_sum is None else grad_sum.double()
    flat = (grad.double() * h).reshape(-1, h.shape[-1])
    return gs + rstd * (d - h * mean), gs.abs() + rstd * (d.abs() + h.abs() * size), flat.sum(0), flat.abs().sum(0)


def gate(u):
    """(gated, its derivative's size with respect to u) of float64 u = (g, p)."""
    g, p = u.chunk(2, -1)
    s = torch.sigmoid(g)
    return g * s * p, (p.abs() * (s * (1 + g.abs() * (1 - s))) + (g * s).abs())


def gate_backward(da, kept):
    """(du, its magnitude) from the gradient of `gated` and the values kept [..., 2, outputs]."""
    g, p, da = kept[..., 0, :], kept[..., 1, :], da.double()
    s = torch.sigmoid(g)
    du = torch.cat([da * p * s * (1 + g * (1 - s)), da * g * s], -1)
    return du, torch.cat([(da * p * s).abs() * (1 + g.abs() * (1 - s)), (da * g * s).abs()], -1)
