"""Every kernel of the products, at the sizes of activation_kernels.py, against 64 bits; what goes past the caches.

The operands are small whole numbers times powers of two, so that 32 bits hold every partial sum exactly, whatever its order: sums over
thousands of values are compared bit by bit, and one that is missing or taken twice shows.  What is no sum has the bounds of
activations_reference.py.  Computed on the GPU, in float64."""
import pytest
import torch

import activation_kernels as K
import activations_reference as R
from test_gpu_activations import A, BF16, F32  # noqa: F401

pytestmark = pytest.mark.gpu


def whole(shape, top, seed):
    return torch.randint(-top, top + 1, shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).float()


def packed(A, rows, cols, seed):  # noqa: F811
    """(Packed8, its values in 64 bits): -2 .. 2 times 1, 2 or 4 by groups of 32."""
    power = 2.0 ** (whole((rows, -(-cols // 32)), 1, seed + 1) + 1)
    v = whole((rows, cols), 2, seed) * power.repeat_interleave(32, 1)[:, :cols]
    x = A.pack8(v)
    assert torch.equal(x.unpack(F32), v)
    return x, v.double()


def weight(rows, cols, seed):
    w = (whole((rows, cols), 3, seed) / 128).to(BF16)
    return w, w.double()


def gradient(rows, cols, seed):
    g = whole((rows, cols), 3, seed).to(BF16)
    return g, g.double()


def near(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    assert not torch.isnan(off).any() and float(off.max()) <= 0, (what, float(off.max()), int(off.argmax()))


def cases(*what):
    some = [c for c in K.CASES if c[0] in what]
    return pytest.mark.parametrize("what,rows,cols,out", [c[:4] for c in some], ids=["-".join(map(str, c[:4] + c[4][3:])) for c in some])


@cases(K.Y)
def test_y(A, what, rows, cols, out):  # noqa: F811
    (x, v), (w, wd) = packed(A, rows, cols, 401), weight(out, cols, 403)
    assert torch.equal(A.linear8(x, w), (v @ wd.T).to(BF16))


@cases(K.GRAD_X, K.GRAD_X_FULL, K.GRAD_WEIGHT)
def test_gradients(A, what, rows, cols, out):  # noqa: F811
    (x, v), (w, wd), (g, gd) = packed(A, rows, cols, 405), weight(out, cols, 407), gradient(rows, out, 408)
    if what == K.GRAD_WEIGHT:
        assert torch.equal(A.linear8_backward(g, x, w, need_x=False)[1], (gd.T @ v).to(BF16))
    else:
        kind = F32 if what == K.GRAD_X_FULL else BF16
        assert torch.equal(A.linear8_backward(g, x, w, need_weight=False, dtype=kind)[0], (gd @ wd).to(kind))


@cases(K.GATED)
def test_gated(A, what, rows, cols, out):  # noqa: F811
    (x, v), (w, wd) = packed(A, rows, cols, 409), weight(2 * out, cols, 411)
    gated, kept = A.gated_linear8(x, w)
    u = v @ wd.T
    want = A.pack8(u.float().reshape(rows, 2, out))
    assert torch.equal(kept.scales, want.scales) and torch.equal(kept.unpack(F32), want.unpack(F32))
    a = R.gate(u)[0]
    error = 2.0 ** -18 * a.abs() + 1e-30
    step = (2.0 ** (R.scale_exponent(a.abs() + error) - 9)).repeat_interleave(32, 1)[:, :out]
    near(gated.unpack(F32), a, torch.maximum((a.abs() + error) * 2.0 ** -4, step / 2) + error, "gated")
    again, none = A.gated_linear8(x, w, keep=False)
    assert none is None and torch.equal(again.codes.view(torch.uint8), gated.codes.view(torch.uint8)) and torch.equal(again.scales, gated.scales)


def halves(A, rows, out, seed):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(seed)
    kept = A.pack8(torch.randn(rows, 2, out, device="cuda", generator=g) * torch.exp(torch.randn(rows, 1, 1, device="cuda", generator=g)))
    return kept, kept.unpack(F32).double()


@cases(K.GATE_GRAD, K.GATE_GRAD_FINE)
def test_gradient_through_the_gate(A, what, rows, cols, out):  # noqa: F811
    (kept, u), (w, wd), (g, gd) = halves(A, rows, cols, 413), weight(out, cols, 414), gradient(rows, out, 415)
    du, size = R.gate_backward(gd @ wd, u)
    fine = what == K.GATE_GRAD_FINE
    got = A.linear_gate8_backward(g, w, kept, fine=fine)
    near(got, du, du.abs() * (2.0 ** -17 if fine else R.half_step(BF16)) + 2.0 ** -18 * size + torch.finfo(F32).smallest_normal, "du")
    assert not fine or not got.memory[..., 2 * cols:].any()


@pytest.mark.parametrize("rows,cols,out", [(33000, 1030, 1100), (3001, 72, 700), (18414, 343, 1029)])
def test_gradients_from_a_fine_one(A, rows, cols, out):  # noqa: F811
    """dy of 11 bits, which takes both of its parts; sums, of values of either sign, are whole numbers of no more than 24."""
    (x, v), (w, wd) = packed(A, rows, cols, 431), weight(out, cols, 433)
    dy = whole((rows, out), 2047, 434)
    grad = A.FineGradient((rows, out), "cuda")
    grad.memory.zero_()
    grad.rounded.copy_(dy)
    grad.rest.copy_(dy - grad.rounded.float())
    assert torch.equal(grad.float(), dy)
    dx, dw = A.linear8_backward(grad, x, w, dtype=F32)
    assert torch.equal(dx, (dy.double() @ wd).float())
    assert torch.equal(dw, (dy.double().T @ v).to(BF16))


def test_norm_past_the_caches(A):  # noqa: F811
    """More than 64 MiB of outputs: the same bits as of its rows in two parts, both ways."""
    rows, cols = 70001, 520
    g = torch.Generator(device="cuda").manual_seed(421)
    x, r, gs = (torch.randn(rows, cols, device="cuda", generator=g).to(BF16) for _ in range(3))
    w = (1 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(BF16)
    whole_ones = A.rms_norm8(x, w, r)
    dx, _ = A.rms_norm8_backward(r, whole_ones[2], whole_ones[3], w, gs)
    for part in (slice(0, 40000), slice(40000, rows)):
        total, normed, kept, rstd = A.rms_norm8(x[part], w, r[part])
        assert torch.equal(whole_ones[0][part], total) and torch.equal(whole_ones[3][part], rstd)
        for a, b in ((whole_ones[1], normed), (whole_ones[2], kept)):
            assert torch.equal(a.codes[part].view(torch.uint8), b.codes.view(torch.uint8)) and torch.equal(a.scales[part], b.scales)
        assert torch.equal(dx[part], A.rms_norm8_backward(r[part], kept, rstd, w, gs[part])[0])


def test_gate_gradient_past_the_caches(A):  # noqa: F811
    """du of more than 192 MiB, by itself; rounded, and fine through the products behind it."""
    rows, out = 50003, 1029
    (kept, u), (g, gd) = halves(A, rows, out, 423), gradient(rows, out, 424)
    du, size = R.gate_backward(gd, u)
    near(A.gate8_backward(g, kept, fine=False), du, du.abs() * R.half_step(BF16) + 2.0 ** -18 * size + torch.finfo(F32).smallest_normal, "du")
    (x, _), (w, wd) = packed(A, rows, 40, 425), weight(2 * out, 40, 427)
    for fine, held in ((False, R.half_step(BF16)), (True, 2.0 ** -17)):
        dx, _ = A.gated_linear8_backward(g, kept, x, w, need_weight=False, fine=fine)
        want = du @ wd
        near(dx, want, want.abs() * R.half_step(BF16) + (held + 2.0 ** -18 + R.sum_error(4 * out)) * (size @ wd.abs()), f"grad_x {fine}")
