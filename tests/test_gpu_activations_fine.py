"""Gradients through the gate with du held as the sum of two bfloat16, on the GPU against their definitions in 64 bits; and the choice to round it.

What is counted: 2^-17 of each of du's values for what two bfloat16 leave, 2^-18 of their magnitudes for the gate's arithmetic (as for du
in bfloat16), the sums in 32 bits over rows twice as long, and one rounding of the result, half a step.
"""
import pytest
import torch

import activations_reference as R
from test_gpu_activations import A, BF16, F32, _block, _offset, packed, rand, weight_of  # noqa: F401

pytestmark = pytest.mark.gpu

HELD = 2.0 ** -17 + 2.0 ** -18
# the gate's gradient by itself: odd sizes, rows that are padded, parts of long sums, tiles of every kind but the largest
GATED = [(1, 40, 3), (1, 64, 700), (70, 64, 33), (300, 96, 130), (513, 343, 205), (3000, 70, 260), (9000, 200, 264)]


@pytest.mark.parametrize("rows,cols,out", GATED)
def test_gradients_of_the_gated_product(A, rows, cols, out):  # noqa: F811
    x, v = packed(A, rand((rows, cols), F32, 201).double())
    w, g = weight_of(2 * out, cols, 202), rand((rows, out), BF16, 203)
    _, kept = A.gated_linear8(x, w.cuda())
    du, size = R.gate_backward(g, R.held(kept))
    wide = 5 if out % 2 else 0
    dx, dw = A.gated_linear8_backward(_offset(g, wide), kept, x, _offset(w, wide))
    wd = w.double()
    want, want_w = du @ wd, du.T @ v
    R.assert_close(dx, want, want.abs() * R.half_step(BF16) + (HELD + R.sum_error(4 * out)) * (size @ wd.abs()), "grad_x")
    R.assert_close(dw, want_w, want_w.abs() * R.half_step(BF16) + (HELD + R.sum_error(2 * rows)) * (size.T @ v.abs()), "grad_weight")
    rounded = A.gated_linear8_backward(g.cuda(), kept, x, w.cuda(), fine=False)
    assert rows < 70 or not torch.equal(rounded[0], dx)
    assert A.gated_linear8_backward(g.cuda(), kept, x, w.cuda(), need_weight=False)[1] is None
    none, again = A.gated_linear8_backward(_offset(g, wide), kept, x, _offset(w, wide), need_x=False)
    assert none is None and torch.equal(again, dw)


@pytest.mark.parametrize("rows,cols,hidden,out", [(1, 32, 32, 32), (130, 343, 70, 90), (200, 96, 130, 520), (5000, 64, 200, 64)])
def test_block(A, rows, cols, hidden, out):  # noqa: F811
    """From what the operators keep: the gradients of x (through the norm), of its weight and of up."""
    x, r, nw, up, _, _, gs = _block(rows, cols, hidden, seed=210)
    down, gy = weight_of(out, hidden, 218), rand((rows, out), BF16, 219)
    _, normed, kept_sum, rstd = A.rms_norm8(x.cuda(), nw.cuda(), r.cuda())
    kept = A.gated_linear8(normed, up.cuda())[1]
    leaves = [t.cuda().requires_grad_(True) for t in (x, nw, up, down, r)]
    y, s = A.feed_forward8(*leaves[:4], residual=leaves[4])
    dx, dnw, dup, ddown, dr = torch.autograd.grad((y, s), leaves, (gy.cuda(), gs.cuda()))
    u, da = R.held(kept), gy.double() @ down.double()
    du, size = R.gate_backward(da, u)
    error = HELD * size + R.gate_backward(R.sum_error(out) * (gy.double().abs() @ down.double().abs()), u)[1]
    v, upd = R.held(normed), up.double()
    want = du.T @ v
    R.assert_close(dup, want, want.abs() * R.half_step(BF16) + error.T @ v.abs() + R.sum_error(2 * rows) * (du.abs().T @ v.abs()), "grad_up")
    dn, dn_error = du @ upd, error @ upd.abs() + R.sum_error(4 * hidden) * (du.abs() @ upd.abs())
    h, rs = R.held(kept_sum), rstd.cpu()
    want, size, want_w, size_w = R.rms_norm_backward(dn, h, rs, nw, gs)
    _, through, _, through_w = R.rms_norm_backward(dn_error, h, rs, nw, None)
    R.assert_close(dx, want, want.abs() * R.half_step(BF16) + size * R.sum_error(cols) + through, "grad_x")
    R.assert_close(dnw, want_w, want_w.abs() * R.half_step(BF16) + size_w * R.sum_error(rows) + through_w, "grad_norm")
    assert torch.equal(dx, dr)
    plain = torch.autograd.grad(A.feed_forward8(*leaves[:4], residual=leaves[4], fine=False), leaves, (gy.cuda(), gs.cuda()))
    assert torch.equal(plain[3], ddown) and (rows == 1 or not torch.equal(plain[2], dup))


def test_infinities_and_nan_stay_what_they_are(A):  # noqa: F811
    """They reach what they reach through the rounded gradient, and nothing else: what becomes an infinity leaves nothing behind."""
    x, v = packed(A, rand((200, 64), F32, 220).double())
    w, g = weight_of(64, 64, 221), rand((200, 32), BF16, 222)
    _, kept = A.gated_linear8(x, w.cuda())
    g[7, 3], g[100, 0] = float("inf"), float("nan")
    one = torch.zeros_like(w)
    one[3, 5] = one[35, 6] = 1.0
    dx, _ = A.gated_linear8_backward(g.cuda(), kept, x, one.cuda(), need_weight=False)
    plain, _ = A.gated_linear8_backward(g.cuda(), kept, x, one.cuda(), need_weight=False, fine=False)
    assert torch.equal(torch.isnan(dx), torch.isnan(plain)) and torch.equal(torch.isinf(dx), torch.isinf(plain))


def test_module_and_no_rows(A):  # noqa: F811
    torch.manual_seed(4)
    block = A.FeedForward8(64, 43)
    x = rand((90, 64), BF16, 223).cuda().requires_grad_(True)
    y, s = block(x)
    got = torch.autograd.grad(y.float().square().sum(), [x, *block.parameters()])
    block.fine = False
    y, s = block(x)
    other = torch.autograd.grad(y.float().square().sum(), [x, *block.parameters()])
    assert all(torch.isfinite(g).all() for g in got) and torch.equal(got[3], other[3]) and not torch.equal(got[2], other[2])
    block.fine = True
    empty = torch.empty(0, 64, dtype=BF16, device="cuda", requires_grad=True)
    y, s = block(empty)
    grads = torch.autograd.grad((y, s), [empty, *block.parameters()], (torch.empty_like(y), torch.empty_like(s)))
    assert grads[0].shape == (0, 64) and not any(g.any() for g in grads[1:])


def test_graph_replays(A):  # noqa: F811
    x, v = packed(A, rand((300, 96), F32, 224).double())
    w, g = weight_of(140, 96, 225).cuda(), rand((300, 70), BF16, 226).cuda()
    _, kept = A.gated_linear8(x, w)
    step = lambda: A.gated_linear8_backward(g, kept, x, w)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(3):
        g.mul_(1.5 if k else 1.0)
        want = [t.clone() for t in step()]
        for t in captured:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, captured)), k


@pytest.mark.parametrize("rows,cols,out", [(1, 40, 3), (70, 64, 33), (300, 96, 130), (513, 343, 205)])
def test_rounded_gradients_are_those_of_their_parts(A, rows, cols, out):  # noqa: F811
    """fine=False: the same bits by one call and by two, whose du is a tensor of bfloat16; and for a block."""
    x, _ = packed(A, rand((rows, cols), F32, 227).double())
    w, g = weight_of(2 * out, cols, 228).cuda(), rand((rows, out), BF16, 229).cuda()
    _, kept = A.gated_linear8(x, w)
    du, fine = A.gate8_backward(g, kept, fine=False), A.gate8_backward(g, kept)
    assert du.dtype is BF16 and torch.equal(du, fine.rounded) and torch.equal(fine.float(), fine.rounded.float() + fine.rest.float())
    assert all(torch.equal(a, b) for a, b in zip(A.gated_linear8_backward(g, kept, x, w, fine=False), A.linear8_backward(du, x, w)))
    xs, r, nw, up, _, _, gs = (t.cuda() for t in _block(rows, cols, out, seed=230))
    down, gy = weight_of(64, out, 238).cuda(), rand((rows, 64), BF16, 239).cuda()
    _, normed, kept_sum, rstd = A.rms_norm8(xs, nw, r)
    _, kept = A.gated_linear8(normed, up)
    dn, dup = A.linear8_backward(A.linear_gate8_backward(gy, down, kept, fine=False), normed, up, dtype=F32)
    want = (*A.rms_norm8_backward(dn, kept_sum, rstd, nw, gs, BF16), dup)
    leaves = [t.detach().requires_grad_(True) for t in (xs, nw, up)]
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(A.feed_forward8(*leaves, down, residual=r, fine=False), leaves, (gy, gs)), want))


@pytest.mark.parametrize("rows,out,following", [(1, 40, 3), (3, 5, 700), (70, 33, 64), (300, 130, 96), (513, 205, 343)])
def test_a_fine_gradient(A, rows, out, following):  # noqa: F811
    """Its values, by either operator that makes one, and what it leaves between its rows."""
    kept, u = packed(A, rand((rows, 2, out), F32, 231).double())
    w, g = weight_of(following, out, 232), rand((rows, following), BF16, 233)
    da = (g.double() @ w.double()).to(BF16)
    for got, da, error in ((A.gate8_backward(da.cuda(), kept), da.double(), torch.zeros(rows, out)),
                           (A.linear_gate8_backward(g.cuda(), w.cuda(), kept), g.double() @ w.double(), R.sum_error(following) * (g.double().abs() @ w.double().abs()))):
        want, size = R.gate_backward(da, u)
        R.assert_close(got, want, HELD * size + R.gate_backward(error, u)[1] + torch.finfo(F32).smallest_normal, "du")
        # (a rest that rounds up to half a step makes a tie: the sum need not round to `rounded` again)
        assert bool((got.rest.float().abs() <= R.half_step(BF16) * got.rounded.float().abs()).all()) and got.rounded.shape == got.shape == (rows, 2 * out)
        assert not got.memory[..., 2 * out:].any()
    assert str((rows, 2 * out)) in repr(got) and got.device == kept.device


def test_fine_gradients_that_do_not_fit_are_refused(A):  # noqa: F811
    x, _ = packed(A, rand((4, 64), F32, 234).double())
    w = weight_of(16, 64, 235).cuda()
    for shape in ((4, 15), (3, 16), (2, 2, 16)):
        with pytest.raises(ValueError):
            A.linear8_backward(A.FineGradient(shape, "cuda"), x, w)
    with pytest.raises(ValueError):
        A.linear8_backward(A.FineGradient((4, 16), "cpu"), x, w)
