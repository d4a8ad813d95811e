"""Operators on activations in 8 bits on the GPU, at the edges of what they take: no rows, many rows, tensors that autograd saves."""
import gc

import pytest
import torch

import activations_reference as R  # noqa: F401
from test_gpu_activations import A, BF16, F32, _block, weight_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fine", [False, True])
@pytest.mark.parametrize("cols,out", [(96, 32), (343, 8), (343, 21), (64, 21)])
def test_gradients_of_no_rows(A, cols, out, fine):  # noqa: F811
    """Weights that have to be laid out, and such that have not."""
    x = A.Packed8(torch.empty(0, cols, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(0, -(-cols // 32), dtype=torch.uint8, device="cuda"))
    w, g = weight_of(2 * out, cols, 301).cuda(), torch.empty(0, 2 * out, dtype=BF16, device="cuda")
    dx, dw = A.linear8_backward(g, x, w)
    assert dx.shape == (0, cols) and dw.shape == w.shape and not dw.any()
    gated, kept = A.gated_linear8(x, w)
    dx, dw = A.gated_linear8_backward(g[:, :out], kept, x, w, fine=fine)
    assert dx.shape == (0, cols) and dw.shape == w.shape and not dw.any()
    assert A.linear_gate8_backward(g, weight_of(2 * out, out, 302).cuda(), kept).shape == (0, 2 * out)


def _kept(A, values, **options):  # noqa: F811
    """What the context hands back of a tensor saved within it, and how many bytes stay allocated meanwhile for one saved alone."""
    class Keep(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, saved):
            ctx.save_for_backward(saved)
            return x.clone()

        @staticmethod
        def backward(ctx, g):
            Keep.back = ctx.saved_tensors[0]
            return g, None

    x = torch.ones(1, device="cuda", requires_grad=True)
    saved = values()
    gc.collect()                                             # earlier classes hold what they were handed
    before = torch.cuda.memory_allocated()
    with A.keep_in_8_bits(**options):
        y = Keep.apply(x, saved)
    after = torch.cuda.memory_allocated()
    torch.autograd.grad(y, x)
    return saved, Keep.back, after - before


@pytest.mark.parametrize("n", [(1 << 20) + 1, 1 << 21, (1 << 21) + 77, 3 * (1 << 20) - 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_saved_rows_of_more_than_a_million_values(A, n, dtype):  # noqa: F811
    """A flattened volume is packed like any other, in groups of 32 of its memory."""
    g = torch.Generator(device="cuda").manual_seed(303)
    for shape in ((n,), (2, n)):
        saved, back, room = _kept(A, lambda: torch.randn(shape, device="cuda", generator=g).to(dtype))
        assert back.dtype is dtype and back.shape == saved.shape and saved.numel() < room < 1.1 * saved.numel() + 4096
        codes, scales = R.pack(saved.reshape(1, -1).cpu())
        assert torch.equal(back.double().cpu().reshape(1, -1), R.values(codes, scales))


def test_a_loss_over_flattened_volumes(A):  # noqa: F811
    """2 (a - b) of the values held."""
    a = torch.randn(128, 128, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(304), requires_grad=True)
    b = torch.randn(128, 128, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(305))
    with A.keep_in_8_bits():
        loss = (a.flatten() - b.flatten()).square().sum()
    got = torch.autograd.grad(loss, a)[0]
    d = (a - b).detach().flatten()
    want = 2.0 * A.pack8(d.reshape(-1, 1024)).unpack(F32).reshape(a.shape)
    assert torch.equal(got, want)


@pytest.mark.parametrize("make", [
    lambda t: t.to_sparse_csr(), lambda t: t.to_sparse(), lambda t: torch._neg_view(t), lambda t: torch.complex(t, t).reshape(-1, 1).conj().imag,
    lambda t: t.as_subclass(type("Tagged", (torch.Tensor,), {})), lambda t: t.t(), lambda t: t.double(), lambda t: t.reshape(-1)[:1 << 21].expand(2, -1),
    lambda t: torch.randn(2, (1 << 21) + 5, device="cuda")[:, :1 << 21],
], ids=["csr", "coo", "negated", "imaginary", "subclass", "across", "64 bits", "expanded", "long rows apart"])
def test_what_is_not_packed_is_kept_as_it_is(A, make):  # noqa: F811
    saved, back, _ = _kept(A, lambda: make(torch.randn(300, 300, device="cuda", generator=torch.Generator(device="cuda").manual_seed(306))))
    assert type(back) is type(saved) and back.layout is saved.layout
    dense = (lambda t: t.to_dense()) if saved.layout is not torch.strided else (lambda t: t.resolve_neg())
    assert torch.equal(dense(back).as_subclass(torch.Tensor), dense(saved).as_subclass(torch.Tensor))


def test_negated_views_are_refused(A):  # noqa: F811
    """Their memory holds the values with the other sign."""
    x, w = torch._neg_view(torch.ones(4, 64, device="cuda")), torch.ones(64, device="cuda")
    for call in (lambda: A.pack8(x), lambda: A.rms_norm8(x, w), lambda: A.rms_norm8(x.resolve_neg(), w, residual=x), lambda: A.rms_norm8(w.reshape(1, -1), torch._neg_view(w)),
                 lambda: A.rms_norm8_backward(x, A.pack8(x.resolve_neg()), torch.ones(4, device="cuda"), w)):
        with pytest.raises(ValueError):
            call()
    assert torch.equal(A.pack8(x.resolve_neg()).unpack(F32), -torch.ones(4, 64, device="cuda"))


# ---- more blocks than one launch takes: what lies at the border between two launches, and at the end ----

CHANNELS = [(0, 40), ((1 << 26) - 40, (1 << 26) + 40), ((1 << 27) - 40, (1 << 27) + 40)]


def _channels(rows, cols, seed):
    return torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed), dtype=torch.float32).to(BF16)


def test_norm_of_many_short_rows(A):  # noqa: F811
    rows, cols = (1 << 27) + 77, 3
    x, w = _channels(rows, cols, 307), torch.tensor([1.0, 0.5, 2.0], device="cuda")
    _, normed, kept, rstd = A.rms_norm8(x, w)
    for begin, end in CHANNELS + [(rows - 50, rows)]:
        _, inverse, v = R.rms_norm(x[begin:end].cpu(), w.cpu(), None, 1e-6, BF16)
        part = A.Packed8(normed.codes[begin:end].contiguous(), normed.scales[begin:end].contiguous())
        R.assert_close(rstd[begin:end], inverse, inverse * R.sum_error(cols), "rstd")
        R.assert_held(part, v, v.abs() * R.sum_error(cols), "normed")
        assert torch.equal(kept.scales[begin:end].cpu(), R.pack(x[begin:end].cpu())[1])


def test_norm_of_many_long_rows(A):  # noqa: F811
    """2^21 rows of 2049: a block each, both ways."""
    rows, cols = (1 << 21) + 5, 2049
    x = torch.empty(rows, cols, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(308))
    w = torch.ones(cols, device="cuda")
    _, normed, kept, rstd = A.rms_norm8(x, w)
    dx, dw = A.rms_norm8_backward(x, kept, rstd, w)
    for begin, end in [(0, 2), ((1 << 21) - 2, (1 << 21) + 2), (rows - 2, rows)]:
        some = x[begin:end].cpu()
        _, inverse, v = R.rms_norm(some, w.cpu(), None, 1e-6, BF16)
        R.assert_close(rstd[begin:end], inverse, inverse * R.sum_error(cols), "rstd")
        R.assert_held(A.Packed8(normed.codes[begin:end].contiguous(), normed.scales[begin:end].contiguous()), v, v.abs() * R.sum_error(cols), "normed")
        held = R.held(A.Packed8(kept.codes[begin:end].contiguous(), kept.scales[begin:end].contiguous()))
        want, size, _, _ = R.rms_norm_backward(some, held, rstd[begin:end].cpu(), w.cpu(), None)
        R.assert_close(dx[begin:end], want, want.abs() * R.half_step(BF16) + size * R.sum_error(cols), "grad_x")


def test_gate_gradient_of_many_short_rows(A):  # noqa: F811
    """du of one gated column; the same through a product of one column; rounded and fine."""
    rows = (1 << 28) + 77
    da = _channels(rows, 1, 309)
    kept = A.Packed8(torch.full((rows, 2, 1), 56, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),        # code 56: 1.0
                     torch.full((rows, 2, 1), 127, dtype=torch.uint8, device="cuda"))
    kept.codes.view(torch.uint8)[1::3, 0] = 64                                                                       # 2.0
    one = torch.ones(1, 1, dtype=BF16, device="cuda")
    for du in (lambda: A.gate8_backward(da, kept, fine=False), lambda: A.linear_gate8_backward(da, one, kept, fine=False),
               lambda: A.gate8_backward(da, kept), lambda: A.linear_gate8_backward(da, one, kept)):
        got = du()
        fine = isinstance(got, A.FineGradient)
        for begin, end in CHANNELS + [((1 << 28) - 40, (1 << 28) + 40), (rows - 50, rows)]:
            want, size = R.gate_backward(da[begin:end].cpu(), R.values(kept.codes[begin:end].view(torch.uint8).cpu(), kept.scales[begin:end].cpu()))
            part = got.rounded[begin:end].float() + got.rest[begin:end].float() if fine else got[begin:end]
            R.assert_close(part, want, want.abs() * (2.0 ** -17 if fine else R.half_step(BF16)) + 2.0 ** -18 * size, "du")
        del got, part


def test_rows_laid_out_by_several_launches(A):  # noqa: F811
    """Codes of one column, in rows of 16 bytes: 2^29 of them are one launch's."""
    rows = (1 << 29) + 300
    x = A.Packed8(torch.full((rows, 1), 56, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.full((rows, 1), 127, dtype=torch.uint8, device="cuda"))
    x.scales[1::2] = 128
    y = A.linear8(x, torch.full((1, 1), 3.0, dtype=BF16, device="cuda"))
    assert bool((y[0::2] == 3.0).all()) and bool((y[1::2] == 6.0).all())


def test_weight_gradient_of_no_rows_and_2_27_values(A):  # noqa: F811
    out, cols = (1 << 14) + 1, 1 << 13
    w = torch.ones(out, cols, dtype=BF16, device="cuda")
    del_me = torch.ones(out, cols, dtype=BF16, device="cuda")
    del del_me                                               # the gradient's memory holds ones
    x = A.Packed8(torch.empty(0, cols, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(0, cols // 32, dtype=torch.uint8, device="cuda"))
    assert not A.linear8_backward(torch.empty(0, out, dtype=BF16, device="cuda"), x, w)[1].any()


def test_parts_within_a_function_of_ones_own(A):  # noqa: F811
    """Forward and backward of linear8 as an autograd.Function, where nothing is recorded, on parameters; and not outside."""
    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            ctx.packed = A.pack8(x)
            ctx.save_for_backward(w)
            return A.linear8(ctx.packed, w)

        @staticmethod
        def backward(ctx, g):
            return A.linear8_backward(g, ctx.packed, ctx.saved_tensors[0])

    x = torch.randn(40, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(310)).to(BF16).requires_grad_(True)
    w = torch.nn.Parameter(weight_of(32, 64, 311).cuda())
    dx, dw = torch.autograd.grad(Linear.apply(x, w).float().square().sum(), (x, w))
    with torch.no_grad():
        packed = A.pack8(x)
        g = (2 * A.linear8(packed, w).float()).to(BF16)
        want = A.linear8_backward(g, packed, w)
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    for call in (lambda: A.pack8(x), lambda: A.linear8(packed, w), lambda: A.gated_linear8(packed, w), lambda: A.rms_norm8(x, torch.ones(64, device="cuda"))):
        with pytest.raises(ValueError, match="records no gradient"):
            call()


@pytest.mark.parametrize("rows,cols,hidden,out,added", [(0, 64, 32, 64, True), (1, 32, 32, 32, True), (130, 343, 70, 90, False), (3000, 512, 256, 512, True)])
def test_a_block_without_a_backward_pass(A, rows, cols, hidden, out, added):  # noqa: F811
    """The same bits as with one, and none of the memory that only a backward pass reads, whether nothing is recorded or nothing wants a gradient."""
    x, r, nw, up, _, _, _ = _block(max(rows, 1), cols, hidden, seed=320)
    x, r, nw, up, down = x[:rows].cuda(), r[:rows].cuda() if added else None, nw.cuda(), up.cuda(), weight_of(out, hidden, 328).cuda()
    wants = [t.clone().requires_grad_(True) for t in (nw, up, down)]
    want_y, want_s = A.feed_forward8(x, *wants, residual=r)
    assert want_y.requires_grad
    for weights, recording in ((wants, False), ((nw, up, down), True)):
        gc.collect()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        with torch.set_grad_enabled(recording):
            y, s = A.feed_forward8(x, *weights, residual=r)
        most = torch.cuda.max_memory_allocated() - before
        assert torch.equal(y, want_y) and torch.equal(s, want_s) and not y.requires_grad
        whole = rows * (2 * out + (2 * cols if added else 0)) + rows * (cols + hidden) * 33 // 32 + 2 * (2 * hidden * (cols + 8) + out * (hidden + 8))
        assert rows < 1000 or most < whole + 65536                        # the packed sum and both halves, 3 MB, are not there
        del y, s


@pytest.mark.parametrize("cols", [40, 512, 2500])
def test_norm_gradient_without_the_weights(A, cols):  # noqa: F811
    x, w = _channels(300, cols, 330), torch.ones(cols, device="cuda")
    _, _, kept, rstd = A.rms_norm8(x, w)
    want, _ = A.rms_norm8_backward(x, kept, rstd, w)
    got, none = A.rms_norm8_backward(x, kept, rstd, w, need_weight=False)
    assert none is None and torch.equal(got, want)


@pytest.mark.parametrize("dtype", [F32, BF16, torch.float16])
def test_the_types_lowest_number_stays_finite(A, dtype):  # noqa: F811
    """As a mask has it: its product with a gradient of zero is zero, not NaN.  Infinities and NaN are still held as NaN."""
    info = torch.finfo(dtype)
    x = torch.randn(300, 300, device="cuda", generator=torch.Generator(device="cuda").manual_seed(331)).to(dtype)
    x[::2, 5::7] = info.min
    x[1::2, 3::5] = info.max
    x[7, 9], x[8, 290], x[9, 0] = float("inf"), float("-inf"), float("nan")
    lost = ~torch.isfinite(x)
    held = R.values(*R.pack(x.cpu())).cuda()
    want = held.clamp(info.min, info.max).to(dtype)                   # NaN stays NaN
    for back in (A.pack8(x).unpack(dtype, finite=True), _kept(A, lambda: x)[1]):
        assert torch.equal(torch.isnan(back), lost) and torch.equal(back[~lost], want[~lost]) and torch.isfinite(back[~lost]).all()
    assert torch.isinf(A.pack8(x).unpack(dtype)[~lost]).any()
    x = x.nan_to_num(0.0, 0.0, 0.0)
    scale = torch.ones(300, 300, dtype=dtype, device="cuda", requires_grad=True)
    with A.keep_in_8_bits():
        value = torch.where(x == info.min, 0.0, (x * scale)).float()
    assert torch.isfinite(torch.autograd.grad(value, scale, torch.zeros_like(value))[0]).all()
    long = torch.full(((1 << 20) + 5,), info.min, dtype=dtype, device="cuda")
    assert torch.equal(_kept(A, lambda: long)[1], long)
