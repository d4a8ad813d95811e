"""Group norm on the GPU against its definition in 64 bits (tests/networks_reference.py says how far a kernel may be off)."""
import gc

import pytest
import torch

import networks_reference as R
from activations_reference import assert_close

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def N():
    from paper_2307_05801_amd import networks
    return networks


def rand(shape, seed, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def inputs(shape, dtype, seed, parameter=None):
    """x with channels of different size and mean, weight, bias, gradient."""
    c = shape[-1]
    x = rand(shape, seed) * torch.exp(0.5 * rand((c,), seed + 1)) + rand((c,), seed + 2)
    parameter = dtype if parameter is None else parameter
    return x.to(dtype), (1 + 0.3 * rand((c,), seed + 3)).to(parameter), (0.3 * rand((c,), seed + 4)).to(parameter), rand(shape, seed + 5, dtype)


def run(N, x, groups, weight, bias, grad, activation, eps=1e-5):
    leaves = [t.cuda().detach().requires_grad_(True) for t in (x, weight, bias) if t is not None]
    rest = iter(leaves[1:])
    y = N.group_norm(leaves[0], groups, *(None if t is None else next(rest) for t in (weight, bias)), activation=activation, eps=eps)
    got = iter(torch.autograd.grad(y, leaves, grad.cuda()))
    return (y.detach(), next(got), *(None if t is None else next(got) for t in (weight, bias)))


def check(got, r):
    for name, t in zip(("y", "grad_x", "grad_weight", "grad_bias"), got):
        if t is not None:
            assert_close(t, getattr(r, name), getattr(r, name + "_off"), name)


SHAPES = [((1, 1, 8), 1), ((1, 1, 6), 2), ((2, 3, 1), 1), ((2, 50, 3), 3), ((3, 7, 5), 1), ((1, 1000, 5), 5), ((2, 333, 20), 4), ((2, 64, 64), 8), ((1, 4097, 12), 3), ((2, 10, 11, 12, 16), 4),
          ((1, 77, 343), 7), ((1, 40, 512), 32), ((2, 33, 2100), 7), ((1, 9, 4096), 2), ((2, 5, 2051), 1), ((5, 17000, 8), 2), ((1, 70001, 7), 7), ((40, 300, 24), 3), ((3, 2, 96), 96), ((700, 9), 3), ((2, 2048, 64), 8), ((1, 1, 16384), 1), ((3, 85, 48), 2), ((60, 3, 24), 1), ((1, 2049, 8), 1)]


@pytest.mark.parametrize("shape,groups", SHAPES)
@pytest.mark.parametrize("dtype,activation", [(F32, "silu"), (BF16, None), (F16, "relu"), (BF16, "silu")])
def test_shapes(N, shape, groups, dtype, activation):
    x, w, b, g = inputs(shape, dtype, 1)
    check(run(N, x, groups, w, b, g, activation), R.GroupNorm(x, groups, w, b, activation, 1e-5, g))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("activation", [None, "relu", "silu"])
def test_parameters(N, dtype, activation):
    """Weights in 32 bits or of x's type, one of them or none."""
    x, w, b, g = inputs((2, 100, 24), dtype, 11, F32)
    for weight, bias in ((w, b), (w, None), (None, b), (None, None)):
        check(run(N, x, 4, weight, bias, g, activation), R.GroupNorm(x, 4, weight, bias, activation, 1e-5, g))


@pytest.mark.parametrize("offset", [10.0, 1000.0, 30000.0])
def test_a_mean_far_larger_than_the_deviation(N, offset):
    x, w, b, g = inputs((2, 3000, 16), F32, 21)
    x = x + offset
    x[:, 0] = -offset                                                # and a first voxel that is far from it
    check(run(N, x, 2, w, b, g, "silu"), R.GroupNorm(x, 2, w, b, "silu", 1e-5, g))


def test_values_all_alike(N):
    """A variance of zero: the bias comes out."""
    x, b = torch.full((2, 70, 8), 3.25), rand((8,), 31)
    y, gx, gw, gb = run(N, x, 2, torch.ones(8), b, torch.ones(2, 70, 8), None)
    assert torch.equal(y.cpu(), b.expand(2, 70, 8)) and torch.isfinite(gx).all() and not gw.any() and torch.equal(gb.cpu(), torch.full((8,), 140.0))


def test_what_is_not_a_number_stays_in_its_group(N):
    x, w, b, g = inputs((2, 40, 12), F32, 41)
    for what in (float("nan"), float("inf")):
        x[1, 7, 5] = what
        for activation in (None, "relu", "silu"):
            bad = torch.zeros(x.shape, dtype=torch.bool)
            bad[1, :, 4:8] = True
            y, gx, _, _ = run(N, x, 3, w, b, g, activation)
            assert torch.equal(torch.isnan(y.cpu()), bad) and not torch.isnan(gx.cpu()[~bad]).any()


@pytest.mark.parametrize("shape,groups", [((2, 30, 20), 4), ((1, 500, 64), 8), ((3, 10, 7), 1)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_a_wider_array(N, shape, groups, dtype):
    """x and the gradient as columns of something wider, from any byte on; items in another order; one without gaps and one with."""
    wide = shape[:-1] + (shape[-1] + 5,)
    (x, w, b, g), r = inputs(shape, dtype, 51), None
    r = R.GroupNorm(x, groups, w, b, "silu", 1e-5, g)

    def within(t):
        to = torch.zeros(wide, dtype=dtype, device="cuda")
        to[..., 3:3 + shape[-1]] = t.cuda()
        return to[..., 3:3 + shape[-1]]

    for a, c in ((within(x), within(g)), (within(x), g.cuda()), (x.cuda(), within(g))):
        check(run(N, a, groups, w, b, c, "silu"), r)
    across = x.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    check(run(N, across, groups, w, b, g, "silu"), r)


def test_channels_last_memory_of_torch(N):
    x, w, b, g = inputs((2, 4, 5, 6, 16), BF16, 61)
    r = R.GroupNorm(x, 4, w, b, "silu", 1e-5, g)
    t = x.cuda().movedim(-1, 1).contiguous(memory_format=torch.channels_last_3d)
    check(run(N, t.movedim(1, -1), 4, w, b, g, "silu"), r)


def test_a_gradient_of_one_number(N):
    """The gradient of a sum, which has distance 0, and one that lies across."""
    x, w, b, g = inputs((2, 30, 16), F32, 71)
    leaf = x.cuda().requires_grad_(True)
    got, = torch.autograd.grad(N.group_norm(leaf, 4, w.cuda(), b.cuda(), activation="silu").sum(), leaf)
    r = R.GroupNorm(x, 4, w, b, "silu", 1e-5, torch.ones(x.shape))
    assert_close(got, r.grad_x, r.grad_x_off)
    r = R.GroupNorm(x, 4, w, b, "silu", 1e-5, g)
    check(run(N, x, 4, w, b, g.transpose(1, 2).contiguous().transpose(1, 2), "silu"), r)


@pytest.mark.parametrize("shape", [(0, 5, 8), (2, 0, 8), (0, 0, 8)])
def test_nothing_to_norm(N, shape):
    x, w, b, g = inputs(shape, BF16, 81)
    y, gx, gw, gb = run(N, x, 2, w, b, g, "silu")
    assert y.shape == shape and gx.shape == shape and not gw.any() and not gb.any()


def test_without_a_backward_pass_and_one_by_one(N):
    x, w, b, g = (t.cuda() for t in inputs((2, 5000, 24), F32, 91))
    want = run(N, x, 3, w, b, g, "silu")
    with torch.no_grad():
        assert torch.equal(N.group_norm(x, 3, w, b, "silu"), want[0])
    for i in range(3):
        leaves = [t.detach().requires_grad_(j == i) for j, t in enumerate((x, w, b))]
        got, = torch.autograd.grad(N.group_norm(leaves[0], 3, *leaves[1:], "silu"), leaves[i], g)
        assert torch.equal(got, want[1 + i])
    module = N.GroupNorm(3, 24, "silu")
    assert torch.equal(module(x), N.group_norm(x, 3, module.weight, module.bias, "silu"))


def test_kept_in_8_bits(N):
    """x packed between the passes: the gradients are those of the values held, with the statistics of the forward pass; a quarter of the memory."""
    from paper_2307_05801_amd import activations as A
    x, w, b, g = (t.cuda() for t in inputs((2, 4096, 64), F32, 101))
    leaf = x.clone().requires_grad_(True)

    def step():
        moved = leaf * 1.0
        gc.collect()
        before = torch.cuda.memory_allocated()
        y = N.group_norm(moved, 8, w, b, "silu")
        moved = None
        return y, torch.cuda.memory_allocated() - before - y.numel() * 4, y

    with A.keep_in_8_bits():
        y, room, _ = step()
    assert room < -x.numel() * 4 + 1.1 * x.numel() + 4096               # x itself is gone
    got, = torch.autograd.grad(y, leaf, g)
    held = A.pack8(x).unpack(F32).reshape(2, -1, 8, 8).double()
    whole = x.double().reshape(2, -1, 8, 8)
    mean = whole.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt((whole - mean).square().mean((1, 3), keepdim=True) + 1e-5)
    h, w8, b8 = (held - mean) * rstd, w.double().view(8, 8), b.double().view(8, 8)
    du = g.double().reshape(h.shape) * R._slope(h * w8 + b8, "silu") * w8
    want = rstd * (du - du.mean((1, 3), keepdim=True) - h * (du * h).mean((1, 3), keepdim=True))
    assert (got.double() - want.reshape(x.shape)).norm() <= 2.0 ** -18 * want.norm()


def test_what_is_kept_is_freed_and_watched(N):
    x, w, b, _ = (t.cuda() for t in inputs((2, 500, 64), F32, 111))
    w.requires_grad_(True)
    gc.collect()
    gc.disable()
    try:
        before = torch.cuda.memory_allocated()
        for turn in range(3):
            y = N.group_norm(x, 8, w, b, "silu")                        # its backward pass never runs
            del y
        assert torch.cuda.memory_allocated() == before
    finally:
        gc.enable()
    y = N.group_norm(x, 8, w, b)
    x.mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_another_stream_and_graph_replays(N):
    x, w, b, g = (t.cuda() for t in inputs((3, 5000, 20), BF16, 121))

    def step(x, w, b, g):
        leaves = [t.detach().requires_grad_(True) for t in (x, w, b)]
        y = N.group_norm(leaves[0], 4, *leaves[1:], "silu")
        return [y.detach(), *torch.autograd.grad(y, leaves, g)]

    want = step(x, w, b, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(x, w, b, g)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    del got
    places, graphs = [[t.clone() for t in (x, w, b, g)] for _ in range(2)], []
    for p in places:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(*p)
        graphs.append((graph, out))
    for turn in range(4):
        graph, out = graphs[turn % 2]
        new = [(t.float() * (1 + 0.01 * turn)).to(t.dtype) for t in (x, w, b, g)]
        for at, n in zip(places[turn % 2], new):
            at.copy_(n)
        for t in out:
            t.zero_()
        graph.replay()
        want = step(*new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, want)), turn


def test_refusals(N):
    x, w = torch.zeros(2, 5, 8, device="cuda"), torch.ones(8, device="cuda")
    good = dict(x=x, groups=2, weight=w, bias=w)
    N.group_norm(**good)
    for change in (dict(x=x.double()), dict(x=x.int()), dict(x=x[0, 0]), dict(x=x.transpose(1, 2)), dict(x=torch._neg_view(x)), dict(x=x[..., :0], groups=1), dict(groups=3), dict(groups=0), dict(activation="gelu"),
                   dict(eps=-1.0), dict(eps=float("nan")), dict(weight=w[:4]), dict(weight=w.half()), dict(weight=w.cpu()), dict(bias=w.double()), dict(weight=w.expand(2, 8)),
                   dict(x=x.half(), weight=w.half()), dict(weight=torch._neg_view(w)), dict(x=torch.zeros(2, 3, 5, 8, device="cuda").transpose(1, 2))):
        with pytest.raises(ValueError):
            N.group_norm(**{**good, **change})


def test_many_voxels(N):
    """More values than 2^31: the ends against the definition (sums of all values in 64 bits)."""
    voxels, channels = (1 << 26) + 3, 33
    x = torch.empty(1, voxels, channels, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(131))
    y = N.group_norm(x, 3)
    for group in range(3):
        sums = [[f(x[0, at:at + (1 << 22), group * 11:group * 11 + 11].double()) for at in range(0, voxels, 1 << 22)] for f in (torch.sum, lambda t: t.square().sum())]
        mean, square = (float(torch.stack(s).sum()) / (voxels * 11) for s in sums)
        rstd = (square - mean * mean + 1e-5) ** -0.5
        for at in (slice(0, 3), slice(voxels - 3, voxels), slice(1 << 25, (1 << 25) + 3)):
            want = (x[0, at, group * 11:group * 11 + 11].double() - mean) * rstd
            assert ((y[0, at, group * 11:group * 11 + 11].double() - want).abs() <= (R.HALF + 1e-5) * want.abs() + 1e-6).all()


@pytest.mark.parametrize("shape,groups", [((100003, 1, 63), 7), ((70001, 2, 21), 1), ((150001, 3, 16), 2), ((20011, 9, 30), 3), ((33000, 64, 9), 1)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_small_items(N, shape, groups, dtype):
    """More than are worked on at once: the weight's and the bias' gradients are sums over all of them."""
    x, w, b, g = inputs(shape, dtype, 141, F32)
    check(run(N, x, groups, w, b, g, "silu"), R.GroupNorm(x, groups, w, b, "silu", 1e-5, g))


def test_memory_of_a_norm_over_rows(N):
    """2^20 rows of 63 channels, 132 MB: y, the gradient and a workspace of no more than four bytes a value and 48 MiB."""
    x = torch.empty(1 << 20, 63, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(151)).requires_grad_(True)
    w = torch.ones(63, device="cuda", requires_grad=True)
    gc.collect()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    y = N.group_norm(x, 7, w)
    got = torch.autograd.grad(y, (x, w), y.detach())
    torch.cuda.synchronize()
    assert torch.cuda.max_memory_allocated() - before <= 2 * x.numel() * 2 + (1 << 20) * 7 * 8 + 4 * x.numel() + (48 << 20) + (1 << 20)
    assert all(torch.isfinite(t).all() for t in got)


def test_sums_over_many_voxels(N):
    """2^30 voxels, each with the slope of its channel's bias as du.  512 such numbers one after the other are off by up to half of 512 times 2^-24 of their sum, a block's threads by 8 steps
    more and the slope itself by some (8 + |u|) units (networks_reference.py)."""
    voxels, channels = 1 << 30, 8
    x = torch.zeros(1, voxels, channels, dtype=BF16, device="cuda")
    b = rand((channels,), 161)
    w, bias = torch.ones(channels, device="cuda", requires_grad=True), b.cuda().requires_grad_(True)
    y = N.group_norm(x, 1, w, bias, "silu")
    assert torch.equal(y[0, 0], y[0, -1]) and torch.equal(y[0, 0], y[0, 1 << 29])
    gw, gb = torch.autograd.grad(y, (w, bias), torch.ones_like(y))
    want = voxels * R._slope(b.double(), "silu")
    assert not gw.any()
    assert ((gb.cpu().double() - want).abs() <= (256 + 8 + 16) * 2.0 ** -24 * want.abs()).all(), (gb.cpu().double() / want - 1)


@pytest.mark.parametrize("shape,groups", [((2, 3000, 20), 4), ((1, 5, 7), 7), ((2, 2048, 64), 8), ((1, 40000, 24), 3)])
@pytest.mark.parametrize("size", [1e20, -1e25, 1e37])
def test_a_mean_whose_square_is_beyond_32_bits(N, shape, groups, size):
    """All values alike, so the bias comes out; and, to 2^55, values about the mean: those are held exactly, at most two units of 2^-24 of the largest apart."""
    x, w, b, g = inputs(shape, F32, 171)
    flat = torch.full(shape, size)
    y, gx, gw, gb = run(N, flat, groups, w, b, g, "silu")
    assert_close(y, torch.nn.functional.silu(b.double()).expand(shape), 16 * 2.0 ** -24 * b.abs().double().expand(shape))
    assert all(torch.isfinite(t).all() for t in (gx, gw, gb))
    if size == 1e20:
        near = (flat.view(torch.int32) + torch.randint(-2, 3, shape, generator=torch.Generator().manual_seed(172), dtype=torch.int32)).view(F32)
        assert (near.double() - size).abs().max() < 2.0 ** 55
        y = N.group_norm(near.cuda(), groups)
        assert torch.isfinite(y).all()
        r = R.GroupNorm(near, groups)
        # the mean, of 32 bits, is off by half a unit of the largest and by what joining adds: as far as values are apart, so y is off by some times one
        assert (y.cpu().double() - r.y).abs().max() <= 4.0


@pytest.mark.parametrize("voxels,groups", [(8, 1), (8, 2), (5000, 1)])
def test_silu_to_32_bits(N, voxels, groups):
    """Values all alike, so u is the bias, from -87 to 30.  Of float32 the sigmoid is off by 5 units of 2^-24 (by half of them where u is positive), two more for each of its exponential's two
    factors and of its reciprocal, the product by one; with gradients of powers of two the sums of a channel are products and, of eight, three roundings.  slope = s (1 + u (1 - s))."""
    channels, unit = 2050 if groups == 2 else 2048, 2.0 ** -24
    b = torch.linspace(-87, 30, channels)
    x = torch.full((1, voxels, channels), 3.25)
    leaves = [t.cuda().requires_grad_(True) for t in (x, torch.ones(channels), b)]
    y = N.group_norm(leaves[0], groups, *leaves[1:], "silu")
    s = torch.sigmoid(b.double())
    want = b.double() * s
    assert ((y[0].detach().cpu().double() - want).abs() <= 12 * unit * want.abs() + 2.0 ** -148).all()
    grad = torch.zeros(x.shape)
    grad[:, :8] = 1.0
    got, = torch.autograd.grad(y, leaves[2], grad.cuda())
    slope = s * (1 + b.double() * (1 - s))
    off = 11 * slope.abs() + s * (b.abs().double() * (11 * s + 1) + 1) + 4 * slope.abs()
    assert ((got.cpu().double() - 8 * slope).abs() <= 8 * (unit * off + 2.0 ** -148)).all()


def test_silu_of_what_is_far_off(N):
    """Beyond what the exponential holds: zeros on one side, the number itself on the other, infinity included."""
    b = torch.tensor([-1e4, -1e30, -torch.finfo(BF16).max, 1e4, 1e30, torch.finfo(BF16).max, torch.inf, 0.0])       # (float32's largest is infinite in bfloat16)
    for dtype in (F32, BF16):
        y = N.group_norm(torch.zeros(1, 4, 8, dtype=dtype, device="cuda"), 1, None, b.to(dtype).cuda(), "silu").cpu()
        assert torch.equal(y, torch.where(b < 0, 0.0, b).to(dtype).expand(1, 4, 8)), y
