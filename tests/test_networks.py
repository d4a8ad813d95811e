"""Attention and group norm, what needs no GPU: the ABI, the refusals, the references and the places of a grid."""
import os
import re

import pytest
import torch

import networks_reference as R
from paper_2307_05801_amd import binding as B
from paper_2307_05801_amd import networks as N

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000                                   # addresses are never touched: every call below is refused before anything is launched


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2307_05801_amd.build import build_library
        build_library()
    return B.load_activations()


def test_every_declared_symbol_is_exported_and_bound(lib):
    header = open(os.path.join(ROOT, "include", "leap_networks.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = dict(re.findall(r"\b(leap_[a-z0-9_]+)\s*\(([^)]*)\)", header))
    assert set(declared) == set(B.NETWORK_EXPORTS)
    for name, arguments in declared.items():
        assert getattr(lib, name) is not None
        assert len(arguments.split(",")) == len(B.NETWORK_EXPORTS[name][1]), name
    assert f"LEAP_ATTENTION_WIDEST = {B.LEAP_ATTENTION_WIDEST}, LEAP_ATTENTION_BUCKETS = {B.LEAP_ATTENTION_BUCKETS}" in header


# batch, queries, keys, heads, kv_heads, width; strides of q, k, v; mask's, differences, buckets; mask, table, buckets, positions; type, scale
GOOD = (2, 5, 7, 4, 2, 64, 1280, 256, 64, 896, 128, 64, 896, 128, 64, 7, 13, 9, P, P, P, P, P, 0, 0.125)
BAD = [(0, -1), (0, 1 << 31), (1, -1), (1, 1 << 31), (2, -1), (3, 0), (3, 3), (4, 0), (4, 3), (5, 0), (5, 129), (6, -1), (7, -5), (8, -1), (9, -1), (10, -1), (11, -1), (12, -1),
       (13, -1), (14, -1), (7, 1 << 58), (15, -1), (16, 0), (16, 1 << 31), (17, 0), (17, 4097), (20, 0), (23, 3), (23, -1), (24, 0.0), (24, -1.0), (24, float("nan")), (24, float("inf"))]


def test_bad_descriptions_are_refused_with_a_message(lib):
    for at, value in BAD:
        d = list(GOOD)
        d[at] = value
        desc = N._DESC.pack(*d)
        assert lib.leap_attention(desc, P, P, P, P, P, P, P, None) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error().decode()
        assert lib.leap_attention_backward(desc, P, 1280, 256, 64, P, P, P, P, P, P, P, P, P, P, P, None) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_attention_backward_work(desc, 1) == 0 and lib.leap_attention_work(desc) == 0
    assert lib.leap_attention(None, P, P, P, P, P, P, P, None) == B.LEAP_INVALID_ARG


def test_bad_arguments_are_refused_with_a_message(lib):
    desc, plain = N._DESC.pack(*GOOD), N._DESC.pack(*GOOD[:16], 0, 0, P, 0, 0, 0, 0, 0, 0.125)
    good = (desc, P, P, P, P, P, P, P, None)
    for at, value in [(1, 0), (2, 0), (3, 0), (4, 0), (5, 0), (6, 0)]:       # statistics and what rounding leaves: both or neither
        arguments = list(good)
        arguments[at] = value
        assert lib.leap_attention(*arguments) == B.LEAP_INVALID_ARG, (at, value)
    good = (desc, P, 1280, 256, 64, P, P, P, P, P, P, P, P, P, P, P, None)
    for at, value in [(1, 0), (2, -1), (3, -1), (4, -1), (3, 1 << 58), (5, 0), (6, 0), (7, 0), (8, 0), (9, 0), (10, 0), (15, 0), (15, P + 8)]:
        arguments = list(good)
        arguments[at] = value
        assert lib.leap_attention_backward(*arguments) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error().decode()
    assert lib.leap_attention_backward(plain, *good[1:]) == B.LEAP_INVALID_ARG       # a gradient of no table


def test_nothing_to_do_is_fine(lib):
    for at in (0, 1):
        d = list(GOOD)
        d[at] = 0
        assert lib.leap_attention(N._DESC.pack(*d), None, None, None, None, None, None, None, None) == B.LEAP_OK


def test_tensors_elsewhere_or_of_other_kinds_are_refused():
    x = torch.zeros(1, 2, 3, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        N.attention(x, x, x)


@pytest.mark.parametrize("shape,near,codes", [((), 1, 1), ((0,), 1, 2), ((4, -1), 1, 2), ((4,), 0, 2), ((4,), 3, 2), ((4, 4, 4), 9, 9), ((1 << 30,), 1, 2)])
def test_grids_that_are_refused(shape, near, codes):
    with pytest.raises(ValueError):
        N.relative_buckets(shape, near, codes, device="cpu")


@pytest.mark.parametrize("shape,near,codes", [((1,), 1, 1), ((7,), 7, 7), ((40,), 4, 7), ((5, 6), 2, 3), ((3, 4, 5), 1, 2), ((3, 1, 9), 5, 8)])
def test_places_of_a_grid(shape, near, codes):
    """Every pair's bucket from its distances along the axes."""
    positions, buckets = N.relative_buckets(shape, near, codes, device="cpu")
    places = torch.cartesian_prod(*[torch.arange(n) for n in shape]).reshape(-1, len(shape)).tolist()
    assert len(positions) == len(places)

    def code(d):
        a = abs(d)
        c, edge = 0, 0                                       # the code's first distance
        while True:
            following = c + 1 if c + 1 <= near else edge * 2
            if a < following or c == codes - 1:
                return (c if d >= 0 else -c) + codes - 1
            c, edge = c + 1, following

    for i, a in enumerate(places):
        for j, b in enumerate(places):
            want = 0
            for u, w in zip(a, b):
                want = want * (2 * codes - 1) + code(w - u)
            assert int(buckets[positions[j] - positions[i] + len(buckets) // 2]) == want


def test_the_references_gradients_are_those_of_differences():
    g = torch.Generator().manual_seed(1)
    q, k, v, grad = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((2, 3, 4, 5), (2, 6, 2, 5), (2, 6, 2, 5), (2, 3, 4, 5)))
    table, buckets = torch.randn(4, 7, generator=g, dtype=torch.float64), torch.randint(0, 7, (9,), generator=g)
    mask = torch.rand(2, 6, generator=g) < 0.7
    qp, kp = torch.tensor([0, 5, 2]), torch.tensor([1, 3, 3, 0, 9, 4])
    r = R.Attention(q, k, v, grad, mask, table, buckets, (qp, kp))

    def value(q, k, v, table):
        return (R.attention(q, k, v, mask, R.bias_of(table, buckets, qp, kp)[0])[0] * grad).sum()

    for name, t in (("grad_q", q), ("grad_k", k), ("grad_v", v), ("grad_table", table)):
        for _ in range(3):
            way = torch.randn(t.shape, generator=g, dtype=torch.float64)
            h = 1e-6
            ends = [value(*(s * h * way + u if u is t else u for u in (q, k, v, table))) for s in (1, -1)]
            got, want = (getattr(r, name) * way).sum(), (ends[0] - ends[1]) / (2 * h)
            assert abs(got - want) <= 1e-7 * (1 + abs(want)), name


# ---- group norm ----


def test_bad_arguments_of_group_norm_are_refused_with_a_message(lib):
    good = (P, 1, 640, 60, P, P, 1, 2, 10, 60, 6, 1e-5, 2, P, P, P, None)
    for at, value in [(0, 0), (1, 3), (2, -1), (3, 59), (3, -1), (6, 2), (6, 7), (7, -1), (7, 1 << 40), (8, -1), (8, 1 << 40), (9, 0), (9, 1 << 21), (10, 0), (10, 7), (11, -1.0), (11, float("nan")), (12, 3),
                      (12, -1), (13, 0), (15, 0), (15, P + 8)]:
        arguments = list(good)
        arguments[at] = value
        assert lib.leap_group_norm(*arguments) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error().decode()
    good = (P, 640, 64, P, 1, 640, 64, P, P, 1, P, 2, 10, 64, 8, 2, P, P, P, P, None)
    for at, value in [(0, 0), (1, -1), (2, 63), (3, 0), (4, 3), (5, -1), (6, 63), (9, 2), (10, 0), (11, -1), (12, -1), (13, 0), (14, 7), (15, 3), (19, 0), (19, P + 4)]:
        arguments = list(good)
        arguments[at] = value
        assert lib.leap_group_norm_backward(*arguments) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error().decode()
    assert lib.leap_group_norm_work(-1, 10, 64, 8) == 0 and lib.leap_group_norm_work(2, 10, 64, 7) == 0 and lib.leap_group_norm_backward_work(2, 10, 0, 1) == 0
    assert lib.leap_group_norm(None, 1, 640, 64, None, None, 1, 0, 10, 64, 8, 1e-5, 2, None, None, None, None) == B.LEAP_OK
    assert lib.leap_group_norm(None, 1, 0, 64, None, None, 1, 2, 0, 64, 8, 1e-5, 2, None, None, None, None) == B.LEAP_OK


def test_group_norm_elsewhere_is_refused():
    with pytest.raises(ValueError, match="GPU"):
        N.group_norm(torch.zeros(1, 2, 8), 2)


def test_the_group_norm_references_gradients_are_those_of_differences():
    g = torch.Generator().manual_seed(2)
    x, w, b, grad = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((2, 5, 6), (6,), (6,), (2, 5, 6)))
    for activation in (None, "silu", "relu"):
        r = R.GroupNorm(x, 2, w, b, activation, 1e-3, grad)
        for name, t in (("grad_x", x), ("grad_weight", w), ("grad_bias", b)):
            way, h = torch.randn(t.shape, generator=g, dtype=torch.float64), 1e-6
            ends = [(R.GroupNorm(*(s * h * way + u if u is t else u for u in (x,)), 2, *(s * h * way + u if u is t else u for u in (w, b)), activation, 1e-3).y * grad).sum() for s in (1, -1)]
            got, want = (getattr(r, name) * way).sum(), (ends[0] - ends[1]) / (2 * h)
            assert abs(got - want) <= 1e-7 * (1 + abs(want)), (activation, name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_what_is_kept_as_bytes_may_have_any_last_stride_where_rows_have_one_value(dtype):
    rows = torch.arange(30).to(dtype).reshape(2, 5, 1, 3).transpose(2, 3)                     # [2, 5, 3, 1], last stride 3
    one = torch.arange(24).to(dtype)[2:].as_strided((5, 1), (2, 9))
    for t in (rows, one):
        assert t.stride(-1) != 1
        assert torch.equal(N._bytes(t).view(dtype), t)
        assert N._bytes(t).data_ptr() == t.data_ptr()


@pytest.mark.parametrize("channels", [1, 3, 7, 8, 20, 63, 64, 343, 2047, 2048])
@pytest.mark.parametrize("voxels", [1, 2, 3, 8, 63, 64, 65, 4096])
def test_the_workspace_of_group_norm_is_no_larger_than_its_arrays(lib, channels, voxels):
    """Of a batch of any number of items: 2.5 bytes a value of x for the forward pass, four for the backward, and 48 MiB that a chip full of blocks takes for small arrays; it was up to
    a hundred bytes a value."""
    for items in (1, 5, 1 << 10, 1 << 14, 1 << 20):
        if items * voxels * channels > 1 << 36 or items * channels > 1 << 31:
            continue
        for groups in {1, channels}:
            values = items * voxels * channels
            assert lib.leap_group_norm_work(items, voxels, channels, groups) <= (48 << 20) + 5 * values // 2, (items, groups)
            assert lib.leap_group_norm_backward_work(items, voxels, channels, groups) <= (48 << 20) + 4 * values, (items, groups)


@pytest.mark.parametrize("shape", [((1 << 23) + 1,), (2049, 2049), (129, 129, 129), (1, 4097, 1025)])
def test_grids_of_more_differences_than_attention_takes_are_refused(lib, shape):
    with pytest.raises(ValueError, match="differences"):
        N.relative_buckets(shape, 1, 2, device="cpu")
    header = open(os.path.join(ROOT, "include", "leap_networks.h")).read()
    assert B.LEAP_ATTENTION_OFFSETS == 1 << 24 and "LEAP_ATTENTION_OFFSETS = 1 << 24" in header
    for offsets, status in ((1 << 24, False), ((1 << 24) + 1, True)):
        d = list(GOOD)
        d[16] = offsets
        assert (lib.leap_attention_work(N._DESC.pack(*d)) == 0) is status


def test_the_largest_grid_is_taken():
    positions, buckets = N.relative_buckets((1 << 23,), 1, 2, device="cpu")
    assert len(positions) == 1 << 23 and len(buckets) == (1 << 24) - 1


def test_a_tangent_is_not_dropped():
    """Forward mode: a dual tensor requires no gradient, but an operator that went by that alone would lose its tangent."""
    from torch.autograd import forward_ad
    from paper_2307_05801_amd import activations as A
    x, leaf = torch.ones(3), torch.ones(3, requires_grad=True)
    assert not A._records(x, None) and A._records(x, leaf, None)
    with torch.no_grad():
        assert not A._records(x, leaf)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones(3))
        assert not dual.requires_grad and A._records(x, None, dual) and not A._records(x)
        with torch.no_grad():
            assert A._records(dual) and not A._records(x, leaf)
        with pytest.raises(ValueError):
            A._not_recorded(dual)
    assert not A._records(x)


def test_a_library_with_the_operators_in_8_bits_alone_is_taken(monkeypatch):
    """Another build under LEAP_LIB_PATH; what it lacks raises when it is called, and not before."""
    class Function:
        pass

    class Library:
        def __init__(self, names):
            self.__dict__.update({name: Function() for name in names})

    monkeypatch.setattr(B, "_activations", None)
    monkeypatch.setattr(B, "load_library", lambda: Library(B.ACTIVATION_EXPORTS))
    lib = B.load_activations()
    assert lib.leap_pack8.argtypes == B.ACTIVATION_EXPORTS["leap_pack8"][1]
    with pytest.raises(AttributeError):
        lib.leap_attention
    monkeypatch.setattr(B, "_activations", None)
    monkeypatch.setattr(B, "load_library", lambda: Library(()))
    with pytest.raises(AttributeError):
        B.load_activations()


def test_positions_and_buckets_that_are_negated_views_are_refused(monkeypatch):
    """Their memory holds the numbers with the other sign."""
    monkeypatch.setattr(N, "_on_gpu", lambda *a: None)
    t = torch.arange(5, dtype=torch.int32)
    N._integers(t, 5, t.device, "buckets")
    with pytest.raises(ValueError, match="negated"):
        N._integers(torch._neg_view(t), 5, t.device, "buckets")


def test_more_blocks_than_a_launch_has_are_refused_by_that_name(lib):
    """2^24 items of one head and query are as many blocks."""
    plain = [1 << 24, 1, 1, 1, 1, 8] + [8, 8, 8] * 3 + [0, 0, 0, 0, 0, 0, 0, 0, 0, 0.5]
    desc = N._DESC.pack(*plain)
    for status in (lib.leap_attention(desc, P, P, P, P, None, None, None, None), lib.leap_attention_backward(desc, P, 8, 8, 8, P, P, P, P, P, P, P, P, P, None, P, None)):
        assert status == B.LEAP_INVALID_ARG and "2^24" in lib.leap_last_error().decode()
