"""Operators on activations in 8 bits, what needs no GPU: the ABI, the refusals, the format's reference."""
import ctypes as C
import os
import re

import pytest
import torch

import activations_reference as R
from paper_2307_05801_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2307_05801_amd.build import build_library
        build_library()
    return B.load_activations()


def test_every_declared_symbol_is_exported_and_bound(lib):
    header = open(os.path.join(ROOT, "include", "leap_activations.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = dict(re.findall(r"\b(leap_[a-z0-9_]+)\s*\(([^)]*)\)", header))
    assert set(declared) == set(B.ACTIVATION_EXPORTS)
    for name, arguments in declared.items():
        assert getattr(lib, name) is not None
        assert len(arguments.split(",")) == len(B.ACTIVATION_EXPORTS[name][1]), name


# Addresses are never touched: every call below is refused before anything is launched.
P = 0x1000


@pytest.mark.parametrize("name,good,bad", [
    ("leap_pack8", (P, 1, 64, 4, 64, P, P, 0), [(1, 3), (1, -1), (2, -1), (2, 63), (2, 1 << 59), (3, -1), (4, 0), (4, 1 << 21), (3, 1 << 40), (0, 0), (5, 0), (6, 0)]),
    ("leap_unpack8", (P, P, 4, 64, P, 1, 0), [(5, 9), (2, -1), (3, 0), (0, 0), (1, 0), (4, 0)]),
    ("leap_rms_norm8", (P, 64, P, 64, 1, P, 1, 4, 64, 1e-6, P, P, P, P, P, P, 0),
     [(4, 3), (6, 2), (6, 5), (7, -4), (8, 0), (1, 63), (3, 63), (9, -1.0), (9, float("nan")), (0, 0), (5, 0), (11, 0), (12, 0), (13, 0), (14, 0), (7, 1 << 32)]),
    ("leap_rms_norm8_backward", (P, 1, 64, P, 64, 1, P, P, P, P, 1, 4, 64, P, P, P, 0),
     [(1, 2), (5, 8), (10, 2), (2, 1), (4, 1), (11, -1), (12, 0), (0, 0), (6, 0), (7, 0), (8, 0), (9, 0), (13, 0), (15, 0), (11, 1 << 32)]),
    ("leap_linear8", (P, P, 4, 64, P, 64, 8, P, P, 0), [(2, -1), (3, 0), (5, 63), (6, 0), (0, 0), (1, 0), (4, 0), (7, 0), (6, 1 << 21)]),
    ("leap_linear8_backward", (P, 8, P, P, 4, 64, P, 64, 8, P, 1, P, P, 0), [(1, 7), (4, -1), (5, 0), (7, 1), (8, 0), (10, 2), (0, 0), (2, 0), (3, 0), (6, 0)]),
    ("leap_gated_linear8", (P, P, 4, 64, P, 64, 8, P, P, P, P, P, 0), [(2, -1), (3, 0), (5, 63), (6, 0), (6, 1 << 20), (0, 0), (1, 0), (4, 0), (7, 0), (8, 0), (9, 0), (10, 0)]),
    ("leap_gate8_backward", (P, 8, P, P, 4, 8, P, 0), [(1, 7), (4, -1), (5, 0), (5, 1 << 20), (0, 0), (2, 0), (3, 0), (6, 0)]),
    ("leap_linear_gate8_backward", (P, 8, P, 16, 8, P, P, 4, 16, P, P, 0), [(1, 7), (3, 15), (4, 0), (7, -1), (8, 0), (8, 1 << 20), (0, 0), (2, 0), (5, 0), (6, 0), (9, 0)]),
])
def test_bad_arguments_are_refused_with_a_message(lib, name, good, bad):
    for at, value in bad:
        arguments = list(good)
        arguments[at] = value
        assert getattr(lib, name)(*arguments) == B.LEAP_INVALID_ARG, (name, at, value)
        assert lib.leap_last_error().decode()


def test_no_rows_is_fine(lib):
    assert lib.leap_pack8(None, 0, 64, 0, 64, None, None, None) == B.LEAP_OK
    assert lib.leap_unpack8(None, None, 0, 64, None, 0, None) == B.LEAP_OK
    assert lib.leap_rms_norm8(None, 64, None, 0, 1, None, 1, 0, 64, 1e-6, *[None] * 7) == B.LEAP_OK
    assert lib.leap_linear8(None, None, 0, 64, None, 64, 8, None, None, None) == B.LEAP_OK
    assert lib.leap_gate8_backward(None, 8, None, None, 0, 8, None, None) == B.LEAP_OK


def test_bad_arguments_of_the_gated_gradient_are_refused_with_a_message(lib):
    good = (P, 8, P, P, P, P, 4, 64, P, 64, 8, P, 1, P, P, 0)
    for at, value in [(1, 7), (6, -1), (7, 0), (9, 63), (10, 0), (10, 1 << 20), (12, 2), (0, 0), (2, 0), (3, 0), (4, 0), (5, 0), (8, 0), (14, 0), (14, P + 8)]:
        arguments = list(good)
        arguments[at] = value
        assert lib.leap_gated_linear8_backward(*arguments) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error()
    # du in rows of whole 16 bytes, which are not copied again
    assert lib.leap_gated_linear8_backward_work(P, 5, 64, P, 64, 9) == 5 * 24 * 2
    assert lib.leap_gated_linear8_backward_work(P, 5, 40, P, 64, 8) == 5 * 16 * 2 + 5 * 48
    assert lib.leap_gated_linear8_backward_work(P, 5, 64, P, 64, 0) == 0 and lib.leap_gated_linear8_backward_work(P, -1, 64, P, 64, 8) == 0


BLOCK_FORWARD = (P, 64, P, 64, P, 1, 4, 64, 1e-6, P, 64, 8, P, 8, 16, P, P, P, P, 0)
BLOCK_BACKWARD = (P, 16, P, 64, P, 1, 4, 64, P, 64, 8, P, 8, 16, P, P, P, P, P, P, 0)


@pytest.mark.parametrize("name,good,bad", [
    ("leap_feed_forward8", BLOCK_FORWARD, [(5, 2), (6, -1), (6, 1 << 32), (7, 0), (7, 1 << 21), (1, 63), (3, 63), (8, -1.0), (10, 63), (11, 0), (11, 1 << 20),
                                           (13, 7), (14, 0), (0, 0), (4, 0), (9, 0), (12, 0), (16, 0), (17, 0), (17, P + 8)]),
    ("leap_feed_forward8_backward", BLOCK_BACKWARD, [(1, 15), (3, 63), (4, 0), (5, 2), (15, 0), (6, -1), (7, 0), (9, 63), (10, 0), (10, 1 << 20), (12, 7), (13, 0), (0, 0), (8, 0), (11, 0), (14, 0),
                                                     (14, P + 4), (19, 0), (19, P + 8)]),
])
def test_bad_arguments_of_a_block_are_refused_with_a_message(lib, name, good, bad):
    for at, value in bad:
        arguments = list(good)
        arguments[at] = value
        assert getattr(lib, name)(*arguments) == B.LEAP_INVALID_ARG, (name, at, value)
        assert lib.leap_last_error()


def test_memory_of_a_block(lib):
    """Codes and scales of the norm's output, of the sum, of the gated rows and of both halves, rstd: each in whole 16 bytes."""
    assert lib.leap_feed_forward8_kept(4, 64, 40) == 2 * (256 + 16) + 160 + 16 + 320 + 16 + 16
    assert lib.leap_feed_forward8_kept(0, 64, 40) == 0 and lib.leap_feed_forward8_kept(4, 64, 0) == 0 and lib.leap_feed_forward8_kept(-1, 64, 40) == 0
    assert lib.leap_feed_forward8_work(4, 64, P, 64, 16, P, 16, 24) == 0 and lib.leap_feed_forward8_work(4, 64, P, 64, 16, P, 16, 0) == 0
    assert lib.leap_feed_forward8_work(4, 64, P, 65, 16, P, 16, 24) == 32 * 64 * 2
    least = 4 * 2 * 16 * 2 + 4 * 64 * 4 + lib.leap_rms_norm8_work(4, 64) * 4
    assert lib.leap_feed_forward8_backward_work(P, 24, 4, 64, P, 64, 16, P, 16, 24) >= least
    assert lib.leap_feed_forward8_backward_work(P, 23, 4, 64, P, 64, 16, P, 16, 24) == 0
    assert lib.leap_feed_forward8(None, 64, None, 64, None, 1, 0, 64, 1e-6, None, 64, 8, None, 8, 16, *[None] * 5) == B.LEAP_OK


def test_workspaces_of_bad_sizes_are_nothing(lib):
    assert lib.leap_rms_norm8_work(-1, 64) == 0 and lib.leap_rms_norm8_work(5, 0) == 0
    assert lib.leap_linear8_work(P, -1, 64, P, 64, 8) == 0 and lib.leap_linear8_backward_work(P, 8, P, 4, 0, P, 64, 8) == 0
    assert lib.leap_linear_gate8_work(P, 8, P, 16, 8, 4, -1) == 0


def test_workspaces_hold_copies_of_what_is_not_laid_out(lib):
    """Codes of 40 columns in rows of 48, weights of 40 in rows of 40 values; addresses and strides that are no multiple of 16 bytes."""
    assert lib.leap_linear8_work(P, 5, 64, P, 64, 8) == 0
    assert lib.leap_linear8_work(P, 5, 40, P, 40, 8) == 5 * 48
    assert lib.leap_linear8_work(P + 1, 5, 64, P, 64, 8) == 5 * 64
    assert lib.leap_linear8_work(P, 5, 64, P, 65, 8) == 8 * 64 * 2
    assert lib.leap_linear8_work(P, 5, 63, P, 64, 8) == 5 * 64 + 8 * 64 * 2
    assert lib.leap_linear8_backward_work(P, 8, P, 5, 64, P, 64, 8) == 0
    assert lib.leap_linear8_backward_work(P, 9, P, 5, 64, P, 64, 9) == 5 * 16 * 2
    assert lib.leap_linear_gate8_work(P + 2, 8, P, 16, 8, 4, 16) == 4 * 8 * 2
    # a missing workspace is refused where one is needed
    assert lib.leap_linear8(P, P, 5, 40, P, 40, 8, P, None, None) == B.LEAP_INVALID_ARG
    assert lib.leap_linear8_backward(P, 9, P, P, 5, 64, P, 64, 9, P, 1, P, None, None) == B.LEAP_INVALID_ARG
    assert lib.leap_linear_gate8_backward(P, 9, P, 16, 9, P, P, 4, 16, P, None, None) == B.LEAP_INVALID_ARG


def test_workspaces_hold_the_parts_of_long_sums(lib):
    """Few outputs of 1024 values of k or more: sums in 32 bits of parts of at least 256."""
    assert lib.leap_linear8_work(P, 5, 1008, P, 1008, 8) == 0
    assert lib.leap_linear8_work(P, 5, 1024, P, 1024, 8) == 4 * 5 * 8 * 4
    assert lib.leap_linear8_work(P, 64 * 65, 1024, P, 1024, 8) == 0
    assert lib.leap_linear8_backward_work(P, 2048, P, 5, 64, P, 64, 2048) == 8 * 5 * 64 * 4
    assert lib.leap_linear8(P, P, 5, 1024, P, 1024, 8, P, None, None) == B.LEAP_INVALID_ARG


def test_rows_far_apart_or_on_top_of_each_other_are_copied(lib):
    """A tile of 256 rows that are 2^23 bytes apart passes 31 bits; rows of one address have nothing beyond the last that reads as zeros."""
    assert lib.leap_linear8_work(P, 5, 64, P, 1 << 21, 8) == 0
    assert lib.leap_linear8_work(P, 5, 64, P, (1 << 21) + 8, 8) == 8 * 64 * 2
    assert lib.leap_linear8_work(P, 5, 64, P, 0, 8) == 8 * 64 * 2
    assert lib.leap_linear8_backward_work(P, 1 << 24, P, 5, 64, P, 64, 8) == 5 * 8 * 2
    assert lib.leap_linear8_backward_work(P, 0, P, 5, 64, P, 64, 8) == 5 * 8 * 2
    assert lib.leap_linear_gate8_work(P, 0, P, 1 << 24, 8, 4, 16) == 4 * 8 * 2 + 8 * 16 * 2


def _packed(rows, cols):
    from paper_2307_05801_amd.activations import Packed8
    return Packed8(torch.zeros(rows, cols).to(torch.float8_e4m3fn), torch.zeros(rows, -(-cols // 32), dtype=torch.uint8))


def test_packed8_checks_its_parts():
    from paper_2307_05801_amd.activations import Packed8
    codes, scales = torch.zeros(3, 40).to(torch.float8_e4m3fn), torch.zeros(3, 2, dtype=torch.uint8)
    assert Packed8(codes, scales).shape == (3, 40)
    for bad in ((codes.view(torch.uint8), scales), (codes, scales.float()), (codes, scales[:, :1]), (codes, scales[:2]),
                (codes.view(torch.uint8).t().contiguous().t().view(torch.float8_e4m3fn), scales)):
        with pytest.raises(ValueError):
            Packed8(*bad)


def test_tensors_on_the_cpu_are_refused():
    from paper_2307_05801_amd import activations as A
    x, w, p = torch.zeros(4, 64, dtype=BF16), torch.ones(64, dtype=BF16), _packed(4, 64)
    big = torch.zeros(8, 64, dtype=BF16)
    for call in (lambda: A.pack8(x), lambda: A.unpack8(p), lambda: A.rms_norm8(x, w), lambda: A.linear8(p, big),
                 lambda: A.gated_linear8(p, big), lambda: A.gate8_backward(x, _packed(4, 64)), lambda: A.feed_forward8(x, w, big, big),
                 lambda: A.rms_norm8_backward(x, p, torch.ones(4), w), lambda: A.linear8_backward(x, p, big)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("make,want", [
    (lambda: torch.zeros(4, 6), (4, 6, 6)),
    (lambda: torch.zeros(6), (1, 6, 6)),
    (lambda: torch.zeros(4, 10)[:, :6], (4, 6, 10)),
    (lambda: torch.zeros(8, 6)[::2], (4, 6, 12)),
    (lambda: torch.zeros(2, 3, 10)[..., 2:8], (6, 6, 10)),
    (lambda: torch.zeros(2, 1, 3, 10)[..., :6], (6, 6, 10)),
    (lambda: torch.zeros(0, 6), (0, 6, 6)),
    (lambda: torch.zeros(3, 0, 10)[..., :6], (0, 6, 6)),
    (lambda: torch.zeros(4, 1), (4, 1, 1)),
    (lambda: torch.zeros(1, 10)[:, :6], (1, 6, 6)),
])
def test_rows_of_a_tensor(make, want):
    from paper_2307_05801_amd.activations import _rows
    assert _rows(make(), "x") == want


@pytest.mark.parametrize("make", [
    lambda: torch.zeros(6, 4).t(), lambda: torch.zeros(4, 12)[:, ::2], lambda: torch.zeros(2, 5, 6)[:, :3], lambda: torch.tensor(1.0),
    lambda: torch.zeros(4, 0), lambda: torch.zeros(1, 6).expand(4, 6), lambda: torch.zeros(9).as_strided((4, 6), (1, 1)),
])
def test_rows_that_are_not_evenly_spaced_are_refused(make):
    from paper_2307_05801_amd.activations import _rows
    with pytest.raises(ValueError):
        _rows(make(), "x")


def test_the_reference_of_the_format_agrees_with_torchs_cast():
    g = torch.Generator().manual_seed(5)
    x = (torch.randn(200, 70, generator=g) * torch.exp(torch.randn(200, 1, generator=g) * 8)).bfloat16().double()
    codes, scales = R.pack(x)
    power = (2.0 ** (scales.double() - 127)).repeat_interleave(32, -1)[..., :70]
    want = (x / power).float().to(torch.float8_e4m3fn)
    assert torch.equal(codes, want.view(torch.uint8))
    assert float((R.grouped(x).abs().amax(-1) / 2.0 ** (scales.double() - 127)).max()) <= 448


def test_the_reference_notices_a_wrong_code():
    """The bound of a held value, on a mistake planted in the reference: every code one too high, and a scale half as large."""
    from paper_2307_05801_amd.activations import Packed8
    x = torch.randn(8, 64, generator=torch.Generator().manual_seed(6)).double()
    codes, scales = R.pack(x)
    none = torch.zeros_like(x)
    R.assert_held(Packed8(codes.view(torch.float8_e4m3fn), scales), x, none)
    for wrong in ((codes + 1, scales), (codes, scales - 1)):
        with pytest.raises(AssertionError):
            R.assert_held(Packed8(wrong[0].view(torch.float8_e4m3fn), wrong[1]), x, none)


def test_bad_arguments_of_the_fine_gradients_are_refused_with_a_message(lib):
    good = (P, 8, P, P, P, P, 4, 64, P, 64, 8, P, 1, P, P, 0)
    for at, value in [(1, 7), (6, -1), (7, 0), (9, 63), (10, 0), (10, 1 << 20), (12, 2), (0, 0), (2, 0), (3, 0), (4, 0), (5, 0), (8, 0), (14, 0), (14, P + 8)]:
        arguments = list(good)
        arguments[at] = value
        assert lib.leap_gated_linear8_backward_fine(*arguments) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error()
    for at, value in [(1, 15), (3, 63), (4, 0), (5, 2), (15, 0), (6, -1), (7, 0), (9, 63), (10, 0), (10, 1 << 20), (12, 7), (13, 0), (0, 0), (8, 0), (11, 0), (14, 0),
                      (14, P + 4), (19, 0), (19, P + 8)]:
        arguments = list(BLOCK_BACKWARD)
        arguments[at] = value
        assert lib.leap_feed_forward8_backward_fine(*arguments) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error()


def test_memory_of_the_fine_gradients(lib):
    """du twice, in rows of whole 16 bytes; the weight twice, zeros between; both halves of the weight's gradient in 32 bits."""
    assert lib.leap_gated_linear8_backward_fine_work(P, 5, 64, P, 64, 9) == 5 * 48 * 2 + (24 + 18) * 64 * 2 + 2 * 24 * 64 * 4
    assert lib.leap_gated_linear8_backward_fine_work(P, 5, 40, P, 40, 8) == 5 * 32 * 2 + 32 * 40 * 2 + 2 * 16 * 40 * 4 + 5 * 48
    assert lib.leap_gated_linear8_backward_fine_work(P, 5, 64, P, 64, 0) == 0 and lib.leap_gated_linear8_backward_fine_work(P, -1, 64, P, 64, 8) == 0
    plain = lib.leap_feed_forward8_backward_work(P, 24, 4, 64, P, 64, 16, P, 16, 24)
    assert lib.leap_feed_forward8_backward_fine_work(P, 24, 4, 64, P, 64, 16, P, 16, 24) >= plain + 4 * 2 * 16 * 2
    assert lib.leap_feed_forward8_backward_fine_work(P, 23, 4, 64, P, 64, 16, P, 16, 24) == 0


def test_no_rows_need_no_workspace(lib):
    """The gradients of nothing: no copy of a weight that is not laid out (343 columns), no parts."""
    assert lib.leap_linear8_backward_work(None, 8, None, 0, 343, None, 343, 8) == 0
    assert lib.leap_gated_linear8_backward_work(None, 0, 343, None, 343, 8) == 0
    assert lib.leap_gated_linear8_backward_fine_work(None, 0, 343, None, 343, 8) == 0
    assert lib.leap_linear8_backward(None, 8, None, None, 0, 343, None, 343, 8, P, 1, None, None, None) == B.LEAP_OK
    for name in ("leap_gated_linear8_backward", "leap_gated_linear8_backward_fine"):
        for work in (None, P):
            assert getattr(lib, name)(None, 8, None, None, None, None, 0, 343, None, 343, 8, P, 1, None, work, None) == B.LEAP_OK


# ---- keep_in_8_bits: what it keeps as it is (on the CPU that is everything) ----


def test_outputs_kept_for_a_backward_pass_that_never_runs_are_freed():
    """exp saves its own output, whose graph leads back to it: the hook must not close that circle."""
    import gc
    import weakref
    from paper_2307_05801_amd.activations import keep_in_8_bits
    x = torch.randn(100, requires_grad=True)
    with keep_in_8_bits():
        y = (x * 1.0).exp()
    alive = weakref.ref(y)
    del y
    gc.collect()
    assert alive() is None


def test_gradients_through_what_is_kept_as_it_is():
    """First and second derivatives, outputs and leaves that are saved, operations in place that save their result."""
    from paper_2307_05801_amd.activations import keep_in_8_bits
    x, w = (torch.randn(50, dtype=torch.float64, generator=torch.Generator().manual_seed(k), requires_grad=True) for k in (1, 2))

    def f():
        return ((torch.tanh(x * w) * w).exp_() * x).sigmoid_().sum()

    want = torch.autograd.grad(f(), (x, w), create_graph=True)
    want += torch.autograd.grad(want[0].square().sum(), (x, w))
    with keep_in_8_bits():
        value = f()
        got = torch.autograd.grad(value, (x, w), create_graph=True)
        got += torch.autograd.grad(got[0].square().sum(), (x, w))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_what_is_kept_as_it_is_must_not_change_before_the_backward_pass():
    """As without the context: an error, not a gradient of other values."""
    from paper_2307_05801_amd.activations import keep_in_8_bits
    x, w = torch.ones(5, requires_grad=True), torch.ones(5, requires_grad=True)
    with keep_in_8_bits():
        saved_output, saved_leaf = (x * 1.0).exp(), (x * w).sum()
    saved_output.mul_(3.0)
    with torch.no_grad():
        w.add_(1.0)
    for value in (saved_output.sum(), saved_leaf):
        with pytest.raises(RuntimeError, match="in place"):
            torch.autograd.grad(value, x)


@pytest.mark.parametrize("make", [lambda: torch._neg_view(torch.zeros(4, 6)), lambda: torch.zeros(4, 1, dtype=torch.complex64).conj().imag])
def test_rows_of_negated_views_are_refused(make):
    """The imaginary part of a conjugate: its memory holds the values with the other sign."""
    from paper_2307_05801_amd.activations import _rows
    with pytest.raises(ValueError, match="negated"):
        _rows(make(), "x")


def test_workspaces_that_are_not_aligned_are_refused(lib):
    """Where one is needed; the copies in it would not be laid out for the kernels."""
    for name, arguments in (("leap_linear8", (P, P, 5, 40, P, 40, 8, P)), ("leap_linear8", (P, P, 5, 1024, P, 1024, 8, P)),
                            ("leap_linear8_backward", (P, 9, P, P, 5, 64, P, 64, 9, P, 1, P)), ("leap_gated_linear8", (P, P, 5, 40, P, 40, 8, P, P, P, P)),
                            ("leap_linear_gate8_backward", (P, 9, P, 16, 9, P, P, 4, 16, P)),
                            ("leap_feed_forward8", (P, 64, None, 0, P, 1, 4, 64, 1e-6, P, 65, 8, P, 8, 16, P, P, P))):
        for work in (P + 8, P + 1, None):
            assert getattr(lib, name)(*arguments, work, None) == B.LEAP_INVALID_ARG, (name, work)
            assert lib.leap_last_error()


def test_parts_refuse_to_cut_a_graph():
    """Tensors that want a gradient, while autograd records: the results would have none.  Without recording they are looked at as ever
    (and refused here for being on the CPU)."""
    from paper_2307_05801_amd import activations as A
    x, w, big, p = torch.zeros(4, 64, dtype=BF16), torch.ones(64, dtype=BF16), torch.zeros(8, 64, dtype=BF16), _packed(4, 64)
    wants = lambda t: t.clone().requires_grad_(True)  # noqa: E731
    kept, rstd = _packed(4, 64), torch.ones(4)
    for call in (lambda: A.pack8(wants(x)), lambda: A.rms_norm8(wants(x), w), lambda: A.rms_norm8(x, wants(w)), lambda: A.rms_norm8(x, w, residual=wants(x)),
                 lambda: A.linear8(p, wants(big)), lambda: A.gated_linear8(p, wants(big)), lambda: A.linear8_backward(wants(x), p, big),
                 lambda: A.gate8_backward(wants(x), p), lambda: A.linear_gate8_backward(wants(x), big, p), lambda: A.gated_linear8_backward(wants(x), kept, p, big),
                 lambda: A.rms_norm8_backward(wants(x), kept, rstd, w), lambda: A.rms_norm8_backward(x, kept, rstd, w, grad_sum=wants(x))):
        with pytest.raises(ValueError, match="records no gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError) as refused:
            call()
        assert "records no gradient" not in str(refused.value)
    # weights' gradients from parameters as they are, in a training step written by hand
    with pytest.raises(ValueError) as refused:
        A.linear8_backward(x, p, wants(big))
    assert "records no gradient" not in str(refused.value)


BLOCK_ALONE = BLOCK_FORWARD[:17] + BLOCK_FORWARD[18:]


def test_a_block_without_a_backward_pass(lib):
    """Refusals, and room for the norm's output and the gated rows alone."""
    for at, value in [(5, 2), (6, -1), (6, 1 << 32), (7, 0), (7, 1 << 21), (1, 63), (3, 63), (8, -1.0), (10, 63), (11, 0), (11, 1 << 20),
                      (13, 7), (14, 0), (0, 0), (4, 0), (9, 0), (12, 0), (16, 0), (17, 0), (17, P + 8)]:
        arguments = list(BLOCK_ALONE)
        arguments[at] = value
        assert lib.leap_feed_forward8_alone(*arguments) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error()
    assert lib.leap_feed_forward8_alone_work(4, 64, P, 64, 16, P, 16, 24) == 256 + 16 + 64 + 16
    assert lib.leap_feed_forward8_alone_work(4, 64, P, 65, 16, P, 16, 24) == 256 + 16 + 64 + 16 + 32 * 64 * 2
    assert lib.leap_feed_forward8_alone_work(4, 64, P, 64, 16, P, 16, 0) == 0 and lib.leap_feed_forward8_alone_work(-1, 64, P, 64, 16, P, 16, 8) == 0
    assert lib.leap_feed_forward8_alone(None, 64, None, 64, None, 1, 0, 64, 1e-6, None, 64, 8, None, 8, 16, *[None] * 4) == B.LEAP_OK


def test_bad_arguments_of_finite_unpacking_are_refused_with_a_message(lib):
    for at, value in [(5, 9), (2, -1), (3, 0), (3, 1 << 21), (0, 0), (1, 0), (4, 0)]:
        arguments = [P, P, 4, 64, P, 1, 0]
        arguments[at] = value
        assert lib.leap_unpack8_finite(*arguments) == B.LEAP_INVALID_ARG, (at, value)
        assert lib.leap_last_error()
    assert lib.leap_unpack8_finite(None, None, 0, 64, None, 0, None) == B.LEAP_OK


def test_bad_arguments_around_a_fine_gradient_are_refused_with_a_message(lib):
    for name, good, bad in (
            ("leap_linear8_backward_fine", (P, P, P, 4, 64, P, 64, 8, P, 1, P, P, 0), [(3, -1), (4, 0), (6, 63), (7, 0), (9, 2), (0, 0), (0, P + 8), (1, 0), (2, 0), (5, 0), (11, 0), (11, P + 8)]),
            ("leap_gate8_backward_fine", (P, 8, P, P, 4, 8, P, 0), [(1, 7), (4, -1), (5, 0), (5, 1 << 20), (0, 0), (2, 0), (3, 0), (6, 0), (6, P + 8)]),
            ("leap_linear_gate8_backward_fine", (P, 8, P, 16, 8, P, P, 4, 16, P, P, 0), [(1, 7), (3, 15), (4, 0), (7, -1), (8, 0), (8, 1 << 20), (0, 0), (2, 0), (5, 0), (6, 0), (9, 0), (9, P + 4)])):
        for at, value in bad:
            arguments = list(good)
            arguments[at] = value
            assert getattr(lib, name)(*arguments) == B.LEAP_INVALID_ARG, (name, at, value)
            assert lib.leap_last_error()
    assert lib.leap_linear8_backward_fine_work(P, 5, 64, P, 64, 9) == (16 + 9) * 64 * 2 + 2 * 16 * 64 * 4
    assert lib.leap_linear8_backward_fine_work(P, 5, 64, P, 64, 0) == 0 and lib.leap_linear8_backward_fine_work(P, 0, 343, P, 343, 8) == 0
    assert lib.leap_linear8_backward_fine(None, None, None, 0, 343, None, 343, 8, P, 1, None, None, None) == B.LEAP_OK
