"""What the operators on activations in 8 bits launch, on the CPU (tests/launches.py): how many blocks, of which kernels."""
import pytest

import activation_kernels as K
from launches import kernels, record
from paper_2307_05801_amd import binding as B

P = 0x1000


def test_a_launch_has_fewer_than_2_32_threads():
    """Many short rows (2^30 voxels of 8 channels), many long ones, a weight of 2^31 values: in several launches that cover them."""
    rows = (1 << 30) + 5
    calls = [                                              # and by how many blocks' worth of the first kernel named they are covered
        ("leap_rms_norm8", (P, 8, P, 8, 1, P, 1, rows, 8, 1e-6, P, P, P, P, P, P, 0), "k_norm", -(-rows // 32)),
        ("leap_rms_norm8", (P, 512, None, 0, 1, P, 0, (1 << 27) + 1, 512, 1e-6, None, P, P, None, None, None, 0), "k_norm", -(-((1 << 27) + 1) // 4)),
        ("leap_rms_norm8", (P, 4096, P, 4096, 1, P, 1, (1 << 25) + 1, 4096, 1e-6, P, P, P, P, P, P, 0), "k_norm_long", (1 << 25) + 1),
        ("leap_rms_norm8_backward", (P, 1, 4096, P, 4096, 1, P, P, P, P, 1, (1 << 25) + 1, 4096, P, P, P, 0), "k_norm_grad_long", (1 << 25) + 1),
        ("leap_rms_norm8_backward", (P, 1, 8, P, 8, 1, P, P, P, P, 1, rows, 8, P, P, P, 0), "k_norm_grad", 1024),
        ("leap_pack8", (P, 1, 8, rows, 8, P, P, 0), "k_pack", None),
        ("leap_unpack8", (P, P, rows, 8, P, 1, 0), "k_unpack", None),
        ("leap_linear8", (P, P, rows, 8, P, 8, 8, P, P, 0), "k_lay_out", -(-rows // 256)),
        ("leap_linear8", (P, P, 1 << 27, 8200, P, 8200, 8, P, P, 0), "k_lay_out", (1 << 27) * 513 // 256),
        ("leap_linear8_backward", (P, 8, P, P, 0, 1 << 15, P, 1 << 15, 1 << 16, P, 1, P, P, 0), "k_add_parts", 1 << 25),
        ("leap_gate8_backward", (P, 8, P, P, rows, 8, P, 0), "k_gate_grad", -(-rows * 4 // 256)),
        ("leap_gated_linear8_backward", (P, 3, P, P, P, P, rows, 8, P, 8, 3, P, 1, P, P, 0), "k_gate_grad", -(-rows * 4 // 256)),
        ("leap_linear_gate8_backward", (P, 8, P, 8, 8, P, P, (1 << 32) + 5, 8, P, P, 0), "k_product", (1 << 25) + 1),
        ("leap_linear_gate8_backward_fine", (P, 8, P, 8, 8, P, P, (1 << 32) + 5, 8, P, P, 0), "k_product", (1 << 25) + 1),
        ("leap_feed_forward8_backward", (P, 8, P, 8, P, 1, rows, 8, P, 8, 3, P, 3, 8, P, P, P, P, P, P, 0), "k_pad_rows", -(-rows // 256)),
    ]
    for (name, arguments, kernel, blocks), (status, launches) in zip(calls, record([c[:2] for c in calls])):
        assert status == B.LEAP_OK, name
        for launch in launches:
            across, along, deep = launch.blocks
            assert across * launch.threads < 1 << 32 and along < 1 << 16 and deep == 1, (name, launch)
        mine = sum(launch.blocks[0] for launch in launches if launch.kernel == kernel)
        assert mine == blocks or blocks is None and mine, (name, kernel, mine, blocks)


def _call(what, rows, cols, out):
    if what == K.Y:
        return "leap_linear8", (P, P, rows, cols, P, cols, out, P, P, 0)
    if what == K.GATED:
        return "leap_gated_linear8", (P, P, rows, cols, P, cols, out, P, P, P, P, P, 0)
    if what in (K.GRAD_X, K.GRAD_X_FULL, K.GRAD_WEIGHT):
        weight = what == K.GRAD_WEIGHT
        return "leap_linear8_backward", (P, out, P, P, rows, cols, P, cols, out, None if weight else P, 0 if what == K.GRAD_X_FULL else 1, P if weight else None, P, 0)
    return "leap_linear_gate8_backward" + ("_fine" if what == K.GATE_GRAD_FINE else ""), (P, out, P, cols, out, P, P, rows, cols, P, P, 0)


def test_sizes_take_the_kernels_they_are_there_for():
    """And every kernel of the product is there: one that no size takes has no test of its values (test_gpu_activation_kernels.py)."""
    taken = set()
    for (what, rows, cols, out, parameters), (status, launches) in zip(K.CASES, record([_call(*c[:4]) for c in K.CASES])):
        assert status == B.LEAP_OK
        products = [launch.parameters for launch in launches if launch.kernel == "k_product"]
        assert parameters in products, (what, rows, cols, out, products)
        taken.add(("k_product", parameters))
    assert taken == {k for k in kernels() if k[0] == "k_product"}
