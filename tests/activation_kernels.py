"""Sizes that take each of the product's kernels: (what, rows, columns, outputs, the kernel's parameters).

The parameters are those of k_product: how its operands lie (0 bfloat16 along the sum, 1 across, 2 codes along, 3 across), what becomes of the
result (0 bfloat16, 1 float, 2 gated, 3 the gate's gradient, 4 the same, fine), the tile, the waves that share it, groups of them, buffers.
Sums are of 17 steps of 64 and more, over the border of two tiles where a block takes several; sizes are odd ones and whole tiles."""

Y, GRAD_X, GRAD_X_FULL, GRAD_WEIGHT, GATED, GATE_GRAD, GATE_GRAD_FINE = "y", "grad_x", "grad_x in 32 bits", "grad_weight", "gated", "gate's gradient", "fine gate's gradient"

LARGE, SMALL = (256, 256, 2, 4, 1, 2), (128, 128, 2, 2, 1, 2)
PAIRED, PAIRED3, PAIRED_LOW = (128, 128, 2, 2, 2, 2), (128, 128, 2, 2, 2, 3), (128, 64, 2, 2, 2, 3)

CASES = [
    (Y, 33000, 1100, 1000, (0, 2, 0) + LARGE),
    (Y, 35072, 1152, 1024, (0, 2, 0) + LARGE),
    (Y, 18414, 1100, 1029, (0, 2, 0) + SMALL),
    (Y, 18432, 1152, 1024, (0, 2, 0) + SMALL),
    (Y, 3000, 1100, 700, (0, 2, 0) + PAIRED3),
    (Y, 1000, 1100, 1300, (0, 2, 0) + PAIRED_LOW),
    (Y, 77, 2300, 130, (0, 2, 1) + PAIRED_LOW),                # in parts
    (GATED, 18414, 1100, 1029, (0, 2, 2) + LARGE),
    (GATED, 18432, 1152, 1024, (0, 2, 2) + LARGE),
    (GATED, 12000, 1090, 1000, (0, 2, 2) + SMALL),
    (GATED, 1000, 1100, 1300, (0, 2, 2) + PAIRED3),
    (GATED, 300, 1090, 520, (0, 2, 2) + PAIRED_LOW),
    (GRAD_X, 33000, 1030, 1100, (1, 0, 0) + LARGE),
    (GRAD_X, 35072, 1024, 1152, (1, 0, 0) + LARGE),
    (GRAD_X, 18414, 1100, 1029, (1, 0, 0) + SMALL),
    (GRAD_X, 3000, 1100, 1100, (1, 0, 0) + PAIRED),
    (GRAD_X, 1000, 1100, 1300, (1, 0, 0) + PAIRED_LOW),
    (GRAD_X, 77, 130, 2300, (1, 0, 1) + PAIRED_LOW),           # in parts
    (GRAD_X_FULL, 52000, 1030, 1100, (1, 0, 1) + LARGE),       # 214 MB: past the caches
    (GRAD_X_FULL, 33000, 1030, 1100, (1, 0, 1) + LARGE),
    (GRAD_X_FULL, 18414, 1100, 1029, (1, 0, 1) + SMALL),
    (GRAD_X_FULL, 3000, 1100, 1100, (1, 0, 1) + PAIRED),
    (GRAD_X_FULL, 1000, 1100, 1300, (1, 0, 1) + PAIRED_LOW),
    (GRAD_WEIGHT, 18414, 1100, 1029, (3, 1, 1) + LARGE),
    (GRAD_WEIGHT, 18432, 1152, 1024, (3, 1, 1) + LARGE),
    (GRAD_WEIGHT, 2100, 1100, 16400, (3, 1, 0) + LARGE),
    (GRAD_WEIGHT, 9000, 1100, 515, (3, 1, 1) + SMALL),
    (GRAD_WEIGHT, 1100, 2100, 2100, (3, 1, 0) + SMALL),
    (GATE_GRAD, 18414, 1100, 1029, (1, 0, 3) + SMALL),
    (GATE_GRAD, 50000, 1024, 1152, (1, 0, 3) + SMALL),         # 205 MB: past the caches
    (GATE_GRAD, 3000, 1100, 1100, (1, 0, 3) + PAIRED),
    (GATE_GRAD, 1000, 1100, 1300, (1, 0, 3) + PAIRED_LOW),
    (GATE_GRAD_FINE, 25000, 1024, 1152, (1, 0, 4) + SMALL),    # 205 MB: past the caches
    (GATE_GRAD_FINE, 9000, 1029, 1100, (1, 0, 4) + SMALL),
    (GATE_GRAD_FINE, 3000, 1100, 1100, (1, 0, 4) + PAIRED),
    (GATE_GRAD_FINE, 1000, 1100, 1300, (1, 0, 4) + PAIRED_LOW),
]
