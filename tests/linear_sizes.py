"""Sizes at which the linear layer's tiled products take each of their tiles: (rows, inputs, outputs, pad, dtypes) and,
for the products x W^T (y, or z of the gradient), dz W (g_x) and dz^T x (g_weight), the tile and whether the sum is cut.
None: streamed, or not looked at."""
ALL, SHORT, FLOAT = ("f32", "bf16", "f16"), ("bf16", "f16"), ("f32",)
KINDS = ("y", "g_x", "g_weight")

T256, T128, P128, T64, P64 = (256, 256, False), (128, 128, False), (128, 128, True), (64, 64, False), (64, 64, True)
TALL, TALL_PARTS, FLAT, FLAT_PARTS = (128, 32, False), (128, 32, True), (32, 128, False), (32, 128, True)

SIZES = [
    # 256: sums of two, three and five steps of 64
    *[(3592, d, 4040, 0, SHORT, (T256, None, None)) for d in (128, 192, 320)],
    *[(3592, 4040, d, 0, SHORT, (None, T256, None)) for d in (128, 192, 320)],
    *[(d, 4040, 3592, 0, SHORT, (None, None, T256)) for d in (128, 192, 320)],
    # 128, whole: odd strides, sums that end inside a step
    (2600, 300, 2605, 3, ALL, (T128, None, None)),
    (2600, 2605, 300, 3, ALL, (None, T128, None)),
    (300, 2605, 2600, 3, ALL, (None, None, T128)),
    (2600, 321, 2600, 0, FLOAT, (T128, None, None)),
    # 128 in parts
    (1000, 4500, 1003, 1, ALL, (P128, None, None)),
    (1003, 1000, 4500, 0, ALL, (None, P128, None)),
    (4500, 1003, 1000, 1, ALL, (None, None, P128)),
    # 64, whole and in parts
    (2000, 200, 500, 3, ALL, (T64, None, None)),
    (90, 1000, 1000, 0, ALL, (P64, P64, None)),
    (2000, 300, 500, 0, ALL, (None, None, P64)),
    # narrow
    (60000, 272, 20, 1, ALL, (TALL, None, FLAT_PARTS)),
    (300, 1100, 24, 5, ALL, (TALL_PARTS, None, FLAT)),
    (24, 900, 1100, 5, ALL, (None, FLAT_PARTS, None)),
    (20011, 9, 300, 0, ALL, (None, TALL, TALL_PARTS)),
    # few rows whose sums are long
    (24, 5000, 300, 5, ALL, (FLAT_PARTS, None, None)),
    (16, 9001, 16, 0, ALL, (P64, None, None)),
    (1, 20000, 40, 0, ALL, (P64, None, None)),
    (50, 2100, 130, 0, ALL, (P64, None, None)),
]
