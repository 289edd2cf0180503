"""Sizes of matrices by the tiles that their products take: X X^T and A A (symmetric), P X and the result, each as the
tile's side and whether its sums are cut into parts."""
# rows, columns, (X X^T, A A, P X and the result)
SIZES = [
    (960, 2560, ((128, True), (32, False), (128, False))),  # an odd number of 64: the last tiles are half empty
    (2560, 960, ((128, True), (32, False), (128, False))),
    (1000, 2700, ((128, True), (64, False), (128, False))),
    (1472, 1472, ((128, True), (128, True), (128, False))),
    (1930, 1921, ((128, False), (128, False), (128, False))),
    (450, 3072, ((64, True), (32, False), (64, False))),
    (4090, 390, ((64, True), (32, False), (64, False))),  # an odd number of 64
    (576, 3648, ((64, True), (32, False), (128, False))),
    (1000, 1100, ((64, False), (64, False), (64, False))),
    (1130, 1030, ((64, False), (64, False), (64, False))),
]
