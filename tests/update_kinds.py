"""Stacks of matrices that between them reach every kind of tiles in each of an update's three products, with operands of one plane and
of pairs: (batch, rows, cols, products, kinds of X X^T, of the polynomial, of the product that updates X)."""

KINDS = ("few", "small", "middle", "large")
FP16, SPLIT = 0, 1  # SPO_PRODUCTS_*
STACKS = [
    (5, 130, 130, FP16, "few", "few", "few"),
    (32, 310, 318, FP16, "small", "few", "small"),
    (64, 250, 256, FP16, "small", "small", "small"),
    (64, 441, 507, FP16, "large", "small", "large"),
    (64, 500, 509, FP16, "large", "large", "large"),
    (16, 930, 955, FP16, "middle", "middle", "large"),
    (64, 190, 955, FP16, "few", "few", "large"),
    (1, 4096, 4096, FP16, "middle", "middle", "large"),
    (4, 1024, 4096, FP16, "few", "small", "large"),
    (5, 130, 130, SPLIT, "few", "few", "few"),
    (64, 250, 256, SPLIT, "small", "few", "small"),
    (64, 310, 318, SPLIT, "small", "small", "few"),
    (3, 60, 5500, SPLIT, "few", "few", "small"),
    (6, 190, 5500, SPLIT, "few", "few", "large"),
    (16, 930, 955, SPLIT, "middle", "middle", "large"),
    (64, 500, 509, SPLIT, "large", "large", "large"),
]
