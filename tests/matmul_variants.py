"""Sizes that reach each kernel of the matrix product over several stages, with ragged edges and a
ragged end of the reduction, and the plan that each is meant to get."""

# name, type, pass, (M, N, K), whether the operands lie on 16 bytes, (tile, splits, stages, groups)
VARIANTS = [
    # 256 x 256, eight waves: one stage, as many as its two buffers, more
    ("256 one stage", "bf16", "forward", (3590, 3608, 40), True, (256, 1, 1, 1)),
    ("256 two stages", "bf16", "dx", (3590, 72, 3608), True, (256, 1, 2, 1)),
    ("256", "bf16", "forward", (3590, 3608, 328), True, (256, 1, 6, 1)),
    ("256", "bf16", "dx", (3590, 200, 3608), True, (256, 1, 4, 1)),
    ("256", "bf16", "dw", (203, 3592, 3608), True, (256, 1, 4, 1)),
    # 128 x 128 with two groups of waves: a second group of fewer stages, of a single one, of none in
    # the last split
    ("two groups, one split", "bf16", "forward", (2000, 1992, 1080), True, (128, 1, 9, 2)),
    ("two groups, one split", "bf16", "dx", (2000, 1080, 1992), True, (128, 1, 9, 2)),
    ("two groups, one split", "bf16", "dw", (1075, 2000, 1992), True, (128, 1, 9, 2)),
    ("two groups, splits", "bf16", "forward", (1000, 1016, 4104), True, (128, 4, 9, 2)),
    ("two groups, splits", "bf16", "dx", (1000, 4104, 1016), True, (128, 4, 9, 2)),
    ("two groups, splits", "bf16", "dw", (4100, 1000, 1016), True, (128, 4, 9, 2)),
    ("two groups, an idle one", "bf16", "forward", (500, 504, 16400), True, (128, 15, 9, 2)),
    ("two groups, an idle one", "bf16", "dx", (500, 16400, 504), True, (128, 15, 9, 2)),
    ("two groups, an idle one", "bf16", "dw", (16395, 496, 504), True, (128, 15, 9, 2)),
    # 128 x 128 with one group: parts of the reduction, the last a stage shorter, or the whole of it
    ("128, splits", "bf16", "forward", (1500, 1496, 3944), True, (128, 3, 21, 1)),
    ("128, splits", "bf16", "dx", (1500, 3944, 1496), True, (128, 3, 21, 1)),
    ("128, splits", "bf16", "dw", (3931, 1504, 1496), True, (128, 3, 21, 1)),
    ("128", "bf16", "forward", (2000, 1992, 936), True, (128, 1, 15, 1)),
    ("128", "bf16", "dx", (2000, 936, 1992), True, (128, 1, 15, 1)),
    ("128", "bf16", "dw", (931, 2000, 1992), True, (128, 1, 15, 1)),
    ("128 without DMA", "bf16", "forward", (2000, 2001, 333), False, (128, 1, 6, 1)),
    ("128 without DMA", "bf16", "dx", (2000, 333, 2001), False, (128, 1, 6, 1)),
    ("128 without DMA", "bf16", "dw", (333, 2000, 2001), False, (128, 1, 6, 1)),
    ("128", "fp32", "forward", (2048, 2040, 520), True, (128, 1, 17, 1)),
    ("128", "fp32", "dx", (2048, 516, 2040), True, (128, 1, 17, 1)),
    ("128", "fp32", "dw", (515, 2048, 2040), True, (128, 1, 17, 1)),
    ("128 without DMA", "fp32", "forward", (4093, 2037, 517), False, (128, 1, 17, 1)),
    ("128 without DMA", "fp32", "dx", (4093, 517, 2037), False, (128, 1, 17, 1)),
    ("128 without DMA", "fp32", "dw", (517, 4093, 2037), False, (128, 1, 17, 1)),
]


def product(which, M, N, K):
    """(R, C, T) of the product: outputs along both directions and the length of the sum."""
    return {"forward": (N, M, K), "dx": (K, M, N), "dw": (K, N, M)}[which]
