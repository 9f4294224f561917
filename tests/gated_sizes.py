"""Sizes of the gated layer by the kernel that takes them on a card of 256 CUs: (tokens, features in, features out).  Each has whole steps enough for the
kernel's loop to reach its steady state and go round its slots, where the choice leaves as many, and most have a ragged end.  test_gated_kernels.py asserts the choice without a GPU, test_gpu_gated_kernels.py
computes with them."""

BITS16, ALL = ("bf16", "f16"), ("bf16", "f16", "f32")

# kernel: (types, sizes)
FORWARD = {
    "large": [(BITS16, (2_040, 389, 3_901)), (BITS16, (2_048, 384, 3_968))],
    "small": [(BITS16, (2_100, 389, 3_901)), (BITS16, (2_304, 384, 3_712)), (("f32",), (1_100, 230, 2_001)), (("f32",), (1_152, 256, 2_048))],
    "few": [(BITS16, (200, 1_000, 300)), (("f32",), (200, 500, 300)), (BITS16, (128, 640, 256))],
    "few, split": [(ALL, (64, 4_096, 500)), (ALL, (131, 4_101, 77))],
    "rows4": [(BITS16, (24, 3_001, 200)), (BITS16, (5, 3_001, 200)), (("f32",), (24, 1_501, 200)), (("f32",), (8, 1_504, 200))],
    "rows2": [(ALL, (24, 1_000, 8_300)), (ALL, (8, 1_000, 8_300))],
    "rows4, split": [(BITS16, (24, 8_301, 3_200)), (("f32",), (24, 3_101, 3_200))],
}
# (features in are the columns of dx; a sum is of gate and of up, features out of each)
BACKWARD = {
    "large": [(BITS16, (4_090, 4_001, 330)), (BITS16, (4_096, 4_096, 384))],
    "middle": [(BITS16, (8_190, 767, 330)), (BITS16, (8_190, 767, 400)), (BITS16, (8_192, 768, 448))],     # (up's steps begin in each of the three slots)
    "small": [(BITS16, (8_190, 1_001, 330)), (BITS16, (8_192, 1_024, 384)), (("f32",), (2_049, 2_100, 230)), (("f32",), (2_176, 2_048, 256))],
    "few": [(BITS16, (300, 500, 330)), (("f32",), (300, 500, 331)), (BITS16, (128, 512, 352))],
    "few, split": [(ALL, (64, 500, 2_100)), (ALL, (131, 77, 2_111))],
    "rows4": [(ALL, (8, 33_000, 1_300))],
    "rows2": [(ALL, (24, 17_000, 505)), (ALL, (8, 17_000, 505))],
    "rows4, split": [(ALL, (24, 70, 3_001)), (ALL, (5, 70, 3_001))],                                       # (a step or two to a wavefront: there are never more)
    "rows2, split": [(ALL, (24, 12_001, 3_001))],
}


def cases(table):
    """-> [(kernel, type, tokens, features in, features out)]"""
    return [(kernel, dtype, *size) for kernel, entries in table.items() for types, size in entries for dtype in types]
