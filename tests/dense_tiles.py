"""Sizes whose launches reach each tile of the dense operators' products, whole and with a split
contraction, with one item a block and several, at widths that are and are not multiples of 8.

A case: kind, dtype, tokens, inputs, outputs, and what the launches are: for the forward product, dx
and dW the tile's columns (256, 128, and for bf16 64 of 128 x 64), "whole" or "split", and "many"
where a block has several items (bf16; a tile of 256 has a compute unit to itself).  tests/test_dense_plan.py holds the library's choice to
these on the host, tests/test_gpu_dense_tiles.py runs them.
"""

W, S = "whole", "split"

CASES = [
    # bf16, forward of large tiles: rows of whole and of partial pieces, split
    ("linear", "bf16", 16739, 776, 1200, dict(forward=(256, W, "many"))),
    ("linear", "bf16", 15155, 192, 1589, dict(forward=(256, W, "many"))),
    ("linear", "bf16", 15248, 784, 1338, dict(forward=(256, W, "many"), dx=(256, W, ""))),
    ("linear", "bf16", 16594, 2678, 192, dict(forward=(256, S, ""), dx=(256, W, "many"))),
    ("linear", "bf16", 11113, 3448, 259, dict(forward=(256, S, ""), dx=(256, W, "many"))),
    ("linear", "bf16", 17232, 192, 392, dict(forward=(128, W, "many"))),
    ("linear", "bf16", 17904, 208, 402, dict(forward=(128, W, "many"))),
    ("linear", "bf16", 1984, 2011, 278, dict(forward=(128, S, ""))),
    ("gated", "bf16", 3520, 192, 3488, dict(forward=(256, W, "many"))),
    ("gated", "bf16", 2054, 808, 4824, dict(forward=(256, W, "many"), dw=(256, W, ""))),
    ("gated", "bf16", 10320, 792, 975, dict(forward=(256, W, "many"), dx=(256, W, ""))),
    ("gated", "bf16", 13535, 192, 916, dict(forward=(256, W, "many"))),
    ("gated", "bf16", 8264, 3048, 216, dict(forward=(256, S, ""), dx=(256, W, "many"))),
    ("gated", "bf16", 4688, 2944, 401, dict(forward=(256, S, ""))),
    ("gated", "bf16", 13072, 7280, 264, dict(forward=(256, S, "many"), dx=(256, W, "many"), dw=(256, S, ""))),
    ("gated", "bf16", 18816, 192, 200, dict(forward=(128, W, "many"))),
    ("gated", "bf16", 14208, 208, 258, dict(forward=(128, W, "many"))),
    ("gated", "bf16", 1424, 1972, 200, dict(forward=(128, S, ""))),
    # bf16, gradients of large tiles
    ("linear", "bf16", 17877, 192, 2800, dict(dx=(256, S, ""))),
    ("linear", "bf16", 11584, 261, 3000, dict(dx=(256, S, ""))),
    ("linear", "bf16", 16640, 396, 7206, dict(forward=(256, W, "many"), dx=(256, S, "many"), dw=(256, S, ""))),
    ("linear", "bf16", 256, 3720, 7552, dict(dw=(256, W, "many"))),
    ("linear", "bf16", 304, 1669, 7096, dict(dw=(256, W, ""))),
    ("linear", "bf16", 2624, 520, 6904, dict(dw=(256, S, ""))),
    ("linear", "bf16", 2936, 526, 6608, dict(dw=(256, S, ""))),
    ("linear", "bf16", 13864, 7232, 536, dict(forward=(256, S, "many"), dx=(256, W, "many"), dw=(256, S, "many"))),
    ("gated", "bf16", 16606, 192, 1368, dict(forward=(256, W, "many"), dx=(256, S, ""))),
    ("gated", "bf16", 12144, 272, 5760, dict(forward=(256, W, "many"), dx=(256, S, ""), dw=(256, S, "many"))),
    ("gated", "bf16", 12352, 272, 6285, dict(forward=(256, W, "many"), dx=(256, S, "many"), dw=(256, S, ""))),
    ("gated", "bf16", 256, 3528, 3544, dict(dw=(256, W, "many"))),
    ("gated", "bf16", 256, 3503, 3576, dict(dw=(256, W, "many"))),
    # bf16 blocks of several items in the smaller tiles
    ("linear", "bf16", 1040, 132, 7480, dict(forward=(64, W, "many"))),
    ("linear", "bf16", 4672, 178, 1703, dict(forward=(64, W, "many"))),
    ("gated", "bf16", 408, 129, 8296, dict(forward=(64, W, "many"))),
    ("gated", "bf16", 782, 176, 4747, dict(forward=(64, W, "many"))),
    ("gated", "bf16", 16, 7816, 8432, dict(forward=(64, S, "many"))),
    ("linear", "bf16", 1466, 5623, 144, dict(dx=(64, W, "many"))),
    ("linear", "bf16", 8352, 931, 134, dict(dx=(128, W, "many"))),
    ("linear", "bf16", 16640, 64, 8256, dict(dx=(128, S, "many"))),
    ("linear", "bf16", 168, 8556, 931, dict(dw=(64, W, "many"))),
    ("linear", "bf16", 136, 8033, 1032, dict(dw=(128, W, "many"))),
    ("linear", "bf16", 19600, 1, 6650, dict(dw=(128, S, "many"))),
    ("gated", "bf16", 2210, 3665, 64, dict(dx=(64, W, "many"))),
    ("gated", "bf16", 18848, 449, 1, dict(dx=(128, W, "many"))),
    ("gated", "bf16", 17952, 64, 4480, dict(dx=(128, S, "many"))),
    ("gated", "bf16", 192, 2380, 1672, dict(dw=(64, W, "many"))),
    ("gated", "bf16", 136, 1017, 4144, dict(dw=(128, W, "many"))),
    ("gated", "bf16", 3200, 1, 8791, dict(dw=(128, S, "many"))),
    # fp32 tiles of 128 (those of 64 are every small call's)
    ("linear", "f32", 4320, 104, 728, dict(forward=(128, W, ""))),
    ("linear", "f32", 1360, 112, 2253, dict(forward=(128, W, ""))),
    ("linear", "f32", 2160, 1347, 80, dict(forward=(128, S, ""), dx=(128, W, ""), dw=(128, S, ""))),
    ("linear", "f32", 2896, 69, 684, dict(dx=(128, S, ""))),
    ("linear", "f32", 105, 2657, 1160, dict(dw=(128, W, ""))),
    ("gated", "f32", 5512, 104, 181, dict(forward=(128, W, ""))),
    ("gated", "f32", 1280, 1185, 24, dict(forward=(128, S, ""))),
    ("gated", "f32", 2816, 78, 341, dict(dx=(128, S, ""))),
    ("gated", "f32", 4928, 603, 40, dict(dx=(128, W, ""))),
    ("gated", "f32", 104, 1538, 984, dict(dw=(128, W, ""))),
    ("gated", "f32", 1552, 66, 960, dict(dw=(128, S, ""))),
]
