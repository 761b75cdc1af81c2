"""Shapes of grouped products that reach each kernel variant, with what they are for; which variant a shape takes is checked on the host
(test_products_rules.py), what it computes on the GPU (test_gpu_products_ways.py)."""

# rows of each expert, N, K -> fragments of 16 rows a pass, fragments of 16 features, wavefronts; rows of an expert beyond a pass make several passes
FEW_ROWS_BF16 = [
    (([1, 1], 192, 8256), (1, 1, 8)),
    (([25] + [1] * 7, 1024, 8256), (1, 1, 8)),                # two passes
    (([0, 17, 0, 1, 0, 0, 1, 13], 576, 10560), (1, 1, 8)),    # two, the second of one row
    (([2, 1, 0, 1], 256, 1024), (1, 1, 4)),
    (([60] + [3] * 63, 1408, 2048), (1, 1, 4)),               # four passes
    (([0] * 62 + [255, 1], 1408, 2112), (1, 1, 4)),           # sixteen
]
FEW_ROWS_FP8 = [
    (([3, 0, 13], 320, 448), (1, 1, 4)),
    (([1], 64, 64), (1, 1, 4)),
    (([27] + [5] * 7, 192, 320), (1, 2, 4)),                  # two passes
    (([27] + [5] * 7, 14336, 4096), (1, 2, 4)),
    (([0, 0, 0, 64, 0, 0, 0, 0], 128, 64), (1, 2, 4)),        # four
    (([31], 192, 320), (2, 2, 4)),                            # a ragged second fragment
    (([1, 0, 24], 704, 1152), (2, 2, 4)),
    (([40] + [8] * 7, 4096, 5056), (2, 2, 4)),                # two passes, the last block of 64
    (([1, 95, 0, 0, 0, 0, 0, 0], 4096, 5056), (2, 2, 4)),     # three
    (([17], 38400, 64), (2, 4, 4)),
    (([40] + [8] * 7, 8192, 2240), (2, 4, 4)),                # two passes, the last block of 64
    (([33, 0, 66, 0, 0, 0, 0, 1], 8192, 2304), (2, 4, 4)),    # three, of one expert two
]
# The small tiles' longest contractions in 8 bits (its scales have room for 56 blocks), and what lies behind them.
SMALL_FP8 = [([40], 64, 7040), ([70], 320, 7040), ([40], 64, 6976), ([100, 0, 33], 320, 6976)]
BEHIND_SMALL_FP8 = [([40], 64, 7104), ([70], 320, 7168)]
# Products whose rows' gradient in 8 bits (the product of exchanged features) takes each way.
GRADIENT_FP8 = [([2, 0, 5], 320, 448, "few"), ([70, 0, 31], 448, 192, "small"), ([600, 31, 450], 2112, 4160, "large"), ([1000, 0, 1], 4160, 2112, "large")]
