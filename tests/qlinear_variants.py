"""Sizes at which a call takes each kernel of many rows: (rows, in, out, gated, products, output, e4m3 instructions, tile, shares of the contraction).  tests/test_host_qlinear_products.py checks that they do, and
tests/test_gpu_qlinear_products.py what comes out."""
TILES = ("128x256", "64x256", "64x128", "32x128", "32x256")      # in the order of QTile
AUTO, WHOLE, E4M3 = 0, 1, 2

VARIANTS = [
    # outputs in fp32 with e4m3 instructions, as the layers of bf16 contexts have them
    (433, 300, 14250, 0, E4M3, "fp32", 1, "128x256", 1),
    (1001, 8449, 6900, 0, E4M3, "fp32", 1, "128x256", 1),
    (129, 200, 13030, 0, E4M3, "fp32", 1, "64x256", 1),
    (65, 515, 11200, 0, E4M3, "fp32", 1, "64x128", 1),
    (65, 2100, 11190, 0, E4M3, "fp32", 1, "64x128", 2),
    (67, 5130, 11200, 0, E4M3, "fp32", 1, "64x128", 4),
    (65, 129, 5101, 0, E4M3, "fp32", 1, "32x128", 1),
    (65, 2100, 5710, 0, E4M3, "fp32", 1, "32x128", 2),
    (67, 3201, 5709, 0, E4M3, "fp32", 1, "32x128", 4),
    # outputs in bf16 of products that enter their sums whole
    (433, 300, 14250, 0, WHOLE, "bf16", 0, "128x256", 1),
    (1001, 8449, 6900, 0, WHOLE, "bf16", 0, "128x256", 1),
    (601, 200, 9980, 0, WHOLE, "bf16", 0, "64x256", 1),
    (257, 515, 14860, 0, WHOLE, "bf16", 0, "64x128", 1),
    (99, 4100, 16690, 0, WHOLE, "bf16", 0, "64x128", 2),
    (65, 129, 7541, 0, WHOLE, "bf16", 0, "32x128", 1),
    (65, 300, 11200, 0, WHOLE, "bf16", 0, "32x128", 2),
    (67, 3201, 5709, 0, WHOLE, "bf16", 0, "32x128", 4),
    # with a gate
    (129, 1281, 13640, 1, WHOLE, "", 0, "128x256", 1),
    (641, 8449, 5700, 1, WHOLE, "", 0, "128x256", 1),
    (65, 700, 11200, 1, WHOLE, "", 0, "64x256", 1),
    (129, 8449, 2600, 1, WHOLE, "", 0, "64x256", 1),
    (65, 100, 100, 1, WHOLE, "", 0, "32x256", 1),
    # what the other choices are where nothing is said
    (129, 1281, 13640, 1, AUTO, "", 1, "128x256", 1),
    (65, 700, 11200, 1, E4M3, "", 1, "64x256", 1),
    (433, 300, 14250, 0, AUTO, "bf16", 1, "128x256", 1),
    (433, 300, 14250, 0, AUTO, "fp32", 0, "128x256", 1),
    (433, 300, 14250, 0, WHOLE, "fp32", 0, "128x256", 1),
    (433, 300, 14250, 0, E4M3, "bf16", 1, "128x256", 1),
    (64, 900, 16300, 0, E4M3, "bf16", 0, "32x128", 2),
]
