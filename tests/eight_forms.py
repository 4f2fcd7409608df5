"""Sizes of products in 8 bits that together reach every kernel behind dlcx_fp8_product, with what they run as.

(rows, m, n), result type, (form, tile, splits) as dlcx_fp8_product_plan gives them.  All but the smallest sums have more
than eight blocks of 128, so a ring of stages comes round and scales are read again, and they end inside a quad of blocks
and inside a block."""
FEW, RING, TILES, WIDE = 0, 1, 2, 3
F32, BF16 = "f32", "bf16"

FORMS = [
    ((1, 90, 300), F32, (FEW, 1, 1)), ((3, 33600, 1200), F32, (FEW, 2, 1)), ((16, 300, 2100), F32, (FEW, 4, 1)),
    ((1, 90, 300), BF16, (FEW, 1, 1)), ((3, 33600, 1200), BF16, (FEW, 2, 1)), ((16, 300, 2100), BF16, (FEW, 4, 1)),
    ((5, 65536, 1200), F32, (FEW, 1, 1)), ((5, 65536, 1200), BF16, (FEW, 1, 1)),
    ((20, 33000, 1300), F32, (RING, 32, 1)), ((20, 90, 5200), F32, (RING, 32, 11)),
    ((64, 20500, 1500), F32, (RING, 64, 1)), ((60, 300, 4000), F32, (RING, 64, 8)),
    ((96, 20500, 1300), F32, (RING, 96, 1)), ((90, 640, 2900), F32, (RING, 96, 6)),
    ((128, 20500, 1300), F32, (RING, 128, 1)), ((126, 80, 2880), F32, (RING, 128, 6)), ((128, 1021, 11000), F32, (RING, 128, 22)),
    ((20, 33000, 1300), BF16, (RING, 32, 1)), ((20, 90, 5200), BF16, (RING, 32, 11)),
    ((64, 20500, 1500), BF16, (RING, 64, 1)), ((60, 300, 4000), BF16, (RING, 64, 8)),
    ((96, 20500, 1300), BF16, (RING, 96, 1)), ((90, 640, 2900), BF16, (RING, 96, 6)),
    ((128, 20500, 1300), BF16, (RING, 128, 1)), ((126, 80, 2880), BF16, (RING, 128, 6)), ((128, 1021, 11000), BF16, (RING, 128, 11)),
    ((1024, 4096, 1100), BF16, (RING, 128, 1)), ((2050, 1021, 4133), BF16, (RING, 128, 1)),
    ((1000, 4000, 1100), F32, (TILES, 64, 1)), ((520, 1000, 2500), F32, (TILES, 64, 5)),
    ((4096, 2048, 1111), F32, (TILES, 128, 1)), ((2050, 1021, 4133), F32, (TILES, 128, 3)),
    ((300, 130, 1300), BF16, (TILES, 64, 1)), ((520, 1000, 2500), BF16, (TILES, 64, 3)),
    ((200, 28672, 1100), BF16, (TILES, 128, 1)), ((3000, 700, 6000), BF16, (TILES, 128, 3)),
    ((4096, 2048, 1000), BF16, (WIDE, 256, 1)), ((4096, 2048, 1111), BF16, (WIDE, 256, 1)),
    ((4000, 2300, 1300), BF16, (WIDE, 256, 1)), ((3000, 2816, 1700), BF16, (WIDE, 256, 1)),
]
