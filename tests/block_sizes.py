"""Sizes of the feed-forward block's products that together reach every variant of
the tile product: what the host tests count is what the GPU tests run."""

# rows, in, out; operands along the reduction and across it
LINEAR = {
    # tiles of 64, 128 (two and four steps in LDS), 256; split tiles of 64 and 128
    "bf16": [(257, 257, 257), (2050, 257, 2050), (1030, 2050, 3000), (3000, 257, 4100), (3080, 264, 4104),
             (257, 2050, 257), (385, 40000, 385)],
    "f16": [(257, 257, 257), (2050, 257, 2050), (1030, 2050, 3000), (3000, 257, 4100), (3080, 264, 4104),
            (257, 2050, 257), (385, 40000, 385)],
    # as they lie and split; in parts by 64 and 128, split by 64 and 128
    "f32": [(257, 257, 257), (257, 520, 257), (385, 385, 385), (1030, 385, 3000), (385, 1030, 777),
            (1030, 2050, 1030)],
}
# two gradients at once, and one after the other by the tiles above
LINEAR_BACKWARD = {
    "bf16": [(257, 257, 257), (4100, 3000, 257), (257, 3000, 4100), (1030, 3000, 2050), (2050, 3000, 1030),
             (40000, 385, 385)],
    "f16": [(257, 257, 257), (4100, 3000, 257), (257, 3000, 4100), (1030, 3000, 2050), (2050, 3000, 1030),
            (40000, 385, 385)],
    "f32": [(257, 257, 257), (257, 257, 520), (2050, 1030, 4100), (257, 3000, 1030)],
}
# matrices, rows, cols
UPDATES = [(1, 100, 100), (1, 257, 100), (1, 100, 777), (1, 777, 100), (12, 100, 4100), (12, 4100, 100),
           (3, 777, 4100), (3, 4100, 777), (1, 1030, 3000), (1, 3000, 1030), (3, 1030, 4100), (3, 4100, 1030),
           (3, 2050, 1536), (3, 3000, 2050), (12, 2050, 1536)]
# updates of two bytes that take several steps at once: sides, steps, spectrum
GROUPED = [((520, 4100), 2, "full"), ((520, 4100), 7, "falling"), ((520, 8200), 4, "low"),
           ((4100, 520), 5, "falling"), ((1030, 4104), 3, "low"), ((1030, 4104), 6, "full"),
           ((2048, 8192), 5, "full"), ((8192, 2048), 5, "falling")]
