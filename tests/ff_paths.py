"""Shapes of the gated feed-forward block that together take every way in which it is cut up (csrc/tr_cut.h).

Of every shape: M, K, F, an element's bytes, and what the forward pass, dx and the weights' gradients take: the kernel for few tokens or
the tiles' size, then the parts of a sum.  K is a multiple of 16 bytes or odd: tiles straight to shared memory, or through registers."""

SHAPES = [
    # large tiles of the forward pass
    (4096, 72, 2048, 2, "large 1 small 8 small 8"), (4096, 73, 2048, 2, "large 1 small 8 small 8"),
    (4096, 72, 2048, 4, "large 1 small 8 small 8"), (4096, 73, 2048, 4, "large 1 small 8 small 8"),
    # large tiles of dx, whole
    (4096, 4096, 100, 2, "small 4 large 1 small 4"), (4096, 4091, 100, 2, "small 4 large 1 small 4"),
    (4096, 4096, 100, 4, "small 12 large 1 small 8"), (4096, 4091, 100, 4, "small 12 large 1 small 8"),
    # and in parts
    (1300, 1296, 7400, 2, "small 1 large 7 small 1"), (1300, 1301, 7400, 2, "small 1 large 7 small 1"),
    (1300, 1296, 3700, 4, "small 1 large 7 small 1"), (1300, 1301, 3700, 4, "small 1 large 7 small 1"),
    # large tiles of the weights' gradients, whole
    (100, 2560, 2560, 2, "small 5 small 10 large 1"), (100, 2561, 2560, 2, "small 5 small 10 large 1"),
    (100, 2560, 2560, 4, "small 10 small 12 large 1"), (100, 2561, 2560, 4, "small 10 small 12 large 1"),
    # and in parts
    (13300, 1032, 770, 2, "small 1 small 1 large 6"), (13300, 1033, 770, 2, "small 1 small 1 large 6"),
    (6700, 1032, 770, 4, "small 1 small 1 large 6"), (6700, 1033, 770, 4, "small 1 small 1 large 6"),
    # the forward pass in parts
    (192, 4096, 1024, 2, "small 8 small 4 small 1"), (100, 4096, 3000, 2, "small 5 small 8 small 1"),
    (200, 2056, 1030, 2, "small 4 small 4 small 1"), (192, 4095, 1024, 2, "small 8 small 4 small 1"),
    (200, 2057, 1030, 2, "small 4 small 4 small 1"),
    (200, 2056, 1030, 4, "small 8 small 7 small 1"), (200, 2057, 1030, 4, "small 8 small 7 small 1"),
    # few tokens
    (16, 1000, 160, 2, "few1 1 small 1 small 1"), (16, 1001, 160, 2, "few1 1 small 1 small 1"),
    (16, 1000, 160, 4, "few1 1 small 2 small 1"), (16, 1001, 160, 4, "few1 1 small 2 small 1"),
    (40, 136, 100, 2, "few2 1 small 1 small 1"), (40, 137, 100, 2, "few2 1 small 1 small 1"),
    (40, 136, 100, 4, "few2 1 small 2 small 1"), (40, 137, 100, 4, "few2 1 small 2 small 1"),
    (300, 136, 600, 2, "few4 1 small 1 small 1"), (300, 137, 600, 2, "few4 1 small 1 small 1"),
    (300, 136, 600, 4, "few4 1 small 9 small 2"), (300, 137, 600, 4, "few4 1 small 9 small 2"),
    # small tiles throughout
    (1021, 136, 1030, 2, "small 1 small 4 small 1"), (1021, 137, 1030, 2, "small 1 small 4 small 1"),
    (1021, 136, 1030, 4, "small 1 small 16 small 7"), (1021, 137, 1030, 4, "small 1 small 16 small 7"),
    (3000, 1600, 600, 2, "small 1 small 1 small 1"), (3000, 1601, 600, 2, "small 1 small 1 small 1"),
    (3000, 1600, 600, 4, "small 1 small 1 small 1"), (3000, 1601, 600, 4, "small 1 small 1 small 1"),
]
