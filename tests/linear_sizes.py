"""Products that reach each kernel: rows, channels, k and whether in 8 bits, on a chip of 256 CUs, for tests of the choice (on the host) and of the
kernels (on the GPU).  Sizes beside a tile's, k that leaves part of a piece, a step or a share."""
SIZES = {
    "any": [(5, 70, 7, False), (130, 65, 15, True), (70, 3, 1, False)],
    "few11": [(1, 300, 1000, False), (16, 1000, 531, True), (3, 17, 8, False), (222, 26, 286, True)],
    "few21": [(50, 1043, 110, False), (31, 2962, 66, True), (669, 129, 150, False)],
    "few22": [(209, 617, 91, False), (66, 1946, 201, False), (1340, 184, 144, True)],
    "few24": [(721, 489, 63, False), (1004, 465, 99, False), (1334, 289, 65, True)],
    "tile64": [(1323, 474, 125, False), (296, 3396, 209, False), (551, 4542, 134, True)],
    "tile64 shares": [(25, 215, 4524, False), (293, 345, 2683, False), (1685, 311, 2249, True)],
    "tile128": [(1193, 4916, 78, False), (1291, 4857, 203, False), (1405, 4779, 74, True)],
    "tile128 shares": [(512, 3322, 3329, False), (2474, 580, 2890, False)],
    "tile192": [(3236, 2694, 90, False), (3873, 4524, 114, False), (2018, 4209, 91, True)],
    "tile256": [(4110, 3091, 91, False), (3178, 4553, 171, False), (4415, 2859, 71, True)],
}
