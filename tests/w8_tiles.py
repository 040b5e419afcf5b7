"""Sizes of 8-bit products that take each kernel and tile on 256 compute units, with what is left over at every border."""

# kernel, 16-row and 16-column pieces of its tile: [(M, K, N)]
TILES = {
    ("rows", 1, 1): [(1, 64, 16), (31, 127, 129), (70, 1000, 33)],
    ("rows", 1, 2): [(64, 9000, 1030), (33, 900, 2000)],
    ("rows", 2, 2): [(300, 2049, 515), (250, 700, 530)],
    ("rows", 4, 2): [(520, 1100, 700), (60, 700, 5000)],
    ("rows", 4, 4): [(250, 1100, 4090), (40, 1089, 9000), (256, 4096, 4096)],
    # whole and partial groups of row tiles, wavefronts and columns that are not there, odd and even counts of 64 rows of W
    ("tiles", 4, 16): [(520, 1100, 2100), (1100, 191, 2071), (45, 200, 8200), (1040, 2100, 3104)],
    ("tiles", 8, 16): [(2100, 300, 4100), (2053, 705, 3001), (3000, 64, 5000), (1025, 4111, 8192)],
}
# rows as far apart as they may be
FAR = {("rows", 2, 2): (300, 200, 600), ("rows", 4, 2): (520, 1100, 700), ("rows", 4, 4): (250, 1100, 4090), ("tiles", 4, 16): (700, 96, 4100),
       ("tiles", 8, 16): (1500, 96, 4100)}
