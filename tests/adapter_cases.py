"""Calls of the adapters that go round the kernels' loops as often as large ones do, and how often that is: (sequences' lengths, adapters, number of
adapters, rank, K, N, matrices) and the rows of a tile, the slices of its columns, the rounds of a wavefront in one, the rows of a piece of the sums."""

# sums over tokens: pieces of 16, 4, 8 and 128 steps of 32 tokens; the last piece is not a multiple of a step
SUMS = [
    (([4100, 3000, 0, 1109], [0, 1, 0, 0], 2, 64, 512, 512, 8), 512),
    (([8201], [0], 1, 16, 264, 520, 2), 128),
    (([4133], [0], 1, 120, 264, 136, 8), 256),
    (([131172], [0], 1, 8, 8, 8, 8), 4096),
]
# one slice, of which a wavefront takes several shares of the columns: `wide` is N forward and K backward, the other one is `narrow`
NARROW, WIDE = 136, 1160
ROUNDS = [
    (([333, 0, 300], [1, 0, 0], 2, 16), 16, 1, 3),
    (([333, 0, 300], [1, 0, 0], 2, 24), 16, 1, 3),
    (([700, 613], [1, 0], 2, 32), 32, 1, 3),
    (([700, 613], [0, 1], 2, 64), 32, 1, 3),
    (([150, 101], [0, 1], 2, 64), 16, 4, 2),
    (([333, 0, 300], [1, 0, 0], 2, 128), 16, 1, 5),
]
# single tokens, gathered by adapter
GATHERED = [((300, 40, 16), 3), ((300, 40, 56), 5), ((300, 40, 128), 5)]
# tiles of 32 rows in slices of their columns, each of which takes h again
SLICES = [
    (([1800, 1000], [1, 0], 2, 64, 264, 4104, 1), 32, 5, 2),
    (([2000, 960], [1, 0], 2, 32, 72, 14336, 1), 32, 8, 4),
]
