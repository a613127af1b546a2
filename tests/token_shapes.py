"""Sizes that the GPU tests of the operators on each token use: together they take every kernel (checked on the CPU by
test_token_refusals.py)."""
# Layer norm: tokens, heads, channels.  Lanes of a wavefront, whole wavefronts, several, whole and broken units of 16 bytes.
NORMS = [(1, 1, 1), (1, 1, 8), (3, 1, 3), (5, 1, 64), (64, 1, 64), (10, 1, 61), (33, 5, 40), (7, 3, 128), (9, 3, 99), (130, 1, 129), (257, 2, 80),
         (12, 2, 200), (6, 1, 250), (19, 1, 483), (40, 1, 512), (11, 1, 777), (300, 1, 1000), (70, 1, 1024), (9, 1, 1025), (6, 1, 2047), (5, 1, 4096),
         (3, 1, 5001), (2, 1, 16384), (2, 1, 16381)]

# Gated projections: tokens, channels, hidden units.
FEW = [(1, 1, 1), (1, 64, 16), (1, 136, 40), (5, 33, 17), (16, 256, 48), (17, 100, 31), (17, 101, 33), (32, 512, 24), (37, 520, 90), (48, 135, 80),
       (64, 1040, 33), (63, 72, 130)]
TILED = [(65, 8, 8), (65, 1, 3), (70, 64, 64), (129, 130, 65), (100, 200, 300), (200, 72, 132), (333, 65, 127), (257, 264, 72), (65, 700, 513)]
# enough tiles for the larger ones, with rows, elements and steps left over
LARGE = [(1500, 136, 1100), (2100, 72, 1928), (3333, 24, 1672), (5000, 200, 1500), (5000, 201, 1500), (2600, 97, 700), (12000, 1048, 264),
         (200, 2072, 3100), (4096, 2040, 100), (150, 2040, 2045)]
