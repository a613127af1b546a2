"""Neighbourhoods whose attention takes the tile kernels in all passes, for the paths that only some of them have:
name -> (dims, periodic, offsets, q heads, kv heads, head_dim)."""
import iso_inputs as gen


def here(d):
    return [(0,) * d]


TILED = {
    # neighbours that are listed two and three times, as they are or by wrapping: a second and third row of one key
    "repeats": ((64, 64), None, [(0, 1), (0, 1), (0, 0), (0, 65), (64, 0), (-3, 2)], 2, 2, 96),
    "repeats_of_shared_heads": ((80, 90), None, [(0, 1), (0, 1), (0, 0), (0, 91), (80, 0), (-3, 2), (1, 1), (1, 0)], 4, 2, 64),
    "wraps_onto_itself": ((3, 256), None, gen.moore(2, 3) + here(2), 2, 1, 64),
    # few rows in common: the order in which rows were found
    "far_and_few": ((40, 132), None, [(17, -11), (-20, 3), (5, 16)], 2, 2, 64),
    "scattered": ((7, 6, 5, 80), None, gen.random_distinct(4, -3, 3, 12, 11), 2, 2, 64),
    "scattered_mesh": ((7, 6, 9, 40), [False, False, True, True], gen.random_distinct(4, -3, 3, 12, 12), 2, 2, 128),
    # neighbours that no rank of a mesh has, and some of the others only at its ends
    "far_mesh": ((12, 208), [False, False], [(11, 12), (-11, 0), (2000000000, 1), (-2000000000, -2), (0, 0)], 2, 2, 64),
    "half_mesh": ((9, 200), [True, False], gen.moore(2, 2), 2, 2, 40),
    "mesh_line": ((1000,), [False], [(c,) for c in range(40)], 2, 2, 128),
    # five to nine dimensions: positions of more than one word, and of three; sizes of 1 to 3; tiles that do not divide them
    "five_dimensions": ((5, 3, 4, 3, 20), None, gen.von_neumann(5, 1) + here(5), 2, 2, 64),
    "five_of_a_mesh": ((5, 3, 4, 3, 26), [True, False, True, True, False], gen.von_neumann(5, 1) + here(5), 2, 2, 128),
    "six_dimensions": ((3, 3, 2, 3, 2, 64), None, gen.von_neumann(6, 1), 2, 2, 80),
    "nine_dimensions": ((2, 1, 2, 2, 3, 2, 2, 2, 44), None, gen.von_neumann(9, 1) + here(9), 2, 2, 32),
}
