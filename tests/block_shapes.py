"""Sizes of products (P, Q, R) and gated blocks (M, F, K) that take every form of the tile kernel, by whether the fp8 pipeline runs: whole tiles one
a workgroup, several, tiles in slices, whole ones and slices, with rows, columns and contractions that end inside a tile (test_block_plan.py says
what which size takes)."""

# (form, several items a workgroup, slices): forms in the order of srq_block_plan.hpp
PRODUCTS = {
    False: {(0, False, False): (2691, 4365, 144), (0, True, False): (3590, 6664, 144), (0, False, True): (3549, 1185, 4112),
            (0, True, True): (4510, 3716, 1168),
            (1, False, False): (454, 4137, 144), (1, True, False): (4366, 1807, 144), (1, False, True): (65, 2626, 2064),
            (1, True, True): (3284, 2436, 400),
            (2, False, False): (3223, 1153, 144), (2, True, False): (3333, 2324, 144), (2, False, True): (3486, 266, 4112),
            (2, True, True): (3626, 1092, 1040),
            (3, False, False): (22, 32, 272), (3, True, False): (2954, 1285, 144), (3, False, True): (25, 17, 1168),
            (3, True, True): (2728, 705, 1168)},
    True: {(0, False, False): (3592, 2242, 144), (0, True, False): (6672, 3586, 144), (0, False, True): (3000, 1000, 8200),
           (0, True, True): (4501, 3720, 1040),
           (1, False, False): (3431, 1158, 144), (1, True, False): (4368, 3611, 144), (1, False, True): (69, 2997, 4112),
           (1, True, True): (4423, 1811, 1040),
           (2, False, False): (525, 3610, 144), (2, True, False): (3349, 2308, 144), (2, False, True): (4240, 195, 4112),
           (2, True, True): (3613, 1096, 1040),
           (3, False, False): (42, 28, 144), (3, True, False): (4181, 913, 144), (3, False, True): (28, 67, 2064),
           (3, True, True): (457, 4185, 2064)}}
# (the two small forms of the gated block run the exact pipeline whatever the flag)
GATED = {
    False: {(0, False, False): (714, 5504, 144), (0, True, False): (2188, 5504, 144), (0, False, True): (132, 4096, 4112),
            (0, True, True): (2950, 2816, 400),
            (1, False, False): (322, 5632, 144), (1, True, False): (1288, 5504, 144), (1, False, True): (67, 1792, 4112),
            (1, True, True): (2369, 3456, 400),
            (2, False, False): (201, 4736, 144), (2, True, False): (641, 5504, 144), (2, False, True): (41, 768, 1040),
            (2, True, True): (326, 5504, 2064),
            (3, False, False): (25, 128, 272), (3, False, True): (25, 128, 1168)},
    True: {(0, False, False): (660, 5504, 144), (0, True, False): (1423, 5504, 144), (0, False, True): (140, 2560, 2064),
           (0, True, True): (1668, 4736, 1040),
           (1, False, False): (163, 5504, 144), (1, True, False): (1550, 4736, 144), (1, False, True): (37, 896, 1040),
           (1, True, True): (651, 5632, 2064),
           (2, False, True): (129, 640, 4112), (3, False, True): (24, 128, 1040)}}
