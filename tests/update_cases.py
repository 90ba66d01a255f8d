"""Matrices whose products between them are cut into every tile that there is a kernel for: what the GPU tests run, and the launch rules' test asks the rules about."""
# rows, cols; sides that no tile divides, wide and tall by turns
EVERY_TILE = [(47, 700), (900, 1001), (1001, 999), (1061, 1063), (1483, 1481), (2021, 2023), (2083, 2081), (2443, 2449), (2503, 2501), (2861, 2863), (3523, 3521), (4029, 4031), (4183, 4181)]
# rows, cols, how many in one call: more of them are cut otherwise than one alone, by tiles that no waves share
CUT_OTHERWISE = [(1061, 1063, 3), (1063, 1061, 6), (1191, 1061, 6), (1061, 1319, 3), (1959, 1061, 3), (1125, 1831, 4), (1381, 2215, 2), (2215, 1445, 5), (186, 5493, 12)]
