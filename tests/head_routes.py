"""Sizes of the head's calls that between them take every form of launch (tests/test_head_plan.py checks which): tokens, vocabulary, width."""
ROUTES = [
    (3, 70001, 40),         # hardly any tokens, many tiles of 128
    (171, 36393, 72),       # logits in 256-wide tiles
    (5, 40585, 32),
    (700, 24100, 72),       # several bands of columns, the last round in quarters
    (165, 81174, 32),       # ... in fp32
    (1, 65989, 200),        # gradient of W in 256-wide tiles, the last round in quarters (fp32)
    (1115, 409, 40),        # gradient of W split over tokens, a compute unit per tile
    (354, 17767, 32),       # ... two tiles per unit (fp32)
    (1429, 5594, 152),
    (1551, 9067, 136),      # ... in 256-wide tiles (fp32)
    (2868, 3887, 144),
    (6970, 1882, 136),      # gradient of H split over the vocabulary in 256-wide tiles (fp32)
    (2, 10177, 1160),       # ... in tiles of 128, two per unit (fp32)
    (64, 9001, 256),        # ... a unit each
    (6551, 290, 1336),      # gradient of H in 256-wide tiles
]
