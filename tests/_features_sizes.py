"""Sizes of the lookup and its gradient, each with the route that it takes: a CPU test holds them against the plans of
csrc/features/scd_plan.h, the GPU tests run them."""

# (route, tokens, rows, dim): the sort (tiles and merge, or radix with 2, 4 or 8 entries a thread) and the digits of a
# key, which are the radix sort's passes.
SORTS = [
    ("tiles 1", 1025, 40, 5), ("tiles 1", 16_384, 2_046, 3), ("radix2 1", 16_385, 2_046, 3), ("tiles 2", 16_385, 2_048, 9),
    ("tiles 2", 32_768, 70_001, 4), ("radix2 2", 32_769, 70_001, 4), ("tiles 3", 32_001, 5_000_001, 2), ("radix2 3", 40_003, 5_000_001, 3),
    ("radix2 2", 200_000, 3_001, 7), ("radix4 1", 200_001, 999, 8), ("radix4 2", 250_007, 300_001, 5), ("radix4 3", 250_007, 4_200_001, 2),
    ("radix4 2", 800_000, 4_097, 3), ("radix8 1", 800_001, 1_500, 4), ("radix8 2", 900_011, 150_001, 16), ("radix8 3", 900_011, 4_200_001, 3),
]

# (threads and groups of lanes of a workgroup of the sums, column ranges, tokens, rows, dim, bytes of the wider element):
# rows of 64 to 256 lanes and of several ranges, and narrow ones.
SUMS = [
    ((512, 8, 1), 2_001, 700, 300, 2), ((512, 4, 1), 2_001, 700, 300, 4), ((512, 4, 1), 20_000, 4_001, 1_000, 2),
    ((512, 4, 1), 20_000, 900, 511, 4), ((512, 2, 1), 2_003, 333, 1_030, 2), ((512, 2, 2), 2_003, 333, 1_030, 4),
    ((512, 2, 2), 2_500, 61, 2_100, 2), ((512, 2, 3), 2_500, 61, 2_100, 4), ((256, 8, 1), 5_000, 900, 250, 2), ((256, 8, 1), 30_001, 300, 128, 4),
    ((256, 64, 1), 40_000, 900, 16, 4), ((256, 128, 1), 40_000, 900, 16, 2), ((256, 32, 1), 3_000, 50, 7, 2),
]

# (tokens, rows, dim, bytes of the wider element): one token's entries make up so many workgroups of the sums that a whole
# workgroup adds their pieces.
LONG_RUNS = [(600_000, 5, 16, 4), (100_000, 9, 40, 4), (20_000, 7, 300, 4), (20_000, 7, 300, 2), (9_000, 3, 1_030, 4), (700_001, 4, 3, 4)]

# (rows in flight, tokens, rows, dim, bytes of the wider element)
LOOKUPS = [
    (1, 70_001, 1_000, 16, 4), (4, 600_003, 1_000, 16, 4), (4, 33_001, 500, 300, 4), (4, 33_001, 500, 303, 2), (4, 5_001, 99, 1_030, 4),
    (4, 9_001, 99, 1_030, 2), (4, 2_100_001, 77, 3, 4), (4, 1_050_001, 77, 7, 2),
]
