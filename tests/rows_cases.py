"""Calls (T, d, E, k) of the kernels between tokens and experts' rows that take forms which ordinary sizes do not: every number of waves a token by every number
of pairs held, dot products in LDS joined across waves, and few experts counted by ballots in many chunks (test_training_sizes_cpu.py)."""
ROWS = [(37, 1000, 8, 1), (41, 520, 8, 2), (29, 1000, 64, 40), (37, 1032, 8, 1), (37, 1440, 8, 4), (35, 2048, 8, 3), (37, 2056, 16, 7), (33, 4104, 8, 8), (29, 2056, 64, 12),
        (5, 1032, 64, 64), (777, 40, 3, 2), (1365, 24, 4, 3), (5000, 8, 1, 1), (4096, 8, 2, 2), (2048, 16, 4, 4), (8191, 8, 3, 1), (301, 8, 4, 2)]
