"""Layers (T, d, F, E, k) that the tests of the experts' gradient run, from one token of the narrowest layer on; among them every tile that the bf16
kernels have (test_training_cpu.py)."""
EXPERTS = [(1, 8, 8, 1, 1), (1, 40, 72, 4, 2), (5, 64, 136, 8, 3), (33, 128, 128, 2, 1), (7, 136, 136, 4, 2), (24, 256, 512, 16, 4), (40, 432, 1152, 8, 2),
           (100, 328, 264, 3, 2), (777, 160, 200, 8, 2), (1500, 264, 520, 4, 1), (64, 520, 1064, 64, 6), (300, 1440, 456, 4, 2), (2, 2048, 256, 8, 2),
           (3000, 264, 2056, 4, 2), (9000, 520, 520, 2, 2), (1500, 264, 1032, 16, 4)]
