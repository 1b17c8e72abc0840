"""Layers of experts in 4 bits that take the tiled products: which tile each of the two products has is checked on the host, the results on the GPU."""
import numpy as np

PATTERNS = 257  # tokens of a case are copies of so many: no tile's rows are a multiple of it, so that each comes to lie everywhere in a tile

# tokens, d_model, d_ff, experts, picks, skew of the loads, rows of a tile of gate/up and of down (32: streamed).  Units of K (256 columns, of d_model for gate/up and of
# d_ff for down) are 1, fewer than a tile has stages, as many, one more, and many; widths are no whole tiles.
TILED = [
    (2003, 264, 256, 5, 4, 0, 64, 32), (2003, 520, 256, 5, 4, 0, 64, 128), (3001, 776, 600, 1, 1, 0, 64, 32), (3001, 2056, 520, 2, 1, 1, 64, 128),
    (3001, 1032, 72, 2, 1, 1, 32, 64), (5000, 520, 520, 2, 1, 1, 128, 64), (5000, 520, 776, 2, 1, 1, 256, 64), (5000, 520, 2056, 2, 1, 1, 256, 64),
    (16003, 136, 72, 3, 2, 1, 128, 128), (9001, 264, 328, 2, 1, 1, 128, 32), (9001, 776, 328, 2, 1, 1, 128, 256), (20011, 136, 776, 2, 1, 1, 256, 128),
    (12007, 264, 72, 5, 4, 0, 256, 256), (9001, 1032, 520, 2, 1, 1, 256, 256), (9001, 2056, 2056, 2, 1, 1, 256, 128), (5000, 2056, 2056, 2, 1, 1, 128, 256),
]


def picks(E, k, skew):
    """idx [PATTERNS, k] int32, gate [PATTERNS, k] fp32"""
    rng = np.random.default_rng(E * 100 + k)
    p = -skew * np.log(np.arange(1, E + 1)) + rng.gumbel(size=(PATTERNS, E))
    gate = rng.random((PATTERNS, k)).astype(np.float32)
    return np.argsort(-p, axis=1)[:, :k].astype(np.int32), gate / gate.sum(1, keepdims=True)
