"""Products of 8-bit floating point codes that take each of the kernel forms, with ragged sizes and more than eight blocks of the reduction
(test infrastructure)."""
import numpy as np

NAMES = ("direct 16", "direct 32", "direct 64", "tile 64", "tile 64x128", "tile 128 deep", "tile 128", "tile 256")   # as Fp8Form has them

# M, N, K, then (form, slices) for a bf16 and a fp32 result
FORMS = [
    (13, 300, 1500, ("direct 16", 1), ("direct 16", 1)),
    (29, 4090, 4000, ("direct 32", 1), ("direct 32", 1)),
    (61, 4090, 4000, ("direct 64", 1), ("direct 64", 1)),
    (250, 500, 1500, ("tile 64", 1), ("tile 64", 1)),
    (200, 1000, 4100, ("tile 64", 1), ("tile 64", 4)),
    (300, 520, 4097, ("tile 64", 4), ("tile 64", 4)),
    (70, 300, 8192, ("tile 64", 8), ("tile 64", 8)),
    (66, 200, 16500, ("tile 64", 16), ("tile 64", 16)),
    (500, 4090, 4000, ("tile 64x128", 1), ("tile 64x128", 1)),
    (700, 4000, 1300, ("tile 128 deep", 1), ("tile 64x128", 1)),
    (2001, 2098, 1500, ("tile 128", 1), ("tile 128", 1)),
    (4093, 8189, 2050, ("tile 256", 1), ("tile 256", 1)),
]


def whole(R, K, seed):
    """Codes [R, K filled up to 128] and scale bytes of small whole numbers times 1, 2 or 4, and what they stand for: sums of up to 2^24 / 144
    products are exact in fp32 in any order."""
    g = np.random.default_rng(seed)
    nb = -(-K // 128)
    q = np.zeros((R, nb * 128), np.float32)
    q[:, :K] = g.integers(-3, 4, (R, K))
    s = np.full((R, -(-nb // 4) * 4), 127, np.uint8)
    s[:, :nb] += g.integers(0, 3, (R, nb)).astype(np.uint8)
    return q, s, q * np.repeat(np.exp2(s[:, :nb].astype(np.float32) - 127), 128, axis=1)
