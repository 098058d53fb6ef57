"""Sizes of the products of a linear layer in 8 bits that stand for each form of their kernels: the test of the plan says that they take it, those on a
GPU that what it computes is right."""
import paper_2510_09103_b200 as A

FORWARD, INPUT, WEIGHT = A.LINEAR8_FORWARD, A.LINEAR8_INPUT_GRAD, A.LINEAR8_WEIGHT_GRAD
BF16, F32 = A.TYPE_BF16, A.TYPE_F32

# product, type of its result, form, tokens, output features, input features
SIZES = [
    (FORWARD, BF16, "lines", 1, 512, 4096), (FORWARD, BF16, "lines", 2, 512, 4096), (FORWARD, F32, "lines", 2, 2056, 1544),
    (FORWARD, BF16, "lines", 1, 40008, 264), (FORWARD, F32, "lines", 2, 24, 12296),
    (FORWARD, BF16, "strips", 3, 4096, 4096), (FORWARD, BF16, "strips", 130, 1032, 2056),
    (FORWARD, BF16, "pairs", 3000, 2056, 512), (FORWARD, F32, "pairs", 3000, 2048, 520),
    (INPUT, BF16, "folded strips", 16, 4104, 1032), (INPUT, BF16, "strips", 17, 4104, 1032), (INPUT, F32, "folded strips", 130, 1032, 520),
    (INPUT, BF16, "pairs", 3000, 2048, 1024), (INPUT, BF16, "pairs", 2500, 520, 2056), (INPUT, BF16, "pairs, K cut", 598, 12904, 304),
    (INPUT, BF16, "pairs, long sums", 5000, 16456, 1024), (INPUT, F32, "pairs", 3000, 2048, 1024), (INPUT, F32, "pairs, K cut", 1000, 6152, 520),
    (WEIGHT, BF16, "folded strips", 2056, 16, 520), (WEIGHT, BF16, "strips", 333, 520, 392), (WEIGHT, F32, "folded strips", 333, 520, 392),
    (WEIGHT, BF16, "pairs", 2000, 2048, 2568), (WEIGHT, BF16, "pairs, K cut", 15083, 528, 80), (WEIGHT, BF16, "pairs, K cut", 9999, 1032, 392),
    (WEIGHT, BF16, "pairs, long sums", 17000, 4096, 2560), (WEIGHT, F32, "pairs", 600, 2048, 2568), (WEIGHT, F32, "pairs, K cut", 4999, 520, 392),
]


def sizes(*which):
    return [s for s in SIZES if s[0] in which]
