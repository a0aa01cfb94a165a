"""Shapes that take every tile size of the operators' products, with k in one part and in
several; test_product_choice_cpu.py holds them to that."""

# (kernel, whether k is split, tokens, outs, dim, dy's type, dw's, padding and first element of rows, accumulate)
GRADIENTS = [
    ("LARGE", False, 71, 1031, 10017, "f16", "f32", 3, 1, False),
    ("LARGE", False, 300, 9216, 3001, "bf16", "bf16", 8, 0, True),
    ("LARGE", True, 4389, 541, 6671, "f16", "f32", 0, 0, False),
    ("LARGE", True, 6392, 5467, 391, "bf16", "f16", 5, 3, True),
    ("BROAD", False, 64, 1001, 9216, "f16", "f32", 0, 0, False),
    ("BROAD", False, 300, 3001, 4001, "bf16", "f32", 1, 1, True),
    ("BROAD", False, 61, 3987, 2083, "f16", "f16", 3, 1, True),
    ("BROAD", False, 66, 11517, 645, "bf16", "bf16", 0, 0, False),
    ("BROAD", True, 3757, 11219, 137, "f16", "f32", 3, 1, True),
    ("MIDDLE", False, 130, 2100, 1500, "f16", "f32", 0, 0, True),
    ("MIDDLE", False, 72, 8391, 197, "bf16", "f16", 5, 1, False),
    ("MIDDLE", False, 1000, 1500, 2048, "f16", "bf16", 8, 0, True),
    ("MIDDLE", True, 4949, 2093, 207, "f16", "f32", 1, 1, False),
    ("MIDDLE", True, 4807, 801, 629, "bf16", "bf16", 3, 1, True),
    ("TINY", False, 61, 3399, 267, "bf16", "f32", 3, 1, True),
    ("TINY", True, 1785, 145, 127, "f16", "f16", 3, 1, True),
    ("FEW", False, 72, 123, 137, "bf16", "f32", 3, 1, True),
]

# (kernel, whether k is split, tokens, rows, dim, x's type, out's, padding and first element of rows, accumulate), of
# packed operands; the same of inputs packed on the way
PRODUCTS = [
    ("WIDE4", False, 1025, 7583, 127, "f32", "f32", 3, 1, False),
    ("WIDE4", False, 2580, 3233, 125, "f16", "f16", 5, 1, True),
    ("WIDE4", True, 2547, 1575, 16039, "bf16", "f32", 1, 1, False),
    ("WIDE4", True, 1153, 3227, 15739, "f16", "bf16", 0, 0, True),
    ("HALF4", False, 2100, 2500, 300, "f16", "f32", 3, 1, True),
    ("HALF4", False, 300, 9216, 1001, "bf16", "bf16", 0, 0, False),
    ("HALF4", False, 199, 8315, 123, "f32", "f16", 5, 3, True),
    ("HALF4", True, 941, 517, 11097, "f16", "f32", 1, 1, False),
    ("HALF4", True, 2058, 209, 10065, "bf16", "f16", 3, 1, True),
    ("SMALL4", False, 71, 123, 137, "f16", "f32", 3, 1, True),
    ("SMALL4", True, 72, 121, 4261, "bf16", "bf16", 3, 1, True),
]
LINEARS = PRODUCTS[:-2] + [
    ("SMALL4", False, 500, 500, 5000, "f16", "f32", 3, 1, True),
    ("SMALL4", True, 72, 121, 4261, "bf16", "bf16", 3, 1, True),
    ("SMALL", False, 71, 123, 137, "f16", "f32", 3, 1, True),
    ("FEW", False, 3, 700, 9216, "f16", "f32", 3, 1, True),
]
