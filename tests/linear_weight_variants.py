"""Sizes of dense weight gradients that reach every tile of each type, with rows of whole pieces and
with cut ones, in one chunk of the rows and in several: (type, rows, C_in, C_out, tile, whole, several
chunks).  test_linear_weight_cpu.py holds the rule to it, test_linear_weight_gpu.py runs the kernels
(whole ones on unaligned views too)."""

TILES = [
    ("bf16", 64, 72, 96, 64, 1, 0), ("bf16", 333, 72, 96, 64, 1, 1),
    ("bf16", 100, 131, 72, 64, 0, 0), ("bf16", 500, 72, 99, 64, 0, 1),
    ("bf16", 64, 2056, 2000, 128, 1, 0), ("bf16", 100000, 72, 72, 128, 1, 1),
    ("bf16", 64, 2001, 2056, 128, 0, 0), ("bf16", 100000, 131, 72, 128, 0, 1),
    ("bf16", 64, 4104, 2000, 256, 1, 0), ("bf16", 5000, 4104, 72, 256, 1, 1),
    ("bf16", 60000, 200, 200, 256, 1, 1), ("bf16", 64, 3000, 2570, 256, 0, 0),
    ("bf16", 7000, 4001, 72, 256, 0, 1), ("bf16", 100000, 131, 300, 256, 0, 1),
    ("bf16", 485480, 174, 96, 256, 0, 1), ("bf16", 3001, 4104, 203, 256, 0, 1),
    ("f32", 64, 72, 96, 64, 1, 0), ("f32", 333, 72, 72, 64, 1, 1),
    ("f32", 64, 131, 72, 64, 0, 0), ("f32", 333, 72, 73, 64, 0, 1),
    ("f32", 64, 2056, 2000, 128, 1, 0), ("f32", 2000, 4104, 72, 128, 1, 1),
    ("f32", 64, 1545, 2570, 128, 0, 0), ("f32", 2000, 2055, 200, 128, 0, 1),
]
