"""Sizes that reach every kernel variant of the grouped products (csrc/rows_plan.h), with what the
rules choose for them: test_rows_plan_cpu.py holds the rules to it, test_rows_variants_gpu.py runs
the kernels.  Groups of very different sizes, an empty one, positions behind the last (TAIL);
reductions of more stages than the rings hold and cut ones; cut tiles of rows and columns."""

FEW, ANY, SHORT, TILES = range(4)
TAIL = 3

# (dtypes, sizes of the groups, reduction, columns, (kernel, tile, ring)); each is run forwards
# and, but for FEW, as an input gradient with the same reduction and columns
_PRODUCTS = [
    ("f32 bf16", [1, 0, 2], 2300, 72, (FEW, 0, 0)),
    ("f32 bf16", [420, 0, 177], 133, 70, (ANY, 64, 1)),
    ("bf16", [5000, 0, 3301], 133, 1931, (ANY, 128, 1)),
    ("f32", [12000, 0, 5001], 133, 1931, (ANY, 128, 1)),
    ("f32 bf16", [300, 0, 197], 184, 72, (TILES, 64, 4)),
    ("f32 bf16", [1700, 0, 801], 184, 1544, (TILES, 64, 3)),
    ("bf16", [5000, 0, 3301], 296, 1928, (TILES, 128, 4)),
    ("f32", [12000, 0, 5001], 152, 1928, (TILES, 128, 4)),
    ("bf16", [30000, 0, 14100], 296, 720, (TILES, 256, 4)),
    # (reductions kept in registers: at least 2^28 results)
    ("bf16", [299000, 0, 195001], 40, 544, (SHORT, 256, 2)),
    ("bf16", [299000, 0, 195001], 104, 544, (SHORT, 256, 4)),
    ("bf16", [299000, 0, 195001], 168, 544, (SHORT, 256, 6)),
    ("bf16", [299000, 0, 195001], 232, 544, (SHORT, 256, 8)),
    ("bf16", [299000, 0, 218001], 256, 520, (SHORT, 256, 8))]
PRODUCTS = [(dt, backward, sizes, red, cols, plan)
            for dtypes, sizes, red, cols, plan in _PRODUCTS for dt in dtypes.split()
            for backward in ((False,) if plan[0] == FEW else (False, True))]

_MANY = [11, 0, 7, 15] * 10                          # groups of one chunk each
# (dtypes, sizes, C_in, C_out, (tile, whole pieces, runs of the chunks' sums: 0 for one chunk))
_WEIGHTS = [
    ("f32 bf16", [3000, 0, 901, 70], 72, 96, (64, True, 8)),
    ("f32 bf16", [3000, 0, 901, 70], 71, 95, (64, False, 8)),
    ("f32 bf16", _MANY, 24, 40, (64, True, 0)),
    ("f32 bf16", _MANY, 23, 41, (64, False, 0)),
    ("bf16", [20000, 0, 7000, 501], 120, 1032, (128, True, 8)),
    ("f32", [12000, 0, 7000, 501], 520, 512, (128, True, 1)),
    ("bf16", [20000, 0, 7000, 501], 517, 510, (128, False, 1)),
    ("f32", [12000, 0, 7000, 501], 517, 510, (128, False, 1)),
    ("f32", [9000, 0, 20000, 300] * 2, 96, 200, (128, True, 8)),
    ("f32", [9000, 0, 20000, 300] * 2, 97, 201, (128, False, 8)),
    ("f32 bf16", _MANY, 120, 2040, (128, True, 0)),
    ("f32 bf16", _MANY, 119, 2041, (128, False, 0)),
    ("bf16", [26000, 0, 13000, 1001], 1024, 520, (256, True, 1)),
    ("bf16", _MANY, 408, 408, (256, True, 0))]
WEIGHTS = [(dt, sizes, ci, co, plan) for dtypes, sizes, ci, co, plan in _WEIGHTS
           for dt in dtypes.split()]
