"""The rule that cuts dense weight gradients, at the sizes that their GPU tests run."""
import ctypes

from tests.linear_weight_variants import TILES
from tests.test_rows_dense_cpu import plans  # noqa: F401


def test_weight_gradients_reach_every_tile(plans):  # noqa: F811
    out, seen = (ctypes.c_int64 * 5)(), set()
    for dt, n, ci, co, tile, whole, several in TILES:
        plans.plan_linear_weight({"f32": 0, "bf16": 1, "e4m3": 2}[dt], n, ci, co, out)
        assert (out[0], out[2] > 1) == (tile, bool(several)), (dt, n, ci, co, list(out))
        vec = 4 if dt == "f32" else 8
        assert (ci % vec == 0 and co % vec == 0) == bool(whole), (dt, n, ci, co)
        seen.add((dt, tile, whole, several))
    assert seen == {(dt, t, w, s) for dt in {v[0] for v in TILES} for w in (0, 1) for s in (0, 1)
                    for t in ((64, 128) if dt == "f32" else (64, 128, 256))}
