"""The dense operators on feature rows without a GPU: bad arguments are refused on the host, the
64-bit statements' gradients are those of differences, and the rules that choose kernels and chunks
keep to their workspace."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_1706_01307_amd import _lib
from tests import rows_dense_ref as ref
from tests.test_rows_cpu import E, ODD, P, ROOT, _refused

HALF = ctypes.c_void_p(4098)         # aligned to 2 bytes


def test_rms_norm_refusals():
    good = [0, P, P, P, 1e-6, P, 0, P, None, P, 4, 8, None]
    _refused("spconv_rms_norm_forward", good, [
        {0: 2}, {0: -1}, {1: None}, {1: HALF}, {2: HALF}, {2: None}, {3: HALF}, {4: -1.0},
        {4: float("nan")}, {4: float("inf")}, {5: HALF}, {6: 1}, {6: 3}, {7: None}, {7: HALF},
        {8: P}, {6: 2, 8: None}, {6: 2, 8: HALF}, {9: HALF}, {10: -1}, {10: 2 ** 31}, {11: 0},
        {11: -5}])
    good = [1, P, 1, P, None, P, P, P, P, P, 4, 8, P, 32, None]
    _refused("spconv_rms_norm_backward", good, [
        {0: 2}, {1: None}, {1: ODD}, {2: 0}, {3: None}, {4: P}, {2: 2, 4: None}, {2: 2, 4: HALF},
        {5: None}, {6: HALF}, {7: ODD}, {8: None}, {9: HALF}, {10: -1}, {11: 0}, {12: None},
        {12: ctypes.c_void_p(4104)}, {13: 31}, {11: 65535 * 256 + 1, 13: 2 ** 62}])
    n, lib = ctypes.c_size_t(), _lib.load()
    assert lib.spconv_rms_norm_backward_workspace(4, 0, ctypes.byref(n)) == E
    assert lib.spconv_rms_norm_backward_workspace(4, 8, None) == E
    assert lib.spconv_rms_norm_backward_workspace(4, 8, ctypes.byref(n)) == 0 and n.value == 32


def test_eight_bit_rows_refusals():
    _refused("spconv_pack_rows", [1, P, ODD, P, 4, 8, None], [
        {0: 2}, {1: None}, {1: ODD}, {2: None}, {3: None}, {3: HALF}, {4: -1}, {5: 0}])
    _refused("spconv_unpack_rows", [ODD, P, 1, 0, P, 4, 8, None], [
        {0: None}, {1: None}, {1: HALF}, {2: -1}, {2: 4}, {3: 2}, {4: None}, {4: HALF}, {5: -1},
        {6: 0}])
    _refused("spconv_activation_backward", [1, P, 1, P, None, 2, P, 4, 8, None], [
        {0: 2}, {1: None}, {2: 0}, {2: 3}, {3: None}, {3: ODD}, {4: P}, {2: 2, 4: None}, {5: 4},
        {6: None}, {6: ODD}, {7: -1}, {8: 0}])


def test_linear_refusals():
    good = [1, P, None, P, P, 2, P, 1, P, P, 9, 8, 8, None]
    _refused("spconv_linear_forward", good, [
        {0: 3}, {0: -1}, {1: None}, {1: ODD}, {2: P}, {0: 2}, {0: 2, 2: HALF}, {3: None}, {3: ODD},
        {4: HALF}, {5: -1}, {5: 4}, {6: ODD}, {7: 2}, {8: None}, {8: ODD}, {9: ODD}, {10: -1},
        {10: 2 ** 31}, {11: 0}, {12: 0}, {11: 2 ** 23 + 1}, {12: 2 ** 23 + 1},
        {11: 2 ** 16, 12: 2 ** 15}])
    good = [1, P, P, 2, 1, P, None, 1, P, 9, 8, 8, None]
    _refused("spconv_linear_backward_data", good, [
        {0: 2}, {1: None}, {1: ODD}, {2: None}, {3: 4}, {4: 0}, {5: None}, {5: ODD}, {6: P},
        {4: 2, 6: None}, {3: 0}, {7: 2}, {8: None}, {8: ODD}, {9: -1}, {10: 0}, {11: 0},
        {10: 2 ** 16, 11: 2 ** 15}])
    good = [1, P, None, P, P, P, 10 ** 6, 64, 64, P, 1 << 40, None]
    _refused("spconv_linear_backward_weight", good, [
        {0: 3}, {1: None}, {1: ODD}, {2: P}, {0: 2}, {3: None}, {3: ODD}, {4: None}, {4: HALF},
        {5: HALF}, {6: -1}, {7: 0}, {8: 0}, {9: None}, {9: ctypes.c_void_p(4104)}, {10: 16},
        {7: 2 ** 16, 8: 2 ** 15}])
    n, lib = ctypes.c_size_t(), _lib.load()
    assert lib.spconv_linear_backward_weight_workspace(3, 9, 8, 8, ctypes.byref(n)) == E
    assert lib.spconv_linear_backward_weight_workspace(1, 9, 0, 8, ctypes.byref(n)) == E
    assert lib.spconv_linear_backward_weight_workspace(1, 9, 8, 8, None) == E
    assert lib.spconv_linear_backward_weight_workspace(2, 9, 8, 8, ctypes.byref(n)) == 0


def test_route_scores_refusals():
    good = [0, P, P, 9, 8, 2, 0, 4, 2, 1, 1.0, P, P, P, P, P, P, 1 << 20, None]
    _refused("spconv_route_scores_forward", good, [
        {0: 2}, {1: None}, {1: HALF}, {2: HALF}, {3: -1}, {4: 0}, {4: 1025, 7: 1, 8: 1}, {5: 0},
        {5: 5}, {4: 32, 5: 17, 7: 1, 8: 1}, {6: 2}, {6: -1}, {7: 0}, {7: 3}, {7: 65, 4: 130},
        {8: 0}, {8: 5}, {9: 2}, {10: 0.0}, {10: -1.0}, {10: float("nan")}, {10: float("inf")},
        {11: None}, {12: None}, {13: None}, {14: None}, {15: None}, {3: 100000, 16: None},
        {3: 100000, 17: 16}, {3: 2 ** 30}])
    _refused("spconv_route_scores_backward", [0, P, P, P, P, 9, 8, 2, 0, 1, 1.0, P, None], [
        {0: 2}, {1: None}, {2: None}, {3: None}, {4: None}, {5: -1}, {6: 0}, {7: 0}, {7: 9}, {8: 2},
        {9: -1}, {10: 0.0}, {11: None}, {8: 1, 9: 0, 2: None}])


def _difference(f, x, d, h=1e-6):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def test_gradients_of_the_statements_are_those_of_differences():
    torch.manual_seed(3)
    r = lambda *s: torch.randn(*s, dtype=torch.float64)
    # norm: dx, dgamma along a direction
    h, g, dy, v, u, eps = r(5, 9), r(9), r(5, 9), r(5, 9), r(9), 1e-3
    (dx, dg), _ = ref.rms_grad(dy, h, ref.rms(h, g, eps)[1], g, None)
    got = (dy * _difference(lambda a: ref.rms(a, g, eps)[0], h, v)).sum()
    assert torch.isclose(got, (dx * v).sum(), rtol=1e-6)
    got = (dy * _difference(lambda a: ref.rms(h, a, eps)[0], g, u)).sum()
    assert torch.isclose(got, (dg * u).sum(), rtol=1e-6)
    # activations
    z = r(400) * 3
    for kind in (None, "relu", "gelu", "silu"):
        got = _difference(lambda a: ref.act(a, kind), z, torch.ones_like(z))
        assert torch.allclose(got, ref.slope(z, kind), atol=1e-7)
    # weights of a fixed choice
    x, dw, v = r(6, 8), r(6, 3), r(6, 8)
    e = torch.stack([torch.randperm(8)[:3] for _ in range(6)])
    e[2, 1:] = -1
    e[3] = -1
    for kind in ("sigmoid", "softmax"):
        for normalize in (True, False):
            f = lambda a: ref.weights(a, e, kind, normalize, 2.5)
            d, _ = ref.weights_grad(x, e, kind, normalize, 2.5, dw)
            got = (dw * _difference(f, x, v)).sum(1)
            assert torch.allclose(got, (d * v).sum(1), rtol=1e-6, atol=1e-8), (kind, normalize)


def test_packed_rows_of_the_statement():
    x = torch.tensor([[448.0, -224.0, 1.0, 0.0], [0.0] * 4, [1e-38, 0.0, 0.0, 0.0],
                      [float("inf"), 1.0, 0.0, 0.0], [float("nan")] * 4])
    q, s = ref.packed(x)
    assert s[0] == 1 and q[0].tolist() == [448.0, -224.0, 1.0, 0.0]
    assert q[1:3].float().abs().max() == 0 and torch.isfinite(s[:3]).all()
    assert torch.isnan(s[3:]).all() and q[3:].float().abs().max() == 0


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    so = str(tmp_path_factory.mktemp("plan") / "plan.so")
    cmd = ["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror",
           "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_1706_01307_amd", "csrc"),
           os.path.join(ROOT, "tests", "linear_plan_driver.cpp"), "-o", so]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lib = ctypes.CDLL(so)
    i, i64, p = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p
    lib.plan_linear.argtypes = [i, i, i64, i, i, i, p]
    lib.plan_linear_short.argtypes = [i64, i, i, i]
    lib.plan_linear_weight.argtypes = [i, i64, i, i, p]
    return lib


def test_products_reach_every_kernel(plans):
    """The sizes that the GPU tests run (PRODUCTS) reach every kernel and tile of each type."""
    from tests.linear_variants import PRODUCTS
    seen, out = set(), (ctypes.c_int * 2)()
    for dt, backward, n, red, cols, want in PRODUCTS:
        vec = 4 if dt == "f32" else 8
        whole = red % (16 if dt == "e4m3" else vec) == 0 and (red if backward else cols) % vec == 0
        plans.plan_linear(0 if dt == "f32" else 1, backward, n, red, cols, whole, out)
        got = (("few", "any", "tiles", "split")[out[0]], out[1])
        assert got == want, (dt, backward, n, red, cols)
        seen.add((dt, backward) + got)
    tiles = {"f32": (64, 128), "bf16": (64, 128, 256), "e4m3": (64, 128, 256)}
    for dt in tiles:
        for backward in (0, 1) if dt != "e4m3" else (0,):
            for t in (64, 128):
                assert (dt, backward, "any", t) in seen
            for t in tiles[dt]:
                assert (dt, backward, "tiles", t) in seen
            assert (dt, backward, "split", 32) in seen
    assert ("f32", 0, "few", 0) in seen and ("f32", 1, "few", 0) in seen


def test_products_that_keep_their_weights(plans):
    """The sizes of SHORT reach every number of stages both ways; small, wide and long ones stay out."""
    from tests.linear_variants import SHORT
    for backward, n, red, cols, stages, residual in SHORT:
        assert plans.plan_linear_short(n, red, cols, 0) == stages, (n, red, cols)
        assert plans.plan_linear_short(n, red, cols, 1) == (stages if residual else 0), (n, red, cols)
        assert (stages - 2) * 32 < red <= stages * 32
    assert {(s[0], s[4]) for s in SHORT} == {(b, k) for b in (0, 1) for k in (2, 4, 6, 8)}
    assert {s[4] for s in SHORT if not s[0] and s[5]} == {2, 4, 6, 8}
    for n, red, cols in ((16320, 64, 256), (70000, 257, 256), (70000, 64, 128), (1, 8, 256), (0, 8, 256)):
        assert plans.plan_linear_short(n, red, cols, 0) == 0
    assert plans.plan_linear_short(2 ** 31 - 1, 256, 2 ** 23, 1) == 8


def test_weight_gradient_chunks_cover_the_rows(plans):
    from tests.linear_variants import WEIGHTS
    out, seen = (ctypes.c_int64 * 5)(), set()
    sizes = [(d, n, ci, co) for d, n, ci, co, _ in WEIGHTS]
    sizes += [(d, n, ci, co) for d in ("f32", "bf16", "e4m3") for n in (0, 1, 63, 64, 65, 1000, 2 ** 31 - 1)
              for ci, co in ((1, 1), (3, 700), (96, 200), (2048, 2048), (2 ** 23, 1), (1, 2 ** 23))]
    for d, n, ci, co in sizes:
        code = {"f32": 0, "bf16": 1, "e4m3": 2}[d]
        plans.plan_linear_weight(code, n, ci, co, out)
        tile, chunk, jobs, tiles, size = out
        bn = 128 if tile == 256 else tile
        assert chunk >= 1 and jobs == max(1, -(-n // chunk))
        assert tiles == -(-ci // tile) * -(-co // bn)
        assert size == (jobs * (ci * co + co) * 4 if jobs > 1 else 0)
        seen.add((d, tile, jobs > 1))
    for d in ("f32", "bf16", "e4m3"):
        for t in (64, 128) if d == "f32" else (64, 128, 256):
            assert any(s[:2] == (d, t) for s in seen), (d, t)
