"""The rules that choose the grouped products' kernels, built for the host: the sizes the GPU tests
run reach every variant, and the chunks of any offsets fit the workspace."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_1706_01307_amd as spc
from paper_1706_01307_amd import _lib
from tests import rows_variants as v

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
CODE = {"f32": spc.F32, "bf16": spc.BF16}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "plan.so")
    cmd = ["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror",
           "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_1706_01307_amd", "csrc"),
           os.path.join(ROOT, "tests", "rows_plan_driver.cpp"), "-o", so]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lib = ctypes.CDLL(so)
    i, i64, p = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p
    lib.plan_grouped.argtypes = [i, i, i, i64, i, i, i, i, p]
    lib.plan_weight.argtypes = [i, i64, i, i, i, i, p]

    class Plans:
        @staticmethod
        def grouped(dt, odt, backward, m, E, red, cols, whole):
            out = (i * 3)()
            lib.plan_grouped(CODE[dt], CODE[odt], backward, m, E, red, cols, whole, out)
            return tuple(out)

        @staticmethod
        def weight(dt, m, E, ci, co, whole):
            """tile, positions of a chunk, chunks, runs, workspace bytes"""
            out = (i64 * 5)()
            lib.plan_weight(CODE[dt], m, E, ci, co, whole, out)
            return tuple(out)
    return Plans


def _whole(dt, *widths):
    return all(w % (4 if dt == "f32" else 8) == 0 for w in widths)


def test_products_reach_every_kernel(plans):
    seen = set()
    for dt, backward, sizes, red, cols, want in v.PRODUCTS:
        m = sum(sizes) + v.TAIL
        # rows of the reduction, weights of it or of the columns
        whole = _whole(dt, red, red if backward else cols)
        for odt in CODE:
            if want[0] == v.SHORT and odt == "f32" and cols % 32:
                continue                             # (no whole lines: tiles)
            assert plans.grouped(dt, odt, backward, m, len(sizes), red, cols, whole) == want, \
                (dt, odt, backward, sizes, red, cols)
        seen.add((dt, backward, want))
    both = [(v.ANY, 64, 1), (v.ANY, 128, 1), (v.TILES, 64, 4), (v.TILES, 64, 3), (v.TILES, 128, 4)]
    bf16 = [(v.TILES, 256, 4)] + [(v.SHORT, 256, ring) for ring in (2, 4, 6, 8)]
    every = {(dt, back, p) for dt in CODE for back in (False, True)
             for p in both + (bf16 if dt == "bf16" else [])}
    assert seen == every | {(dt, False, (v.FEW, 0, 0)) for dt in CODE}


def test_reductions_in_registers_are_for_many_results_of_large_groups(plans):
    """256-row workgroups with their rows in registers lose to the tiles on few results, on small
    groups, on few columns and on fp32 results of cut lines."""
    for m, E, red, cols, odt, short in (
            (700000, 16, 256, 1024, "bf16", True), (700000, 16, 256, 1024, "f32", True),
            (700000, 16, 128, 384, "bf16", True), (131072, 256, 256, 2048, "bf16", True),
            (16384, 256, 256, 1024, "bf16", False), (65536, 256, 256, 256, "bf16", False),
            (65536, 16, 256, 1024, "bf16", False), (16384, 1, 64, 256, "bf16", False),
            (700000, 16, 64, 256, "bf16", False), (2097152, 16, 256, 144, "bf16", False),
            (1016800, 16, 40, 264, "f32", False), (20000, 256, 256, 16384, "bf16", False),
            (700000, 16, 264, 1024, "bf16", False)):
        for backward in (False, True):
            got = plans.grouped("bf16", odt, backward, m, E, red, cols, True)
            assert (got[0] == v.SHORT) == short, (m, E, red, cols, odt, got)


def test_weight_gradients_reach_every_kernel(plans):
    seen, runs = set(), set()
    for dt, sizes, ci, co, (tile, whole, run) in v.WEIGHTS:
        assert _whole(dt, ci, co) == whole
        got = plans.weight(dt, sum(sizes) + v.TAIL, len(sizes), ci, co, whole)
        assert (got[0], got[3]) == (tile, run), (dt, sizes, ci, co, got)
        assert (got[1] == 0) == (run == 0)
        seen.add((dt, tile, whole, run > 0))
        runs.add(run)
    every = {(dt, tile, whole, chunks) for dt in CODE for tile in (64, 128)
             for whole in (True, False) for chunks in (True, False)}
    assert seen == every | {("bf16", 256, True, chunks) for chunks in (True, False)}
    assert runs == {0, 1, 8}


def test_plan_is_the_library_s(plans):
    """The workspace the library asks for is the larger of the plan's with and without whole
    pieces."""
    n = ctypes.c_size_t()
    for dt, sizes, ci, co, _ in v.WEIGHTS:
        m, E = sum(sizes) + v.TAIL, len(sizes)
        assert _lib.load().spconv_grouped_backward_weight_workspace(
            CODE[dt], m, E, ci, co, ctypes.byref(n)) == 0
        assert n.value == max(plans.weight(dt, m, E, ci, co, w)[4] for w in (True, False))


def test_chunks_of_any_offsets_fit_the_workspace(plans):
    """Groups cut at the running maximum of their offsets never have more chunks than planned;
    each pair of offsets on its own can."""
    g = np.random.default_rng(1)
    more = 0
    for _ in range(400):
        dt = ("f32", "bf16")[int(g.integers(2))]
        m, E = int(10 ** g.uniform(1, 5.8)), int(10 ** g.uniform(0, 2.5))
        ci, co = (int(10 ** g.uniform(0.9, 3)) for _ in range(2))
        _, chunk, jobs, _, _ = plans.weight(dt, m, E, ci, co, bool(g.integers(2)))
        if not chunk:
            continue
        for off in (np.sort(g.integers(0, m + 1, E + 1)), g.integers(-m, 2 * m, E + 1),
                    np.arange(E + 1) % 2 * m):
            off = np.clip(off, 0, m)
            cut = np.diff(np.maximum.accumulate(off))
            assert -(-cut // chunk).sum() <= jobs
            more += -(-np.diff(off).clip(0) // chunk).sum() > jobs
    assert more > 20
