"""Operators on feature rows without a GPU: the library exports what spconv_rows.h
declares, refuses bad arguments on the host, and the 64-bit reference's generator
and gradients are pinned."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_1706_01307_amd as spc
from paper_1706_01307_amd import _lib
from tests import rows_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E = _lib.EINVAL
P = ctypes.c_void_p(4096)            # an address that no refused call follows
ODD = ctypes.c_void_p(4097)


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "spconv_rows.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(spconv_[a-z_]+)\s*\(", text))
    lib = _lib.load()
    assert names == set(_lib.ROWS_SIGNATURES)
    for n in names:
        assert hasattr(lib, n), n
    assert int(re.search(r"MAX_EXPERTS (\d+)", text).group(1)) == spc.ROUTE_MAX_EXPERTS
    assert int(re.search(r"MAX_SLOTS (\d+)", text).group(1)) == spc.ROUTE_MAX_SLOTS


def _refused(name, good, bad):
    """Each of `bad` ({argument index: value}) put into the call `good` is refused."""
    fn = getattr(_lib.load(), name)
    for change in bad:
        args = list(good)
        for i, v in change.items():
            args[i] = v
        assert fn(*args) == E, (name, change)


def test_layer_norm_refusals():
    good = [0, P, P, P, 1e-5, P, P, P, 4, 8, None]
    _refused("spconv_layer_norm_forward", good, [
        {0: 2}, {0: -1}, {1: None}, {1: ODD}, {2: ODD}, {3: ODD}, {4: -1e-5}, {4: float("nan")},
        {4: float("inf")}, {5: None}, {5: ODD}, {6: None}, {7: None}, {8: -1}, {8: 2 ** 31},
        {9: 0}, {9: -3}])
    good = [0, P, P, P, P, P, P, P, P, 4, 8, P, 64, None]
    _refused("spconv_layer_norm_backward", good, [
        {0: 2}, {1: None}, {2: None}, {3: None}, {4: None}, {5: ODD}, {6: None}, {7: None},
        {8: None}, {9: -1}, {10: 0}, {11: None}, {11: ctypes.c_void_p(4100)}, {12: 63}])
    n = ctypes.c_size_t()
    lib = _lib.load()
    assert lib.spconv_layer_norm_backward_workspace(4, 0, ctypes.byref(n)) == E
    assert lib.spconv_layer_norm_backward_workspace(4, 8, None) == E
    assert lib.spconv_layer_norm_backward_workspace(4, 8, ctypes.byref(n)) == 0 and n.value >= 64


def test_layer_norm_refuses_more_columns_than_its_sums_launch():
    good = [0, P, P, P, P, P, P, P, P, 4, 8, P, 2 ** 62, None]
    _refused("spconv_layer_norm_backward", good, [
        {10: 65535 * 256 + 1}, {10: 2 ** 31 - 256}, {9: 2 ** 31 - 1, 10: 65535 * 256}])


def test_dropout_refusals():
    _refused("spconv_dropout_forward", [0, P, P, 0.5, 1, 2, P, P, 8, None], [
        {0: 2}, {1: None}, {1: ODD}, {2: ODD}, {3: -0.1}, {3: 1.0}, {3: float("nan")},
        {6: ctypes.c_void_p(4100)}, {7: None}, {7: ODD}, {8: -1}, {8: 2 ** 34}])
    _refused("spconv_dropout_backward", [0, P, 0.5, 1, 2, None, P, 8, None], [
        {0: 2}, {1: None}, {2: 1.0}, {6: None}, {7: -1}])


def test_route_refusals():
    good = [0, P, 9, 8, 2, 1, P, P, P, P, P, P, 1 << 20, None]
    _refused("spconv_route_forward", good, [
        {0: 2}, {1: None}, {2: -1}, {3: 0}, {3: 1025}, {4: 0}, {4: 9}, {3: 32, 4: 17}, {5: 2},
        {6: None}, {7: None}, {8: None}, {9: None}, {10: None}, {8: ODD},
        {2: 100000, 11: None}, {2: 100000, 12: 16}, {2: 2 ** 30, 4: 2}])
    _refused("spconv_route_backward", [0, P, P, P, P, 9, 8, 2, 0, P, None], [
        {0: 2}, {1: None}, {2: None}, {3: None}, {4: None}, {5: -1}, {6: 0}, {7: 0}, {8: 2},
        {9: None}])
    n = ctypes.c_size_t()
    assert _lib.load().spconv_route_workspace(9, 8, 9, ctypes.byref(n)) == E
    assert _lib.load().spconv_route_workspace(9, 8, 2, None) == E


def test_grouped_refusals():
    good = [0, P, 9, P, P, P, P, 1, 0, P, 9, 4, 8, 8, None]
    _refused("spconv_grouped_forward", good, [
        {0: 2}, {1: None}, {1: ODD}, {2: -1}, {3: None}, {4: None}, {4: ODD}, {5: ODD},
        {5: None, 2: 8}, {6: ODD}, {7: 2}, {8: 2}, {9: None}, {10: -1}, {11: 0}, {11: 65536},
        {12: 0}, {13: 0}])
    _refused("spconv_grouped_backward_data", [0, P, P, P, P, 0, P, 9, 4, 8, 8, None], [
        {0: 2}, {1: None}, {2: None}, {3: None}, {4: ODD}, {5: 2}, {6: None}, {7: -1}, {8: 0},
        {9: 0}, {10: 0}])
    good = [0, P, 9, P, P, P, P, P, 9, 4, 8, 8, P, 1 << 30, None]
    _refused("spconv_grouped_backward_weight", good, [
        {0: 2}, {1: None}, {2: -1}, {3: None}, {4: None}, {5: ODD}, {5: None, 2: 8}, {6: None},
        {7: ODD}, {8: -1}, {9: 0}, {10: 0}, {11: 0},
        {2: 10 ** 6, 8: 10 ** 6, 12: None}, {2: 10 ** 6, 8: 10 ** 6, 13: 16}])
    n = ctypes.c_size_t()
    lib = _lib.load()
    assert lib.spconv_grouped_backward_weight_workspace(0, 9, 0, 8, 8, ctypes.byref(n)) == E
    assert lib.spconv_grouped_backward_weight_workspace(0, 9, 4, 8, 8, None) == E


def test_combine_refusals():
    _refused("spconv_combine_forward", [0, P, 9, P, P, P, P, 5, 2, 8, None], [
        {0: 2}, {1: None}, {2: -1}, {3: None}, {3: ODD}, {4: ODD}, {5: ODD}, {6: None}, {7: -1},
        {8: 0}, {8: 17}, {9: 0}])
    _refused("spconv_combine_backward", [0, P, P, P, P, P, P, P, 9, 5, 2, 8, None], [
        {0: 2}, {1: None}, {2: None}, {3: None}, {4: ODD}, {5: ODD}, {6: None}, {7: ODD}, {8: -1},
        {9: -1}, {10: 0}, {10: 17}, {11: 0}])


def test_binding_takes_cuda_tensors_only():
    x = torch.zeros(3, 4)
    for call in (lambda: spc.layer_norm_forward(x), lambda: spc.dropout_forward(x, 0.1, 0),
                 lambda: spc.route_forward(x, 1), lambda: spc.grouped_forward(x, x, x),
                 lambda: spc.combine_forward(x, x), lambda: spc.combine_backward(x, x, x)):
        with pytest.raises(TypeError):
            call()


def test_generator_gives_the_published_words():
    """The generator's published test vectors (7 and 10 rounds)."""
    for rounds, word, key, want in (
            (7, 0, 0, (0x5f6fb709, 0x0d893f64, 0x4f121f81, 0x4f730a48)),
            (7, 0xffffffff, 0xffffffff, (0x5207ddc2, 0x45165e59, 0x4d8ee751, 0x8c52f662)),
            (10, 0, 0, (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            (10, 0xffffffff, 0xffffffff, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd))):
        got = ref.philox(np.full((1, 4), word, np.uint32), (key, key), rounds)
        assert tuple(int(v) for v in got[0]) == want, (rounds, word)


def _difference(f, x, i, h=1e-6):
    a, b = x.clone(), x.clone()
    a.view(-1)[i] += h
    b.view(-1)[i] -= h
    return float((f(a) - f(b)) / (2 * h))


def test_reference_gradients_are_the_differences():
    """The gradients the GPU tests compare with, against central differences in 64 bits."""
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    x, ga, be, dy = r(3, 5), r(5), r(5), r(3, 5)
    y, mean, rstd, _ = ref.layer_norm(x, ga, be, 1e-3)
    (dx, dg, db), _ = ref.layer_norm_grad(dy, x, mean, rstd, ga)
    f = lambda a, b, c: (ref.layer_norm(a, b, c, 1e-3)[0] * dy).sum()
    for i in range(15):
        assert abs(_difference(lambda t: f(t, ga, be), x, i) - float(dx.view(-1)[i])) < 1e-7
    for i in range(5):
        assert abs(_difference(lambda t: f(x, t, be), ga, i) - float(dg[i])) < 1e-7
        assert abs(_difference(lambda t: f(x, ga, t), be, i) - float(db[i])) < 1e-7

    off, rows = np.array([0, 2, 2, 5]), torch.tensor([0, 3, 1, 0, 2])
    x, w, b, dy = r(4, 3), r(3, 3, 2), r(3, 2), r(5, 2)
    (dx, dw, db), _ = ref.grouped_grad(x, dy, w, off, rows, None)
    f = lambda a, v, c: (ref.grouped(a, v, off, rows, c, False)[0] * dy).sum()
    per_row = torch.zeros(4, 3, dtype=torch.float64).index_add_(0, rows, dx)
    for t, got, call in ((x, per_row, lambda v: f(v, w, b)), (w, dw, lambda v: f(x, v, b)),
                         (b, db, lambda v: f(x, w, v))):
        for i in range(t.numel()):
            assert abs(_difference(call, t, i) - float(got.reshape(-1)[i])) < 1e-7

    y, pos, wt, do = r(6, 3), torch.tensor([[0, 5], [2, -1], [4, 1]]), r(3, 2), r(3, 3)
    dy, dw, _ = ref.combine_grad(do, y, pos, wt)
    f = lambda a, v: (ref.combine(a, pos, v, None)[0] * do).sum()
    for t, got, call in ((y, dy, lambda v: f(v, wt)), (wt, dw, lambda v: f(y, v))):
        for i in range(t.numel()):
            assert abs(_difference(call, t, i) - float(got.reshape(-1)[i])) < 1e-7

    lg, dwt = r(4, 6), r(4, 2)
    for normalize in (True, False):
        e, wt, *_ = ref.route(lg.numpy(), 2, normalize)
        d = ref.route_grad(dwt.numpy(), lg.numpy(), e, wt, normalize)

        def f(t):
            p = torch.exp(t)
            p = p.gather(1, torch.from_numpy(e)) / (p.gather(1, torch.from_numpy(e)) if normalize
                                                    else p).sum(1, keepdim=True)
            return (p * dwt).sum()
        for i in range(24):
            assert abs(_difference(f, lg, i) - d.reshape(-1)[i]) < 1e-7
