"""libdscores on the host: exported symbols, refusals of the C ABI and of the binding.  No call here
reaches a kernel: each is refused, or has no rows."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests import scoreutil as SU

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_1111_1373_amd")

dt = pytest.importorskip("paper_1111_1373_amd.dtree", reason="libdtree.so not built")
sc = pytest.importorskip("paper_1111_1373_amd.scores", reason="libdscores.so not built")

A = 4096                          # an aligned address that no refused call reads
INVALID, UNSUPPORTED = dt.DT_ERR_INVALID_ARG, dt.DT_ERR_UNSUPPORTED
NAN, INF = float("nan"), float("inf")


def test_every_declared_symbol_is_exported():
    src = open(os.path.join(ROOT, "include", "dtree_scores.h")).read()
    names = set(re.findall(r"\b(ds_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", src, flags=re.S)))
    assert names == set(sc._PROTOS)
    out = subprocess.run(["nm", "-D", "--defined-only", sc.LIB_PATH], capture_output=True,
                         text=True, check=True).stdout
    assert names <= set(re.findall(r"\sT\s(\w+)$", out, re.M))


def test_header_is_c11(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    src = tmp_path / "t.c"
    src.write_text('#include "dtree_scores.h"\n'
                   "int main(void) { return ds_distill_work_bytes(0, 1) == 0 && "
                   "ds_sample(0, DT_F32, -1, 1, 1, 0, 0, 0, 0) == DT_ERR_INVALID_ARG && "
                   "ds_last_error()[0] != 0 ? 0 : 1; }\n")
    exe = str(tmp_path / "t")
    subprocess.run(["gcc", "-std=c11", "-pedantic", "-Wall", "-Wextra", "-Werror",
                    "-I" + os.path.join(ROOT, "include"), str(src), "-L" + PKG, "-ldscores",
                    "-Wl,-rpath," + PKG, "-o", exe], check=True, capture_output=True, text=True)
    assert subprocess.run([exe], timeout=120).returncode == 0


def _top(x=A, type=0, n=4, classes=10, ld=10, k=2, values=A, index=A, lse=A):
    return sc._lib.ds_top_scores(x, type, n, classes, ld, k, values, index, lse, None)


def _sample(x=A, type=0, n=4, classes=10, ld=10, u=A, labels=A, settings=True, **set):
    s = sc.Sampling(temperature=1.0, top_p=1.0)
    for name, v in set.items():
        setattr(s, name, v)
    return sc._lib.ds_sample(x, type, n, classes, ld, u, ctypes.byref(s) if settings else None,
                             labels, None)


def _distill(x=A, type=0, n=4, classes=10, ld=10, values=A, index=A, k=2, t=1.0, g=A, loss=A,
             stats=A, grad=A, ld_grad=10, work=None, bytes=0):
    return sc._lib.ds_distill(x, type, n, classes, ld, values, index, k, t, g, loss, stats, grad,
                              ld_grad, work, bytes, None)


def _backward(x=A, type=0, n=4, classes=10, ld=10, values=A, index=A, k=2, t=1.0, stats=A, g=A,
              grad=A, ld_grad=10):
    return sc._lib.ds_distill_backward(x, type, n, classes, ld, values, index, k, t, stats, g, grad,
                                       ld_grad, None)


ROWS = [(INVALID, dict(x=None)), (INVALID, dict(type=4)), (INVALID, dict(type=-1)),
        (INVALID, dict(n=-1)), (INVALID, dict(classes=0)), (INVALID, dict(ld=9)),
        (INVALID, dict(x=A + 2)), (INVALID, dict(x=A + 1, type=1)),
        (UNSUPPORTED, dict(classes=(1 << 20) + 1, ld=1 << 21)), (UNSUPPORTED, dict(n=1 << 31)),
        (UNSUPPORTED, dict(ld=1 << 41))]


@pytest.mark.parametrize("call", [_top, _sample, _distill, _backward])
@pytest.mark.parametrize("status,args", ROWS)
def test_refused_rows(call, status, args):
    assert call(**args) == status
    assert sc._lib.ds_last_error()


@pytest.mark.parametrize("args", [dict(k=0), dict(k=11), dict(k=257, classes=1000, ld=1000),
                                  dict(values=None), dict(index=None), dict(lse=None),
                                  dict(values=A + 1), dict(index=A + 2), dict(lse=A + 3)])
def test_refused_top_scores(args):
    assert _top(**args) == INVALID


@pytest.mark.parametrize("args", [dict(u=None), dict(labels=None), dict(settings=False),
                                  dict(temperature=-0.5), dict(temperature=NAN),
                                  dict(temperature=INF), dict(top_p=-0.1), dict(top_p=NAN),
                                  dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=NAN),
                                  dict(u=A + 1), dict(labels=A + 2), dict(d_temperature=A + 1),
                                  dict(d_top_k=A + 2), dict(d_top_p=A + 1), dict(d_min_p=A + 3)])
def test_refused_sample(args):
    assert _sample(**args) == INVALID


TEACH = [dict(type=3), dict(k=0), dict(k=257), dict(t=0.0), dict(t=-1.0), dict(t=NAN), dict(t=INF),
         dict(t=1e-39), dict(values=None), dict(index=None), dict(values=A + 1),
         dict(index=A + 2), dict(g=None), dict(grad=None), dict(g=A + 1), dict(grad=A + 2),
         dict(ld_grad=9), dict(stats=None), dict(stats=A + 4)]


@pytest.mark.parametrize("args", TEACH)
def test_refused_backward(args):
    assert _backward(**args) == INVALID


@pytest.mark.parametrize("args", TEACH + [dict(loss=None), dict(loss=A + 2)])
def test_refused_distill(args):
    assert _distill(**args) == INVALID


def test_workspace():
    need = sc._lib.ds_distill_work_bytes(3, 50_000)
    assert need > 0 and need % 8 == 0
    long = dict(n=3, classes=50_000, ld=50_000, ld_grad=50_000)
    assert _distill(**long) == INVALID
    assert _distill(**long, work=A, bytes=need - 1) == INVALID
    assert _distill(**long, work=A + 4, bytes=need) == INVALID
    for n, classes in ((0, 50_000), (-3, 9), (1 << 20, 50_000), (4, 100), (4, 0), (4, 1 << 21)):
        assert sc._lib.ds_distill_work_bytes(n, classes) == 0


def test_no_rows_launch_nothing():
    assert _top(x=None, n=0, values=None, index=None, lse=None) == 0
    assert _sample(x=None, n=0, u=None, labels=None) == 0
    assert _distill(x=None, n=0, values=None, index=None, g=None, loss=None, stats=None, grad=None) == 0
    assert _backward(x=None, n=0, values=None, index=None, g=None, stats=None, grad=None) == 0


def test_the_binding_refuses_what_is_not_on_a_gpu():
    x = torch.zeros(3, 5)
    with pytest.raises(TypeError):
        sc.top_scores(x, 2)
    with pytest.raises(TypeError):
        sc.sample(x.numpy(), torch.zeros(3))
    with pytest.raises(TypeError):
        sc.distill_loss(x, torch.zeros(3, 1), torch.zeros(3, 1, dtype=torch.int32))


def test_votes_are_an_answer_of_forests_on_the_device():
    n = np.zeros(3, dtype=dt.NODE_DTYPE)
    n["cls"] = (-1, 0, 1)
    n["left"][0] = 1
    assert dt.OUT_KINDS["votes_u8"] == 3
    assert dt._lib.dt_forest_classify_host(None, None, None, 0, 1, None, 3, 0, None) == INVALID
    assert b"classes" in dt._lib.dt_last_error()


# ---- the plain implementations that the GPU tests compare with ------------------------------

def test_oracle_by_hand():
    x = np.array([[1.0, 3.0, 3.0, -INF, NAN]], dtype=np.float32)
    v, i, l = SU.top_scores(x, 4)
    assert i.tolist() == [[1, 2, 0, -1]] and v[0, 3] == -INF
    assert abs(l[0] - np.log(2 * np.exp(3) + np.exp(1))) < 1e-12
    votes = np.array([[1, 0, 5, 2, 2]], dtype=np.uint8)
    # in the classes' order: 1, 0, 5, 2, 2 of 10
    for u, c in ((0.0, 0), (0.0999, 0), (0.1, 2), (0.59, 2), (0.6, 3), (0.79, 3), (0.8, 4)):
        assert SU.sample(votes, [u]) == c
    assert SU.sample(votes, [0.99], top_k=2) == 3               # 5 and the first 2
    assert SU.sample(votes, [0.99], top_p=0.5) == 2             # 5 of 10 is half
    assert SU.sample(votes, [0.99], top_p=0.51) == 3
    assert SU.sample(votes, [0.99], min_p=0.5) == 2
    assert SU.sample(votes, [0.99], min_p=0.375) == 4
    assert SU.sample(votes, [0.99], temperature=0) == 2
    assert SU.sample(np.zeros((1, 3), np.uint8), [0.5]) == -1


def test_oracle_gradient_is_the_loss_slope():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 6))
    values, index = rng.standard_normal((2, 3)), np.array([[0, 2, 2], [5, -1, 1]])
    g = np.array([0.3, 2.0])
    _, grad = SU.distill(x, values, index, 1.5, g)
    h = 1e-6
    for r in range(2):
        for c in range(6):
            d = np.zeros_like(x)
            d[r, c] = h
            slope = (SU.distill(x + d, values, index, 1.5, g)[0][r]
                     - SU.distill(x - d, values, index, 1.5, g)[0][r]) / (2 * h)
            assert abs(g[r] * slope - grad[r, c]) < 1e-8
