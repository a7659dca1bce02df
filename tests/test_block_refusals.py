"""Layer norm, dropout and the gated feed-forward block: argument errors that are found before any device work, through the C
ABI and through the binding, and the oracle's gradients against differences.  No GPU needed."""
import ctypes
import math
import os

import pytest
import torch

import block_oracle as bo
import paper_2502_11490_amd as ann

P = ctypes.c_void_p(4096)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ann.lib_path()):
        from paper_2502_11490_amd.build import build

        build()
    return ann.load_library()


def _ln(lib, x=P, ld=8, gamma=P, beta=P, M=4, d=8, dtype=0, eps=1e-5, out=P, ld_out=8, mean=None, rstd=None):
    return lib.ann_layer_norm(x, ld, gamma, beta, M, d, dtype, eps, out, ld_out, mean, rstd, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(out=None), dict(d=0), dict(M=-1), dict(ld=7), dict(ld_out=7), dict(dtype=2),
                                 dict(dtype=9), dict(eps=-1e-5), dict(eps=math.nan), dict(eps=math.inf), dict(d=(1 << 24) + 1, ld=BIG),
                                 dict(x=ctypes.c_void_p(4098)), dict(gamma=ctypes.c_void_p(4097)), dict(mean=ctypes.c_void_p(4098))])
def test_layer_norm_refuses(lib, bad):
    assert _ln(lib, **bad) == -1 and lib.ann_last_error()


def test_rows_that_lie_on_each_other_are_refused_and_columns_side_by_side_are_not(lib):
    """4 fp32 rows of 8 about address 4096.  No device is reached: where the rows are in order a later check refuses."""
    at = lambda elements: ctypes.c_void_p(4096 + 4 * elements)  # noqa: E731
    assert _ln(lib, x=at(0), out=at(1)) == -1 and b"in common" in lib.ann_last_error()
    assert _ln(lib, x=at(0), ld=16, out=at(4), ld_out=16) == -1 and b"in common" in lib.ann_last_error()
    assert _ln(lib, x=at(0), ld=16, out=at(0), ld_out=24) == -1 and b"in common" in lib.ann_last_error()
    assert _ln(lib, x=at(0), ld=16, out=at(8), ld_out=16, gamma=ctypes.c_void_p(4097)) == -1 and b"aligned" in lib.ann_last_error()
    assert _ln(lib, x=at(8), ld=16, out=at(0), ld_out=16, gamma=ctypes.c_void_p(4097)) == -1 and b"aligned" in lib.ann_last_error()
    assert _ln(lib, x=at(0), out=at(0), gamma=ctypes.c_void_p(4097)) == -1 and b"aligned" in lib.ann_last_error()
    assert _ln_back(lib, dout=at(0), x=at(1 << 16), dx=at(1)) == -1 and b"dout_dev and dx_dev" in lib.ann_last_error()
    assert _ln_back(lib, dout=at(0), x=at(1 << 16), dx=at((1 << 16) + 8)) == -1 and b"x_dev and dx_dev" in lib.ann_last_error()
    assert lib.ann_dropout(at(0), None, at(1), 16, 0, 0.5, 1, 0, None, None) == -1 and b"overlap" in lib.ann_last_error()
    assert lib.ann_dropout(at(64), at(0), at(1), 16, 0, 0.5, 1, 0, None, None) == -1 and b"overlap" in lib.ann_last_error()
    assert _ffn(lib, x=at(0), ld=16, out=at(4), ld_out=16) == -1 and b"overlap" in lib.ann_last_error()
    assert _ffn(lib, x=at(0), ld=16, out=at(8), ld_out=16, ws=None) == -1 and b"workspace" in lib.ann_last_error()
    assert _ffn(lib, x=at(24), ld=16, out=at(0), ld_out=16, ws=None) == -1 and b"workspace" in lib.ann_last_error()


def test_layer_norm_of_no_rows(lib):
    assert _ln(lib, x=None, out=None, M=0) == 0


def _ln_back(lib, dout=P, ld_dout=8, x=P, ld=8, gamma=P, mean=P, rstd=P, M=4, d=8, dtype=0, dx=P, ld_dx=8, dg=P, db=P, ws=P, wb=BIG):
    return lib.ann_layer_norm_backward(dout, ld_dout, x, ld, gamma, mean, rstd, M, d, dtype, dx, ld_dx, dg, db, ws, wb, None)


@pytest.mark.parametrize("bad", [dict(dout=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(ws=None), dict(ld=7),
                                 dict(ld_dout=7), dict(ld_dx=7), dict(d=0), dict(dtype=2), dict(ws=ctypes.c_void_p(4100)),
                                 dict(dg=ctypes.c_void_p(4097)), dict(rstd=ctypes.c_void_p(4098))])
def test_layer_norm_backward_refuses(lib, bad):
    assert _ln_back(lib, **bad) == -1 and lib.ann_last_error()


def test_layer_norm_backward_workspace(lib):
    need = lib.ann_layer_norm_backward_workspace_bytes(4, 8, 0)
    assert need > 0 and _ln_back(lib, wb=need - 1) == -5
    assert lib.ann_layer_norm_backward_workspace_bytes(4, 0, 0) == 0 and lib.ann_layer_norm_backward_workspace_bytes(-1, 8, 0) == 0
    assert _ln_back(lib, dx=None, dg=None, db=None, ws=None, wb=0) == 0  # nothing is wanted


@pytest.mark.parametrize("bad", [dict(x=None), dict(out=None), dict(n=-1), dict(dtype=2), dict(p=-0.1), dict(p=1.1), dict(p=math.nan),
                                 dict(x=ctypes.c_void_p(4098)), dict(draw_dev=ctypes.c_void_p(4100)), dict(n=1 << 47)])
def test_dropout_refuses(lib, bad):
    a = dict(x=P, residual=None, out=P, n=16, dtype=0, p=0.5, draw_dev=None) | bad
    assert lib.ann_dropout(a["x"], a["residual"], a["out"], a["n"], a["dtype"], a["p"], 1, 0, a["draw_dev"], None) == -1
    assert lib.ann_last_error()


def test_dropout_of_nothing(lib):
    assert lib.ann_dropout(None, None, None, 0, 0, 0.5, 1, 0, None, None) == 0


def _ffn(lib, x=P, ld=8, wi=P, bi=None, wo=P, bo_=None, M=4, D=8, F=16, O=8, act=0, dtype=0, out=ctypes.c_void_p(1 << 20), ld_out=8,
         pre=None, ws=P, wb=BIG):
    return lib.ann_gated_ffn(x, ld, wi, bi, wo, bo_, M, D, F, O, act, dtype, out, ld_out, pre, ws, wb, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(wi=None), dict(wo=None), dict(out=None), dict(ws=None), dict(ld=7), dict(ld_out=7),
                                 dict(D=0), dict(F=0), dict(O=0), dict(M=-1), dict(M=1 << 31), dict(act=4), dict(act=-1), dict(dtype=2),
                                 dict(F=(1 << 20) + 1), dict(bi=ctypes.c_void_p(4097)), dict(pre=ctypes.c_void_p(4098)),
                                 dict(ws=ctypes.c_void_p(4100)), dict(out=ctypes.c_void_p(4096 + 64))])
def test_gated_ffn_refuses(lib, bad):
    assert _ffn(lib, **bad) == -1 and lib.ann_last_error()


def test_gated_ffn_sizes_and_no_rows(lib):
    need = lib.ann_gated_ffn_workspace_bytes(4, 8, 16, 8, 0)
    assert need > 0 and _ffn(lib, wb=need - 1) == -5
    assert lib.ann_gated_ffn_workspace_bytes(4, 8, 0, 8, 0) == 0 and lib.ann_gated_ffn_backward_workspace_bytes(4, 8, 16, 8, 2) == 0
    assert _ffn(lib, x=None, out=None, ws=None, M=0) == 0


def _ffn_back(lib, dout=P, ld_dout=8, x=P, ld=8, pre=P, wi=P, wo=P, M=4, D=8, F=16, O=8, act=0, dtype=0, dx=ctypes.c_void_p(1 << 20),
              ld_dx=8, dwi=P, dbi=P, dwo=P, dbo=P, ws=P, wb=BIG):
    return lib.ann_gated_ffn_backward(dout, ld_dout, x, ld, pre, wi, wo, M, D, F, O, act, dtype, dx, ld_dx, dwi, dbi, dwo, dbo, ws, wb,
                                      None)


@pytest.mark.parametrize("bad", [dict(dout=None), dict(x=None), dict(pre=None), dict(wi=None), dict(wo=None), dict(ws=None), dict(ld=7),
                                 dict(ld_dout=7), dict(ld_dx=7), dict(D=0), dict(act=7), dict(dtype=5), dict(dx=P),
                                 dict(dwi=ctypes.c_void_p(4097)), dict(pre=ctypes.c_void_p(4097)), dict(ws=ctypes.c_void_p(4100))])
def test_gated_ffn_backward_refuses(lib, bad):
    assert _ffn_back(lib, **bad) == -1 and lib.ann_last_error()


def test_gated_ffn_backward_workspace(lib):
    assert _ffn_back(lib, wb=lib.ann_gated_ffn_backward_workspace_bytes(4, 8, 16, 8, 0) - 1) == -5


@pytest.mark.parametrize("dtype", [0, 1, 3])
def test_gated_ffn_takes_no_more_rows_than_its_kernels_count(lib, dtype):
    """A reduction over M rows is counted in 32 bits, some steps past its end."""
    for M in ((1 << 29) + 1, (1 << 31) - 64, (1 << 31) - 1):
        assert lib.ann_gated_ffn_workspace_bytes(M, 1, 1, 1, dtype) == 0
        assert lib.ann_gated_ffn_backward_workspace_bytes(M, 1, 1, 1, dtype) == 0
        assert _ffn(lib, M=M, dtype=dtype) == -1 and b"2^29" in lib.ann_last_error()
        assert _ffn_back(lib, M=M, dtype=dtype) == -1 and b"2^29" in lib.ann_last_error()
    assert lib.ann_gated_ffn_workspace_bytes(1 << 29, 1, 1, 1, dtype) > 0
    assert lib.ann_gated_ffn_backward_workspace_bytes(1 << 29, 1, 1, 1, dtype) > 0


def test_binding_refuses():
    x, w = torch.zeros(4, 8), torch.zeros(8)
    for f in (lambda: ann.ann_layer_norm(x),                                     # not on a device
              lambda: ann.ann_layer_norm(x, torch.zeros(7)),
              lambda: ann.ann_layer_norm(x, w, out=torch.zeros(4, 9)),
              lambda: ann.ann_layer_norm(x.t(), torch.zeros(4)),
              lambda: ann.ann_layer_norm(x[:, :0]),
              lambda: ann.ann_layer_norm(torch.zeros(1, 8).expand(4, 8), w),     # rows that lie on each other
              lambda: ann.ann_layer_norm_backward(x[:3], x, w, torch.zeros(4), torch.zeros(4)),
              lambda: ann.ann_layer_norm_backward(x, x, w, torch.zeros(3), torch.zeros(4)),
              lambda: ann.ann_dropout(x, 0.5, 1),
              lambda: ann.ann_dropout(x.t(), 0.5, 1),
              lambda: ann.ann_dropout(x, 0.5, 1, residual=torch.zeros(4, 9)),
              lambda: ann.ann_dropout(x, 0.5, 1, draw_dev=torch.zeros(2, dtype=torch.int64)),
              lambda: ann.ann_gated_ffn(x, torch.zeros(32, 8), torch.zeros(8, 16)),
              lambda: ann.ann_gated_ffn(x, torch.zeros(31, 8), torch.zeros(8, 16)),
              lambda: ann.ann_gated_ffn(x, torch.zeros(32, 7), torch.zeros(8, 16)),
              lambda: ann.ann_gated_ffn(x, torch.zeros(32, 8), torch.zeros(8, 16), torch.zeros(31)),
              lambda: ann.ann_gated_ffn_backward(x, x, torch.zeros(4, 31), torch.zeros(32, 8), torch.zeros(8, 16))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ann.ann_layer_norm(x.double()), lambda: ann.ann_dropout(x.int(), 0.5, 1),
              lambda: ann.ann_layer_norm(x, w.half()), lambda: ann.ann_gated_ffn(x, torch.zeros(32, 8).half(), torch.zeros(8, 16)),
              lambda: ann.ann_layer_norm_backward(x, x, w, torch.zeros(4).double(), torch.zeros(4))):
        with pytest.raises(TypeError):
            f()


def test_oracle_draws_the_published_words():
    import json
    import numpy as np

    path = os.path.join(os.path.dirname(__file__), "golden", "philox4x32_10_kat.json")
    for c in json.load(open(path))["vectors"]:
        ctr, key, out = ([int(v, 16) for v in c[k]] for k in ("ctr", "key", "out"))
        got = bo.philox_words(np.array([ctr[0] | ctr[1] << 32], dtype=np.uint64), ctr[2], ctr[3], key[0], key[1])[0]
        assert [int(v) for v in got] == out


@pytest.mark.parametrize("act", range(4))
def test_oracle_gradients_against_differences(act):
    """Central differences of the definitions in fp64: a step of 1e-5 leaves about 1e-10 (third derivatives) + 1e-11 (rounding)."""
    g = torch.Generator().manual_seed(act)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, wi, wo, bi, bo_, dy = r(5, 7), r(12, 7), r(3, 6), r(12), r(3), r(5, 3)
    f = lambda x, wi, wo, bi, b: (bo.ffn(x, wi, wo, bi, b, act, torch.float32)[0] * dy).sum()  # noqa: E731
    pre = bo.ffn(x, wi, wo, bi, bo_, act, torch.float32)[1]
    grads = bo.ffn_grad(dy, x, pre, wi, wo, act, torch.float32)[0]
    args = [x, wi, wo, bi, bo_]
    for i, grad in enumerate(grads):
        v = r(*args[i].shape)
        plus, minus = ([a + s * 1e-5 * v if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        assert abs((f(*plus) - f(*minus)) / 2e-5 - (grad * v).sum()) < 1e-6 * max(1.0, float(grad.norm() * v.norm()))
    gamma, beta, eps = r(7), r(7), 1e-3
    dy = r(5, 7)
    f = lambda x, g_, b: (bo.layer_norm(x, g_, b, eps)[0] * dy).sum()  # noqa: E731
    _, mean, rstd, _ = bo.layer_norm(x, gamma, beta, eps)
    for i, grad in enumerate(bo.layer_norm_grad(dy, x, gamma, mean, rstd)[0]):
        args = [x, gamma, beta]
        v = r(*args[i].shape)
        plus, minus = ([a + s * 1e-5 * v if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        assert abs((f(*plus) - f(*minus)) / 2e-5 - (grad * v).sum()) < 1e-6 * max(1.0, float(grad.norm() * v.norm()))
