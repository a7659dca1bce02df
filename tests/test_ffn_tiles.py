"""Every tile of the gated feed-forward block's products against the definition: both tile sizes of either kind of type, every
layout of the operands and every epilogue, whole and cut along k.  Which tile a size takes is the library's choice; it is
asked for it, so that a change of that choice shows here and does not leave a tile without a test."""
import ctypes
import os

import pytest
import torch

import paper_2502_11490_amd as ann

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STORE, GATE, GRAD = 0, 1, 2

# (rows, d_in, d_hidden, d_out): odd sizes, which are packed and end inside a tile, and multiples of 8, which are not packed
SIZES16 = [(71, 71, 65, 91), (65, 69, 939, 67), (65, 605, 65, 121), (821, 69, 83, 71), (1165, 3747, 1691, 123),
           (1160, 3744, 1688, 120), (3873, 787, 3847, 1263), (3872, 784, 3848, 1264), (6613, 2017, 605, 1883),
           (6616, 2016, 608, 1880)]
SIZES32 = [(71, 65, 71, 113), (75, 67, 569, 95), (71, 589, 75, 75), (549, 67, 75, 103), (5075, 77, 1805, 71), (5076, 80, 1808, 72),
           (3211, 2351, 97, 2013), (69, 151, 3497, 4487)]


class Cut(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("cols", ctypes.c_int), ("splits", ctypes.c_int)]


def _cuts(kind, M, D, F, O):
    """How each product of the block and of its gradient is cut: {(product, columns of the tile, whether k is cut)}."""
    if not os.path.exists(ann.lib_path()):
        from paper_2502_11490_amd.build import build

        build()
    f = getattr(ann.load_library(), "_ZN5gmpgr7ffn_cutEillli")  # gmpgr::ffn_cut(kind, M, N, K, epilogue)
    f.restype, f.argtypes = Cut, [ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_int]
    products = [("gate", M, F, D, GATE), ("out", M, O, F, STORE), ("grad", M, F, O, GRAD), ("dx", M, D, 2 * F, STORE),
                ("dw", 2 * F, D, M, STORE), ("dw", O, F, M, STORE)]
    cuts = [(name, f(kind, m, n, k, epi)) for name, m, n, k, epi in products]
    return {(name, c.cols, c.splits > 1) for name, c in cuts}


@pytest.mark.parametrize("kind,sizes,tiles", [(ann.ANN_F32, SIZES32, (64, 128)), (ann.ANN_BF16, SIZES16, (128, 256)),
                                              (ann.ANN_F16, SIZES16, (128, 256))])
def test_sizes_take_every_tile(kind, sizes, tiles):
    want = {(p, t, cut) for p in ("gate", "out", "grad", "dx", "dw") for t in tiles for cut in (False, True) if p != "grad" or not cut}
    for some in (sizes,) if kind == ann.ANN_F32 else (sizes, [s for s in sizes if all(w % 8 for w in s)]):
        assert set().union(*(_cuts(kind, *s) for s in some)) == want
    assert {c for s in sizes if all(w % 8 == 0 for w in s[1:]) for c in _cuts(kind, *s) if c[1] == tiles[1]}


def _check(sizes, dtype):
    from test_gpu_block import _check_ffn, _ffn_case

    print(sizes, dtype, flush=True)
    _check_ffn(*_ffn_case(*sizes, dtype, True), act=sum(sizes) % 4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("sizes", SIZES16, ids=str)
def test_tiles_of_the_16_bit_products(sizes, dtype):
    _check(sizes, TYPES[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES32, ids=str)
def test_tiles_of_the_fp32_products(sizes):
    _check(sizes, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M", [17, 20, 32, 33, 50, 64])
def test_few_rows_of_a_wide_gate(M, dtype):
    """From 32 x 256 gate columns on a workgroup of the few-row kernel takes 32 of them."""
    _check((M, 129, 8195, 40), TYPES[dtype])
