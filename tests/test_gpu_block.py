"""Layer norm, dropout and the gated feed-forward block on the device against their definitions in fp64."""
import numpy as np
import pytest
import torch

import block_oracle as bo
import paper_2502_11490_amd as ann

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]


def _randn(gen, *shape, dtype=torch.float32, scale=1.0, shift=0.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dtype)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _slice_of(t, left=1, right=2):
    """The same values as rows of a wider array, at an odd element offset."""
    wide = torch.full((t.shape[0], t.shape[1] + left + right), 7.0, dtype=t.dtype, device=t.device)
    wide[:, left:left + t.shape[1]] = t
    return wide[:, left:left + t.shape[1]], wide


# ---- layer norm


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("M,d", [(1, 1), (3, 2), (257, 7), (64, 32), (33, 100), (1025, 256), (5, 513), (130, 1000), (9, 2051),
                                 (700, 4096), (6, 4099), (3, 8200), (2, 16384), (3, 16391), (2, 40001)])
def test_layer_norm_and_gradient(M, d, dtype):
    gen = _gen(M * 7 + d)
    x = (torch.randn(M, d, generator=gen, device="cuda") * (torch.rand(M, 1, generator=gen, device="cuda") + 0.1)
         + 3 * torch.randn(M, 1, generator=gen, device="cuda")).to(dtype)
    gamma, beta = _randn(gen, d, dtype=dtype, scale=0.3, shift=1), _randn(gen, d, dtype=dtype)
    dout, eps = _randn(gen, M, d, dtype=dtype), 1e-3
    out, mean, rstd = ann.ann_layer_norm(x, gamma, beta, eps, save=True)
    want, wm, wr, bound = bo.layer_norm(x, gamma, beta, eps)
    bo.assert_close(out, want, bound, "out")
    row = x.double().abs().amax(1)
    n = (d / 1024 + 48) * bo.U
    bo.assert_close(mean, wm, n * row, "mean")
    # a relative change of var + eps by e changes rstd by e / 2: the deviations are off by n row, the sum by n of itself
    bo.assert_close(rstd, wr, wr * (n + n * row * wr * 2 + (n * row * wr) ** 2 + 4 * bo.U), "rstd")
    got = ann.ann_layer_norm_backward(dout, x, gamma, mean, rstd)
    values, bounds = bo.layer_norm_grad(dout, x, gamma, mean, rstd)
    for name, a, b, c in zip(("dx", "dgamma", "dbeta"), got, values, bounds):
        bo.assert_close(a, b, c, name)
    again = ann.ann_layer_norm_backward(dout, x, gamma, mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_layer_norm_without_parameters_constant_rows_and_bad_rows(dtype):
    x = torch.randn(5, 300, device="cuda").to(dtype)
    x[1] = 2.5            # variance 0: out = 0
    x[2, 7] = float("inf")
    x[3, 299] = float("nan")
    out, mean, rstd = ann.ann_layer_norm(x, eps=1e-5, save=True)
    assert bool((out[1] == 0).all()) and bool(out[2].isnan().all()) and bool(out[3].isnan().all())
    for r in (0, 4):
        want, _, _, bound = bo.layer_norm(x[r:r + 1], None, None, 1e-5)
        bo.assert_close(out[r:r + 1], want, bound)
    dx, dg, db = ann.ann_layer_norm_backward(torch.ones_like(x), x, None, mean, rstd)
    assert bool(dx[2].isnan().all()) and bool(dx[[0, 1, 4]].isfinite().all())
    assert bool((db == 5).all())


@pytest.mark.parametrize("d", [37, 1032, 5001, 20003])
def test_layer_norm_strides_in_place_and_neighbours(d):
    gen = _gen(d)
    x, dout = _randn(gen, 11, d, dtype=torch.float16), _randn(gen, 11, d, dtype=torch.float16)
    gamma, beta = (_randn(gen, d + 1, dtype=torch.float16)[1:] for _ in range(2))  # at an odd element
    want, mean, rstd = ann.ann_layer_norm(x, gamma, beta, save=True)
    xs, _ = _slice_of(x)
    out, wide = _slice_of(torch.zeros_like(x))
    assert ann.ann_layer_norm(xs, gamma, beta, out=out) is out and torch.equal(out, want)
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, -2:] == 7).all())
    dx, dg, db = ann.ann_layer_norm_backward(_slice_of(dout)[0], xs, gamma, mean, rstd)
    for a, b in zip((dx, dg, db), ann.ann_layer_norm_backward(dout, x, gamma, mean, rstd)):
        assert torch.equal(a, b)
    # the C entry writes dx over dout
    lib, mine = ann.load_library(), dout.clone()
    ws = torch.empty(ann.ann_layer_norm_backward_workspace_bytes(11, d, ann.ANN_F16), dtype=torch.uint8, device="cuda")
    dgb = torch.empty(2, d, dtype=torch.float16, device="cuda")
    rc = lib.ann_layer_norm_backward(mine.data_ptr(), d, x.data_ptr(), d, gamma.data_ptr(), mean.data_ptr(), rstd.data_ptr(), 11, d,
                                     ann.ANN_F16, mine.data_ptr(), d, dgb[0].data_ptr(), dgb[1].data_ptr(), ws.data_ptr(),
                                     ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(mine, dx) and torch.equal(dgb[0], dg) and torch.equal(dgb[1], db)
    ann.ann_layer_norm(x, gamma, beta, out=x)
    assert torch.equal(x, want)


def test_layer_norm_of_no_rows_and_parts_not_wanted():
    x = torch.empty(0, 9, device="cuda")
    out, mean, rstd = ann.ann_layer_norm(x, save=True)
    assert out.shape == (0, 9) and mean.shape == (0,)
    dx, dg, db = ann.ann_layer_norm_backward(x, x, None, mean, rstd)
    assert dx.shape == (0, 9) and bool((dg == 0).all()) and bool((db == 0).all())
    x = torch.randn(6, 9, device="cuda")
    out, mean, rstd = ann.ann_layer_norm(x, save=True)
    full = ann.ann_layer_norm_backward(out, x, None, mean, rstd)
    assert torch.equal(ann.ann_layer_norm_backward(out, x, None, mean, rstd, need_dparams=False)[0], full[0])
    part = ann.ann_layer_norm_backward(out, x, None, mean, rstd, need_dx=False)
    assert part[0] is None and torch.equal(part[1], full[1]) and torch.equal(part[2], full[2])


def test_layer_norm_offsets_past_32_bits():
    M, d = (1 << 20) + 3, 2051
    x = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    x.normal_()
    out, mean, rstd = ann.ann_layer_norm(x, save=True)
    dx, _, db = ann.ann_layer_norm_backward(out, x, None, mean, rstd)
    want, _, _, bound = bo.layer_norm(x[-3:], None, None, 1e-5)
    bo.assert_close(out[-3:], want, bound)
    values, bounds = bo.layer_norm_grad(out[-3:], x[-3:], None, mean[-3:], rstd[-3:])
    bo.assert_close(dx[-3:], values[0], bounds[0])


# ---- dropout


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [1, 7, 8, 9, 1000, 65543])
@pytest.mark.parametrize("p,seed,draw", [(0.25, 5, 0), (0.9, (7 << 40) + 3, (3 << 33) + 1)])
def test_dropout(n, p, seed, draw, dtype):
    gen = _gen(n)
    x, r = _randn(gen, n, dtype=dtype), _randn(gen, n, dtype=dtype)
    k, scale = bo.kept(np.arange(n), p, seed, draw)
    k = torch.from_numpy(k).cuda()
    want = torch.where(k, x.double() * scale, 0.0)
    bo.assert_close(ann.ann_dropout(x, p, seed, draw), want, 4 * bo.U * want.abs())
    bo.assert_close(ann.ann_dropout(x, p, seed, draw, residual=r), want + r.double(), 4 * bo.U * (want.abs() + r.double().abs()))
    # at an odd element, and in place
    xo, ro = (torch.cat((t[:1], t))[1:] for t in (x, r))
    assert torch.equal(ann.ann_dropout(xo, p, seed, draw, residual=ro, out=ro), ann.ann_dropout(x, p, seed, draw, residual=r))
    assert torch.equal(ann.ann_dropout(xo, p, seed, draw, out=xo), ann.ann_dropout(x, p, seed, draw))


def test_dropout_keeps_all_or_nothing_and_selects():
    x, r = torch.randn(4099, device="cuda"), torch.randn(4099, device="cuda")
    assert torch.equal(ann.ann_dropout(x, 0.0, 1), x)
    assert torch.equal(ann.ann_dropout(x, 1.0, 1, residual=r), r)
    k = torch.from_numpy(bo.kept(np.arange(4099), 0.5, 9, 2)[0]).cuda()
    bad = x.masked_fill(~k, float("nan"))
    bad[~k & (r > 0)] = float("inf")
    assert torch.equal(ann.ann_dropout(bad, 0.5, 9, 2), ann.ann_dropout(x, 0.5, 9, 2))
    assert ann.ann_dropout(torch.empty(0, 5, device="cuda"), 0.5, 1).shape == (0, 5)
    # 2^22 draws: the number kept is within 6 standard deviations
    n, p = 1 << 22, 0.3
    kept = int((ann.ann_dropout(torch.ones(n, device="cuda"), p, 3) != 0).sum())
    assert abs(kept - n * (1 - p)) < 6 * (n * p * (1 - p)) ** 0.5


def test_dropout_words_are_not_the_noise_words():
    """Under one seed and draw the two operators draw apart: the uniforms behind the noise do not choose what is dropped."""
    n = 1 << 16
    noise = ann.ann_users_add_noise(torch.zeros(1, n, device="cuda"), 1.0, 11, 4)[0]
    kept = ann.ann_dropout(torch.ones(n, device="cuda"), 0.5, 11, 4) != 0
    for shift in (1, 2):
        a = noise.abs()[::shift][:n // 2] > 0.6745
        assert abs(float((a == kept[:n // 2]).float().mean()) - 0.5) < 6 * 0.5 / (n // 2) ** 0.5


def test_dropout_offsets_past_32_bits():
    n = (1 << 32) + 13
    x = torch.ones(n, dtype=torch.float16, device="cuda")
    out = ann.ann_dropout(x, 0.5, 21, 3, out=x)
    at = np.arange(n - 4000, n)
    assert torch.equal(out[-4000:].cpu(), torch.from_numpy(bo.kept(at, 0.5, 21, 3)[0]).half() * 2)
    assert torch.equal(out[:4000].cpu(), torch.from_numpy(bo.kept(np.arange(4000), 0.5, 21, 3)[0]).half() * 2)


def test_dropout_replays_draw_anew():
    x, step = torch.randn(5000, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ann.ann_dropout(x, 0.5, 7, 100, draw_dev=step)
    for i in range(4):
        step.fill_(i * i)
        graph.replay()
        assert torch.equal(out, ann.ann_dropout(x, 0.5, 7, 100 + i * i))


# ---- gated feed-forward block


def _ffn_case(M, D, F, O, dtype, bias, seed=0):
    gen = _gen(M + 3 * D + 5 * F + 7 * O + seed)
    x = _randn(gen, M, D, dtype=dtype)
    w_in, w_out = _randn(gen, 2 * F, D, dtype=dtype, scale=D ** -0.5), _randn(gen, O, F, dtype=dtype, scale=F ** -0.5)
    b_in, b_out = (_randn(gen, 2 * F, dtype=dtype), _randn(gen, O, dtype=dtype)) if bias else (None, None)
    return x, w_in, w_out, b_in, b_out, _randn(gen, M, O, dtype=dtype)


def _check_ffn(x, w_in, w_out, b_in, b_out, dout, act):
    dtype = x.dtype
    out, pre = ann.ann_gated_ffn(x, w_in, w_out, b_in, b_out, act, save=True)
    want, z, bound, z_err = bo.ffn(x, w_in, w_out, b_in, b_out, act, dtype)
    bo.assert_close(pre, z, z_err, "pre")
    bo.assert_close(out, want, bound, "out")
    bo.assert_close(ann.ann_gated_ffn(x, w_in, w_out, b_in, b_out, act), want, bound, "out without pre")
    got = ann.ann_gated_ffn_backward(dout, x, pre, w_in, w_out, act, bias=True)
    values, bounds = bo.ffn_grad(dout, x, pre, w_in, w_out, act, dtype)
    for name, a, b, c in zip(("dx", "dw_in", "dw_out", "db_in", "db_out"), got, values, bounds):
        bo.assert_close(a, b, c, name)
    return out, pre, got


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("M,D,F,O", [(1, 1, 1, 1), (1, 64, 128, 64), (1, 2048, 500, 72), (2, 8, 16, 24), (3, 33, 65, 17), (16, 128, 256, 128),
                                     (17, 72, 200, 40), (37, 256, 513, 129), (64, 1024, 256, 256), (65, 512, 1024, 8), (129, 136, 264, 72),
                                     (200, 100, 36, 300), (257, 384, 640, 192), (1000, 72, 1032, 64), (5, 3000, 40, 2000),
                                     (520, 520, 520, 520)])
def test_gated_ffn_and_gradient(M, D, F, O, dtype):
    _check_ffn(*_ffn_case(M, D, F, O, dtype, (M + F) % 2 == 0), act=(M + D) % 4)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("act", range(4))
def test_gated_ffn_activations(act, dtype):
    x, *rest = _ffn_case(70, 48, 104, 56, dtype, True, seed=act)
    x[:20] *= 8  # far into the activations' tails
    _check_ffn(x, *rest, act=act)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("M", [1, 9, 300])
def test_gated_ffn_strides_alignment_and_neighbours(M, dtype):
    x, w_in, w_out, b_in, b_out, dout = _ffn_case(M, 72, 136, 40, dtype, True)
    out, pre, got = _check_ffn(x, w_in, w_out, b_in, b_out, dout, ann.ANN_GELU)
    want, z, bound, z_err = bo.ffn(x, w_in, w_out, b_in, b_out, ann.ANN_GELU, dtype)
    off = lambda t: torch.cat((t.flatten()[:1], t.flatten()))[1:].view(t.shape)  # noqa: E731  at an odd element
    xs, dos = _slice_of(x)[0], _slice_of(dout)[0]
    res, wide = _slice_of(torch.zeros_like(out))
    ann.ann_gated_ffn(xs, off(w_in), off(w_out), off(b_in), off(b_out), ann.ANN_GELU, out=res)
    bo.assert_close(res, want, bound)
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, -2:] == 7).all())
    values, bounds = bo.ffn_grad(dout, x, pre, w_in, w_out, ann.ANN_GELU, dtype)
    for a, b, c in zip(ann.ann_gated_ffn_backward(dos, xs, off(pre), off(w_in), off(w_out), ann.ANN_GELU, bias=True), values, bounds):
        bo.assert_close(a, b, c)
    # rows 16-byte aligned but wider than the vectors: the direct loads with a stride of their own
    big = torch.full((M, 104), 7.0, dtype=dtype, device="cuda")
    big[:, 8:80] = x
    bo.assert_close(ann.ann_gated_ffn(big[:, 8:80], w_in, w_out, b_in, b_out, ann.ANN_GELU), want, bound)


def test_gated_ffn_parts_not_wanted_no_rows_and_workspace():
    x, w_in, w_out, b_in, b_out, dout = _ffn_case(40, 64, 96, 32, torch.bfloat16, True)
    _, pre = ann.ann_gated_ffn(x, w_in, w_out, b_in, b_out, save=True)
    full = ann.ann_gated_ffn_backward(dout, x, pre, w_in, w_out, bias=True)
    a = ann.ann_gated_ffn_backward(dout, x, pre, w_in, w_out, need_dw=False)
    assert torch.equal(a[0], full[0]) and a[1:] == (None,) * 4
    b = ann.ann_gated_ffn_backward(dout, x, pre, w_in, w_out, need_dx=False, bias=True)
    assert b[0] is None and all(torch.equal(p, q) for p, q in zip(b[1:], full[1:]))
    out, pre0 = ann.ann_gated_ffn(x[:0], w_in, w_out, save=True)
    assert out.shape == (0, 32)
    g = ann.ann_gated_ffn_backward(dout[:0], x[:0], pre0, w_in, w_out, bias=True)
    assert g[0].shape == (0, 64) and all(bool((t == 0).all()) for t in g[1:])
    ws = torch.empty(ann.ann_gated_ffn_workspace_bytes(40, 64, 96, 32, ann.ANN_BF16), dtype=torch.uint8, device="cuda")
    ws.fill_(255)  # NaN in every type: nothing that the call has not written is read
    assert torch.equal(ann.ann_gated_ffn(x, w_in, w_out, b_in, b_out, workspace=ws), ann.ann_gated_ffn(x, w_in, w_out, b_in, b_out))
    wb = torch.empty(ann.ann_gated_ffn_backward_workspace_bytes(40, 64, 96, 32, ann.ANN_BF16), dtype=torch.uint8, device="cuda").fill_(255)
    for p, q in zip(ann.ann_gated_ffn_backward(dout, x, pre, w_in, w_out, bias=True, workspace=wb), full):
        assert torch.equal(p, q)
    with pytest.raises(ann.AnnError):
        ann.ann_gated_ffn(x, w_in, w_out, workspace=ws[:256])
    with pytest.raises(ann.AnnError):
        ann.ann_gated_ffn(x, w_in, w_out, act=9)
    with pytest.raises(ann.AnnError):
        ann.ann_gated_ffn(x, w_in, w_out, out=x[:, :32])  # out over x


@pytest.mark.parametrize("M", [1, 12, 150])
def test_gated_ffn_keeps_rows_apart(M):
    """A row of NaN or infinities leaves the other rows as they are, and the rows behind the last one are not touched."""
    x, w_in, w_out, b_in, b_out, _ = _ffn_case(M + 3, 200, 120, 56, torch.bfloat16, True)
    want = ann.ann_gated_ffn(x[:M].clone(), w_in, w_out, b_in, b_out)
    x[M] = float("nan")
    x[M + 1] = float("inf")
    out = torch.full((M + 3, 56), 7.0, dtype=torch.bfloat16, device="cuda")
    ann.ann_gated_ffn(x[:M], w_in, w_out, b_in, b_out, out=out[:M])
    assert torch.equal(out[:M], want) and bool((out[M:] == 7).all())


def test_gated_ffn_offsets_past_32_bits():
    """pre, and the gradient of gate and up, hold more than 2^31 elements."""
    M, D, F, O = 70000, 64, 16384, 64
    x, w_in, w_out, b_in, b_out, dout = _ffn_case(M, D, F, O, torch.bfloat16, False)
    out, pre = ann.ann_gated_ffn(x, w_in, w_out, save=True)
    dx, _, _, _, _ = ann.ann_gated_ffn_backward(dout, x, pre, w_in, w_out, need_dw=False)
    want, z, bound, z_err = bo.ffn(x[-5:], w_in, w_out, None, None, 0, torch.bfloat16)
    bo.assert_close(out[-5:], want, bound)
    bo.assert_close(pre[-5:], z, z_err)
    values, bounds = bo.ffn_grad(dout[-5:], x[-5:], pre[-5:], w_in, w_out, 0, torch.bfloat16)
    bo.assert_close(dx[-5:], values[0], bounds[0])


# ---- together, on other streams and in graphs


def _block(x, gamma, beta, w_in, w_out, b_in, b_out, dout, p, seed, draw, stream=None):
    """A training step of y = x + dropout(ffn(layer_norm(x)))."""
    kw = dict(stream=stream)
    h, mean, rstd = ann.ann_layer_norm(x, gamma, beta, save=True, **kw)
    f, pre = ann.ann_gated_ffn(h, w_in, w_out, b_in, b_out, save=True, **kw)
    y = ann.ann_dropout(f, p, seed, draw, residual=x, **kw)
    df = ann.ann_dropout(dout, p, seed, draw, **kw)
    dh, dw_in, dw_out, db_in, db_out = ann.ann_gated_ffn_backward(df, h, pre, w_in, w_out, bias=True, **kw)
    dx, dgamma, dbeta = ann.ann_layer_norm_backward(dh, x, gamma, mean, rstd, **kw)
    return y, dx, dgamma, dbeta, dw_in, dw_out, db_in, db_out


def _block_case(M, d, F, dtype, seed):
    gen = _gen(seed)
    x, w_in, w_out, b_in, b_out, dout = _ffn_case(M, d, F, d, dtype, True, seed)
    return x, _randn(gen, d, dtype=dtype, scale=0.1, shift=1), _randn(gen, d, dtype=dtype), w_in, w_out, b_in, b_out, dout


@pytest.mark.parametrize("M,d,F", [(37, 72, 100), (300, 128, 256)])
def test_block_of_a_projector_against_differences(M, d, F):
    """The fp32 gradients of a whole block against central differences of its definition in fp64.  A step of 1e-5 leaves 1e-9
    of the scale; fp32 sums of up to 300 * 256 terms leave less than 1e-4 of the gradient's norm."""
    case = _block_case(M, d, F, torch.float32, 3)
    x, gamma, beta, w_in, w_out, b_in, b_out, dout = case
    y, *grads = _block(*case, 0.3, 17, 5)
    k, scale = bo.kept(np.arange(M * d), 0.3, 17, 5)
    mask = torch.from_numpy(k).cuda().view(M, d) * scale

    def definition(x, gamma, beta, w_in, w_out, b_in, b_out):
        return x + mask * bo.ffn(bo.layer_norm(x, gamma, beta, 1e-5)[0], w_in, w_out, b_in, b_out, 0, torch.float32)[0]

    args = [t.double() for t in case[:-1]]
    want = definition(*args)
    assert float((y.double() - want).norm() / want.norm()) < 1e-5
    order = [0, 1, 2, 3, 4, 5, 6]  # x (without its residual path), gamma, beta, w_in, w_out, b_in, b_out
    gen = _gen(1)
    for i, grad in zip(order, grads):
        v = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        plus, minus = ([a + s * 1e-5 * v if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        numeric = float(((definition(*plus) - definition(*minus)) / 2e-5 * dout.double()).sum())
        mine = float((grad.double() * v).sum()) + (float((dout.double() * v).sum()) if i == 0 else 0.0)
        assert abs(numeric - mine) < 1e-4 * float(grad.double().norm() * v.norm()) + 1e-6, i


def test_block_makes_the_queries_of_a_search():
    """A projector block on the users of a workload, its output the queries of a search: the same ids as from a search on the
    definition's vectors."""
    import oracle
    from gpu_util import open_handles, oracle_mlp, same_list_fraction
    from workloads import PRESETS, make_workload, scaled, to_host

    cfg = scaled(PRESETS["C1"], 4000, n_clusters=8, Q=32)
    wl = make_workload(cfg, seed=5)
    g, m, dev = open_handles(wl)
    h = to_host(wl)
    x = dev["users"]
    d = x.shape[1]
    _, gamma, beta, w_in, w_out, b_in, b_out, _ = _block_case(32, d, 4 * d, torch.float32, 8)
    f = ann.ann_gated_ffn(ann.ann_layer_norm(x, gamma, beta), w_in, w_out, b_in, b_out)
    users = ann.ann_dropout(f, 0.1, 3, residual=x)
    k, scale = bo.kept(np.arange(x.numel()), 0.1, 3, 0)
    ref = bo.ffn(bo.layer_norm(x, gamma, beta, 1e-5)[0], w_in, w_out, b_in, b_out, 0, torch.float32)[0]
    ref = (x.double() + torch.from_numpy(k).cuda().view_as(x) * scale * ref).float()
    assert float((users - ref).abs().max()) < 1e-4 * float(ref.abs().max())
    ids, _ = ann.ann_search(g, m, users, dev["entries"], cfg.W, cfg.L, cfg.k, 0)
    want = oracle.search(h["emb"], h["adj"], ref.cpu().numpy(), oracle_mlp(h), h["entries"], cfg.W, cfg.L, cfg.k, 0, n_threads=8)
    assert same_list_fraction(ids.cpu().numpy(), want["ids"]) >= 0.99


@pytest.mark.parametrize("M", [1, 200])
def test_block_on_another_stream_and_in_two_graphs(M):
    """Eager on the current stream, on a stream of its own, and as two recorded graphs that are replayed in turn and overlap with
    eager work: the same bits every time."""
    one, two = _block_case(M, 136, 264, torch.bfloat16, 1), _block_case(M, 136, 264, torch.bfloat16, 2)
    want = [[t.clone() for t in _block(*c, 0.2, 5, 1)] for c in (one, two)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _block(*one, 0.2, 5, 1, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graphs, outs = [], []
    for c in (one, two):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_block(*c, 0.2, 5, 1))
        graphs.append(g)
    for _ in range(3):
        for i in (0, 1):
            for t in outs[i]:
                t.zero_()
        graphs[0].replay()
        graphs[1].replay()
        eager = _block(*two, 0.2, 5, 1)
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))
        assert all(torch.equal(a, b) for a, b in zip(eager, want[1]))
    # inputs changed between replays are read anew
    one[0].mul_(0.5)
    graphs[0].replay()
    assert all(torch.equal(a, b) for a, b in zip(outs[0], _block(*one, 0.2, 5, 1)))
