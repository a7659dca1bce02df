"""The operators of a projector block from their definitions, in fp64, with bounds on what the kernels may differ by.

The bounds count roundings: u = 2^-24 for every fp32 operation on the way (sums of n terms: n u times the sum of the
terms' magnitudes), half a step of the 16-bit type (eps / 2, and half the smallest subnormal) for every rounding to it, and
2^-18 (times max(1, |z|)) for the activation and its slope, whose exponential has a relative error of |z| u."""
import numpy as np
import torch

U = 2.0 ** -24
ACT_ERR = 2.0 ** -18


def half_step(t, dtype):
    """Largest error of rounding values of magnitude |t| to dtype."""
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    return t.abs() * (torch.finfo(dtype).eps / 2) + tiny / 2


def philox_words(blocks, c2, c3, k0, k1):
    """Philox4x32-10 of counters (block low, block high, c2, c3), as [blocks][4] uint64 arrays of 32-bit words."""
    blocks = np.asarray(blocks, dtype=np.uint64)
    m = np.uint64(0xFFFFFFFF)
    x = [blocks & m, blocks >> np.uint64(32), np.full_like(blocks, c2), np.full_like(blocks, c3)]
    for r in range(10):
        p0, p1 = np.uint64(0xD2511F53) * x[0], np.uint64(0xCD9E8D57) * x[2]
        a, b = np.uint64((k0 + r * 0x9E3779B9) & 0xFFFFFFFF), np.uint64((k1 + r * 0xBB67AE85) & 0xFFFFFFFF)
        x = [(p1 >> np.uint64(32)) ^ x[1] ^ a, p1 & m, (p0 >> np.uint64(32)) ^ x[3] ^ b, p0 & m]
    return np.stack(x, 1)


def kept(elements, p, seed, draw):
    """(truth values, scale) of dropout at these element numbers."""
    elements = np.asarray(elements, dtype=np.uint64)
    w = philox_words(elements // np.uint64(8), draw & 0xFFFFFFFF, draw >> 32, seed & 0xFFFFFFFF, (seed >> 32) ^ 0x64726F70)
    j = (elements % np.uint64(8)).astype(np.int64)
    half = (w[np.arange(len(j)), j // 2] >> (np.uint64(16) * (j % 2).astype(np.uint64))) & np.uint64(0xFFFF)
    t = int(np.floor(p * 65536 + 0.5))
    return half >= t, (65536 / (65536 - t) if t < 65536 else 0.0)


def layer_norm(x, gamma, beta, eps):
    """(out, mean, rstd, bound of out before its rounding)."""
    x, d = x.double(), x.shape[-1]
    g = torch.ones(d, dtype=x.dtype, device=x.device) if gamma is None else gamma.double()
    b = torch.zeros(d, dtype=x.dtype, device=x.device) if beta is None else beta.double()
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    xh = (x - mean) * rstd
    # a thread adds at most d / 1024 + 32 terms, then 10 levels of a tree: n roundings of at most the row's largest magnitude
    n = d / 1024 + 48
    worst = x.abs().amax(-1, keepdim=True) * rstd
    bound = n * U * (g.abs() * (worst * (1 + 2 * xh.abs()) + 4 * xh.abs()) + 2 * b.abs())
    return xh * g + b, mean[..., 0], rstd[..., 0], bound


def layer_norm_grad(dout, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) and their bounds, for the statistics given."""
    x, dy, m, r = x.double(), dout.double(), mean.double()[:, None], rstd.double()[:, None]
    d, M = x.shape[-1], x.shape[0]
    g = torch.ones(d, dtype=x.dtype, device=x.device) if gamma is None else gamma.double()
    xh, q = (x - m) * r, dy * g
    dx = r * (q - q.mean(-1, keepdim=True) - xh * (q * xh).mean(-1, keepdim=True))
    n = d / 1024 + 48
    off = (x.abs() + m.abs()) * r  # the magnitudes that x - mean was formed of
    bound = n * U * r * (q.abs() + q.abs().mean(-1, keepdim=True) + off * (q * xh).abs().mean(-1, keepdim=True)
                         + (xh.abs() + 1) * (q.abs() * off).mean(-1, keepdim=True))
    k = (M + 16) * U
    return (dx, (dy * xh).sum(0), dy.sum(0)), (bound, k * (dy.abs() * (off + xh.abs())).sum(0), k * dy.abs().sum(0))


def act_of(act, z):
    """(value, slope): 0 = SiLU, 1 = GELU, 2 = sigmoid, 3 = ReLU."""
    if act == 3:
        return z.clamp_min(0), (z > 0).to(z.dtype)
    if act == 1:
        cdf = 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (2 * np.pi) ** -0.5
    s, c = torch.sigmoid(z), torch.sigmoid(-z)
    return (z * s, s * (1 + z * c)) if act == 0 else (s, s * c)


def ffn(x, w_in, w_out, b_in, b_out, act, dtype):
    """out, pre and their bounds (out's before its rounding)."""
    x, wi, wo = x.double(), w_in.double(), w_out.double()
    F, D = wo.shape[1], wi.shape[1]
    z, z_mag = x @ wi.t(), x.abs() @ wi.abs().t()
    if b_in is not None:
        z, z_mag = z + b_in.double(), z_mag + b_in.double().abs()
    z_err = (D + 20) * U * z_mag
    g, u = z[:, :F], z[:, F:]
    a, _ = act_of(act, g)
    h = a * u
    h_err = (u.abs() * (1.2 * z_err[:, :F] + ACT_ERR * g.abs().clamp_min(1)) + a.abs() * z_err[:, F:]
             + z_err[:, :F] * z_err[:, F:] * 1.2)
    if dtype != torch.float32:
        h_err = h_err + half_step(h.abs() + h_err, dtype)
    out = h @ wo.t()
    bound = h_err @ wo.abs().t() + (F + 20) * U * ((h.abs() + h_err) @ wo.abs().t())
    if b_out is not None:
        out = out + b_out.double()
        bound = bound + 2 * U * b_out.double().abs()
    return out, z, bound + 2 * U * out.abs(), z_err


def ffn_grad(dout, x, pre, w_in, w_out, act, dtype):
    """dx, dw_in, dw_out, db_in, db_out and their bounds before their rounding, for the gate and up values given."""
    dy, x, z, wi, wo = dout.double(), x.double(), pre.double(), w_in.double(), w_out.double()
    F, O, M = wo.shape[1], wo.shape[0], x.shape[0]
    g, u = z[:, :F], z[:, F:]
    a, da = act_of(act, g)
    zs = g.abs().clamp_min(1)
    dh, dh_err = dy @ wo, (O + 20) * U * (dy.abs() @ wo.abs())
    h, dz = a * u, torch.cat((dh * u * da, dh * a), 1)
    h_err = u.abs() * ACT_ERR * zs + 4 * U * h.abs()
    dz_err = torch.cat(((dh_err * da.abs() + (dh.abs() + dh_err) * ACT_ERR * zs) * u.abs(),
                        dh_err * a.abs() + (dh.abs() + dh_err) * ACT_ERR * zs), 1) + 4 * U * dz.abs()
    if dtype != torch.float32:
        h_err = h_err + half_step(h.abs() + h_err, dtype)
        dz_err = dz_err + half_step(dz.abs() + dz_err, dtype)
    dzm, hm = dz.abs() + dz_err, h.abs() + h_err
    k = (M + 20) * U
    values = (dz @ wi, dz.t() @ x, dy.t() @ h, dz.sum(0), dy.sum(0))
    bounds = (dz_err @ wi.abs() + (2 * F + 20) * U * (dzm @ wi.abs()), dz_err.t() @ x.abs() + k * (dzm.t() @ x.abs()),
              dy.abs().t() @ h_err + k * (dy.abs().t() @ hm), dz_err.sum(0) + k * dzm.sum(0), k * dy.abs().sum(0))
    return values, bounds


def assert_close(got, want, bound, what=""):
    """got is want within `bound`, rounded to got's type."""
    limit = bound + half_step(want.abs() + bound, got.dtype)
    err = (got.double() - want).abs()
    bad = ~(err <= limit)
    if bool(bad.any()):
        i = int((err - limit).nan_to_num(float("inf")).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, worst at {i}: got {float(got.flatten()[i])}, "
                             f"want {float(want.flatten()[i])} +- {float(limit.flatten()[i])}")
