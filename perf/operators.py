"""The operators of a projector block, as cases that can be timed and compared.

A projector (the network that makes the user and item vectors a search works on) is built of residual blocks
y = x + dropout(ffn(layer_norm(x))).  A case is one operator of such a block on one size and type:

    ln           layer norm of rows, as in serving
    ln_grad      layer norm and its gradient, as in a training step
    drop         dropout added to the residual, as in the forward pass
    drop_grad    the same and the gradient through it
    ffn          gated feed-forward block without a gradient: one request, a small batch, a table of items
    ffn_grad     the block and all its gradients

`run` computes the operators by elementary torch operations in fp32, or, with `own`, by the library's entry points.
`exact` computes them from their definitions in fp64.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ACTS = ("silu", "gelu", "sigmoid", "relu")
M32 = 0xFFFFFFFF
EPS = 1e-5


def _ln(name, op, dtype, rows, d):
    return dict(name=name, op=op, dtype=dtype, rows=rows, d=d)


def _drop(name, op, dtype, rows, d, p):
    return dict(name=name, op=op, dtype=dtype, rows=rows, d=d, p=p)


def _ffn(name, op, dtype, rows, d, hidden, d_out, act, bias):
    return dict(name=name, op=op, dtype=dtype, rows=rows, d=d, hidden=hidden, d_out=d_out, act=act, bias=bias)


def listed():
    return [
        # the smallest batch of users the repository searches for, reference precision: latency
        _ln("ln_users_f32", "ln", "f32", 64, 32),
        # a batch of the training of a narrow tower whose width is no power of two
        _ln("ln_train_f16", "ln_grad", "f16", 10007, 1000),
        # a training step's rows through a wide tower: bound by memory
        _ln("ln_train_bf16", "ln_grad", "bf16", 16384, 4096),
        # dropout on the user vectors of one batch: latency
        _drop("drop_users_bf16", "drop", "bf16", 1024, 64, 0.1),
        # sizes that divide by nothing, both directions
        _drop("drop_odd_f32", "drop_grad", "f32", 3001, 1009, 0.25),
        # a training step's rows through a wide tower: bound by memory, then by the generator
        _drop("drop_train_bf16", "drop_grad", "bf16", 32768, 4096, 0.1),
        # one request through a wide block: bound by reading the weights
        _ffn("ffn_one_bf16", "ffn", "bf16", 1, 2048, 8192, 2048, "silu", False),
        # a handful of requests that arrived together
        _ffn("ffn_few_f16", "ffn", "f16", 37, 1024, 4096, 1024, "gelu", True),
        # the users of the headline batch through the last block, which ends in item vectors of 128
        _ffn("ffn_users_bf16", "ffn", "bf16", 4096, 512, 2048, 128, "silu", True),
        # a training step of a wide block: bound by the matrix cores
        _ffn("ffn_train_bf16", "ffn_grad", "bf16", 8192, 2048, 8192, 2048, "silu", False),
        # a ragged batch through widths that divide by nothing
        _ffn("ffn_odd_f16", "ffn_grad", "f16", 1537, 1003, 2731, 777, "gelu", True),
        # the same training in reference precision
        _ffn("ffn_train_f32", "ffn_grad", "f32", 2048, 512, 1300, 256, "relu", True),
    ]


def _between(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("ln", "ln_grad", "drop", "drop_grad", "ffn", "ffn", "ffn_grad", "ffn_grad"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16", "f16"))
    if op.startswith("ffn"):
        if dtype == "f32":
            c = _ffn("", op, dtype, _between(rng, 1, 4096), _between(rng, 32, 1024), _between(rng, 64, 2048),
                     _between(rng, 32, 1024), rng.choice(ACTS), rng.random() < 0.5)
        else:
            c = _ffn("", op, dtype, _between(rng, 1, 8192), _between(rng, 32, 4096), _between(rng, 64, 8192),
                     _between(rng, 32, 2048), rng.choice(ACTS), rng.random() < 0.5)
        for key in ("rows", "d", "hidden", "d_out"):
            if rng.random() < 0.5:  # half of the sizes are the round ones that towers mostly have
                c[key] = max(1, c[key] // 64 * 64)
        most = work(next(x for x in listed() if x["name"] == ("ffn_train_f32" if dtype == "f32" else "ffn_train_bf16")))
        while work(c)["flops"] > most["flops"]:
            c["rows"] = max(1, c["rows"] // 2)
    else:
        d = _between(rng, 16, 16384)
        rows = _between(rng, 1, max(1, (1 << 26) // d))
        if rng.random() < 0.5:
            d = d // 16 * 16
        c = _drop("", op, dtype, rows, d, rng.choice((0.0, 0.05, 0.1, 0.5, 0.9))) if op.startswith("drop") else _ln("", op, dtype, rows, d)
    del c["name"]
    return c


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, shift=0.0):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(scale).add_(shift).to(t)

    rows, d, op = case["rows"], case["d"], case["op"]
    s = dict(op=op)
    if op.startswith("ln"):
        # rows of a residual stream: their own offsets and scales
        x = torch.randn(rows, d, generator=gen, device="cuda")
        x.mul_(torch.rand(rows, 1, generator=gen, device="cuda") * 2 + 0.25).add_(torch.randn(rows, 1, generator=gen, device="cuda"))
        s.update(x=x.to(t), gamma=normal(d, scale=0.1, shift=1.0), beta=normal(d, scale=0.1))
    elif op.startswith("drop"):
        s.update(x=normal(rows, d), residual=normal(rows, d), p=case["p"], seed=(seed * 0x9E3779B97F4A7C15 + 12345) & (2 ** 64 - 1),
                 draw=seed % 1000)
    else:
        hidden, d_out = case["hidden"], case["d_out"]
        s.update(x=normal(rows, d), w_in=normal(2 * hidden, d, scale=d ** -0.5), w_out=normal(d_out, hidden, scale=hidden ** -0.5),
                 act=case["act"], b_in=None, b_out=None)
        if case["bias"]:
            s.update(b_in=normal(2 * hidden, scale=0.1), b_out=normal(d_out, scale=0.1))
    if op.endswith("_grad"):
        s["dout"] = normal(rows, case.get("d_out", d))
    return s


# ---- plain forms: elementary operations in fp32, rounded once at the end


def _plain_ln(s):
    x, gamma, beta = s["x"].float(), s["gamma"].float(), s["beta"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    xh = c * rstd
    out = {"out": (xh * gamma + beta).to(s["x"].dtype)}
    if "dout" in s:
        dy = s["dout"].float()
        g = dy * gamma
        dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * rstd
        out.update(dx=dx.to(s["x"].dtype), dgamma=(dy * xh).sum(0).to(s["x"].dtype), dbeta=dy.sum(0).to(s["x"].dtype))
    return out


def _kept(n, seed, draw, threshold, device):
    """Truth values [n]: the half-word of each element is at least the threshold."""
    block = torch.arange((n + 7) // 8, device=device)
    c0, c1 = block & M32, block >> 32
    c2, c3 = torch.full_like(block, draw & M32), torch.full_like(block, draw >> 32)
    k0, k1 = seed & M32, (seed >> 32) ^ 0x64726F70
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # the low 64 bits; the shifts below are masked
        c0, c1, c2, c3 = ((b >> 32) & M32) ^ c1 ^ k0, b & M32, ((a >> 32) & M32) ^ c3 ^ k1, a & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    words = torch.stack((c0, c1, c2, c3), 1)
    return (torch.stack((words & 0xFFFF, words >> 16), 2) >= threshold).reshape(-1)[:n]


def _plain_drop(s):
    x = s["x"]
    threshold = int(s["p"] * 65536 + 0.5)
    kept = _kept(x.numel(), s["seed"], s["draw"], threshold, x.device).view_as(x)
    scale = 65536.0 / (65536 - threshold)
    out = {"out": (s["residual"].float() + torch.where(kept, x.float() * scale, 0.0)).to(x.dtype)}
    if "dout" in s:
        out["dx"] = torch.where(kept, s["dout"].float() * scale, 0.0).to(x.dtype)
    return out


def _plain_act(name, z):
    """The activation and its derivative."""
    if name == "relu":
        return z.clamp_min(0.0), (z > 0).float()
    if name == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    if name == "silu":
        return z * sig, sig * (1.0 + z * (1.0 - sig))
    return sig, sig * (1.0 - sig)


def _plain_ffn(s):
    t = s["x"].dtype
    x, w_in, w_out = s["x"].float(), s["w_in"].float(), s["w_out"].float()
    hidden = w_out.shape[1]
    z = x @ w_in.t()
    if s["b_in"] is not None:
        z = z + s["b_in"].float()
    gate, up = z[:, :hidden], z[:, hidden:]
    a, slope = _plain_act(s["act"], gate)
    h = a * up
    y = h @ w_out.t()
    if s["b_out"] is not None:
        y = y + s["b_out"].float()
    out = {"out": y.to(t)}
    if "dout" in s:
        dy = s["dout"].float()
        dh = dy @ w_out
        dz = torch.cat((dh * up * slope, dh * a), 1)
        out.update(dx=(dz @ w_in).to(t), dw_in=(dz.t() @ x).to(t), dw_out=(dy.t() @ h).to(t))
        if s["b_in"] is not None:
            out.update(db_in=dz.sum(0).to(t), db_out=dy.sum(0).to(t))
    return out


# ---- the library's entry points


def _own(s):
    import paper_2502_11490_amd as ann

    op = s["op"]
    if op == "ln":
        return {"out": ann.ann_layer_norm(s["x"], s["gamma"], s["beta"], EPS)}
    if op == "ln_grad":
        y, mean, rstd = ann.ann_layer_norm(s["x"], s["gamma"], s["beta"], EPS, save=True)
        dx, dgamma, dbeta = ann.ann_layer_norm_backward(s["dout"], s["x"], s["gamma"], mean, rstd)
        return {"out": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if op.startswith("drop"):
        out = {"out": ann.ann_dropout(s["x"], s["p"], s["seed"], s["draw"], residual=s["residual"])}
        if op == "drop_grad":
            out["dx"] = ann.ann_dropout(s["dout"], s["p"], s["seed"], s["draw"])
        return out
    act = {"silu": ann.ANN_SILU, "gelu": ann.ANN_GELU, "sigmoid": ann.ANN_SIGMOID, "relu": ann.ANN_RELU}[s["act"]]
    if op == "ffn":
        return {"out": ann.ann_gated_ffn(s["x"], s["w_in"], s["w_out"], s["b_in"], s["b_out"], act)}
    y, pre = ann.ann_gated_ffn(s["x"], s["w_in"], s["w_out"], s["b_in"], s["b_out"], act, save=True)
    dx, dw_in, dw_out, db_in, db_out = ann.ann_gated_ffn_backward(s["dout"], s["x"], pre, s["w_in"], s["w_out"], act,
                                                                  bias=s["b_in"] is not None)
    out = {"out": y, "dx": dx, "dw_in": dw_in, "dw_out": dw_out}
    if s["b_in"] is not None:
        out.update(db_in=db_in, db_out=db_out)
    return out


def run(state):
    if own:
        return _own(state)
    op = state["op"]
    return _plain_ln(state) if op.startswith("ln") else _plain_drop(state) if op.startswith("drop") else _plain_ffn(state)


def work(case):
    e, rows, d, op = SIZE[case["dtype"]], case["rows"], case["d"], case["op"]
    n = rows * d
    if op == "ln":
        return {"bytes": e * (2 * n + 2 * d), "flops": 8 * n}
    if op == "ln_grad":  # x and dout in; out, dx and the two parameters' gradients back
        return {"bytes": e * (4 * n + 4 * d), "flops": 22 * n}
    if op == "drop":
        return {"bytes": e * 3 * n, "flops": 2 * n}
    if op == "drop_grad":
        return {"bytes": e * 5 * n, "flops": 3 * n}
    hidden, d_out = case["hidden"], case["d_out"]
    weights = 2 * hidden * d + d_out * hidden + (2 * hidden + d_out if case["bias"] else 0)
    flops = 2 * rows * hidden * (2 * d + d_out)
    if op == "ffn":
        return {"bytes": e * (weights + n + rows * d_out), "flops": flops}
    return {"bytes": e * (2 * weights + 2 * n + 2 * rows * d_out), "flops": 3 * flops}


# ---- the definitions in fp64


def _words64(n, seed, draw, device):
    """The generator's half-words of n elements, its 32 x 32 bit products formed from 16-bit halves."""
    def product(a, m):
        al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
        low, mid1, mid2 = al * ml, ah * ml, al * mh
        mid = (low >> 16) + (mid1 & 0xFFFF) + (mid2 & 0xFFFF)
        return ah * mh + (mid1 >> 16) + (mid2 >> 16) + (mid >> 16), ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    i = torch.arange(-(-n // 8), device=device, dtype=torch.int64)
    ctr = [i % 2 ** 32, i // 2 ** 32, torch.zeros_like(i) + draw % 2 ** 32, torch.zeros_like(i) + draw // 2 ** 32]
    key = [seed % 2 ** 32, (seed // 2 ** 32) ^ 0x64726F70]
    for r in range(10):
        h0, l0 = product(ctr[0], 0xD2511F53)
        h1, l1 = product(ctr[2], 0xCD9E8D57)
        ctr = [h1 ^ ctr[1] ^ ((key[0] + r * 0x9E3779B9) % 2 ** 32), l1, h0 ^ ctr[3] ^ ((key[1] + r * 0xBB67AE85) % 2 ** 32), l0]
    halves = torch.empty(i.numel(), 8, dtype=torch.int32, device=device)
    for j in range(8):
        halves[:, j] = ((ctr[j // 2] >> (16 * (j % 2))) % 65536).int()
    return halves.flatten()[:n]


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    grad = op.endswith("_grad")
    x = s["x"].double()
    if op.startswith("ln"):
        gamma, beta, n = s["gamma"].double(), s["beta"].double(), x.shape[1]
        mu = x.sum(1) / n
        sd = ((x - mu[:, None]).square().sum(1) / n + EPS).sqrt()
        z = (x - mu[:, None]) / sd[:, None]
        out = {"out": beta + gamma * z}
        if grad:
            dy = s["dout"].double()
            q = dy * gamma
            out["dx"] = (q - (q.sum(1) / n)[:, None] - z * ((q * z).sum(1) / n)[:, None]) / sd[:, None]
            out["dgamma"], out["dbeta"] = (dy * z).sum(0), dy.sum(0)
        return out
    if op.startswith("drop"):
        t = math.floor(s["p"] * 65536 + 0.5)
        factor = (_words64(x.numel(), s["seed"], s["draw"], x.device) >= t).double().view_as(x) * (65536 / (65536 - t))
        out = {"out": s["residual"].double() + factor * x}
        if grad:
            out["dx"] = factor * s["dout"].double()
        return out
    w_in, w_out = s["w_in"].double(), s["w_out"].double()
    hidden = w_out.shape[1]
    zero = torch.zeros((), dtype=torch.float64, device=x.device)
    b_in, b_out = (s["b_in"].double(), s["b_out"].double()) if case["bias"] else (zero.expand(2 * hidden), zero)
    g = torch.matmul(x, w_in[:hidden].t()) + b_in[:hidden]
    u = torch.matmul(x, w_in[hidden:].t()) + b_in[hidden:]
    phi = 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
    a = {"silu": lambda: g * torch.sigmoid(g), "gelu": lambda: g * phi, "sigmoid": lambda: torch.sigmoid(g),
         "relu": lambda: torch.maximum(g, zero)}[case["act"]]()
    h = a * u
    out = {"out": torch.matmul(h, w_out.t()) + b_out}
    if grad:
        sg = torch.sigmoid(g)
        da = {"silu": lambda: sg + g * sg * torch.sigmoid(-g),
              "gelu": lambda: phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi),
              "sigmoid": lambda: sg * torch.sigmoid(-g), "relu": lambda: (g > 0).double()}[case["act"]]()
        dy = s["dout"].double()
        dh = torch.matmul(dy, w_out)
        dg, du = dh * u * da, dh * a
        out["dx"] = torch.matmul(dg, w_in[:hidden]) + torch.matmul(du, w_in[hidden:])
        out["dw_in"] = torch.cat((torch.matmul(dg.t(), x), torch.matmul(du.t(), x)), 0)
        out["dw_out"] = torch.matmul(dy.t(), h)
        if case["bias"]:
            out["db_in"], out["db_out"] = torch.cat((dg.sum(0), du.sum(0))), dy.sum(0)
    return out
