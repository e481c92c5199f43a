"""The sequence operators in 64 bits, written from their definitions, and how far a kernel may be
from them.

Error model (u: half a unit in the last place of the tensors' type, 2^-8 bf16, 2^-11 fp16; e32 =
2^-23 for sums and products in fp32): a result is rounded once (u |ref|); operands that a kernel
rounds on the way (p, ds, g) contribute independent errors of at most u of each term, so their sum
is held to 6 u times the root of the sum of the squared terms (the standard deviation is below
u / sqrt 3 of that root: more than ten of them); sums over n terms in fp32 are held to n e32 times
the sum of the terms' magnitudes.  fp16 adds half its smallest subnormal, 2^-25, per rounding."""
import math

import torch

E32 = 2.0 ** -23
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def check(name, got, ref, tol):
    """Every element within its tolerance; NaN and infinity only where the reference has the same."""
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    same = (got == ref) | (got.isnan() & ref.isnan())
    bad = ~same & ~((got - ref).abs() <= tol)
    if bad.any():
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} elements off, first at {i}: "
                             f"{got[i].item()} instead of {ref[i].item()}, allowed {tol[i].item():.3e}")


# ---- attention ---------------------------------------------------------------------------------

def visible(q_len, kv_len, ql, kl, causal):
    i, j = torch.arange(q_len)[:, None], torch.arange(kv_len)[None]
    m = (i < ql) & (j < kl)
    return m & (j <= i + kl - ql) if causal else m


def attention(q, k, v, scale, causal=False, q_lens=None, kv_lens=None, dout=None, dtype=None):
    """[batch, heads, length, dim] tensors; a dict of results and one of tolerances (dtype: the
    type of the kernel's tensors)."""
    u, tiny = U[dtype or q.dtype], TINY[dtype or q.dtype]
    q, k, v = q.double(), k.double(), v.double()
    B, H, Q, D = q.shape
    G, K = k.shape[1:3]
    n = H // G
    res = {"o": torch.zeros(B, H, Q, D, dtype=torch.float64),
           "lse": torch.full((B, H, Q), -math.inf, dtype=torch.float64)}
    if dout is not None:
        dout = dout.double()
        res.update(dq=torch.zeros_like(q), dk=torch.zeros(B, G, K, D, dtype=torch.float64),
                   dv=torch.zeros(B, G, K, D, dtype=torch.float64))
    tol = {name: torch.zeros_like(t) for name, t in res.items()}
    var = {name: torch.zeros_like(t) for name, t in res.items()}
    for b in range(B):
        ql = Q if q_lens is None else int(q_lens[b])
        kl = K if kv_lens is None else int(kv_lens[b])
        if ql == 0 or kl == 0:
            continue
        seen = visible(ql, kl, ql, kl, causal)
        some = seen.any(1)
        for h in range(H):
            g = h // n
            qq, kk, vv = q[b, h, :ql], k[b, g, :kl], v[b, g, :kl]
            s = (qq @ kk.T * scale).masked_fill(~seen, -math.inf)
            top = s.amax(1, keepdim=True).nan_to_num(neginf=0.0, nan=math.nan, posinf=math.inf)
            p = torch.exp(s - top)
            total = p.sum(1, keepdim=True)
            p = torch.where(total == 0, 0.0, p / total)
            o = p @ vv
            res["o"][b, h, :ql] = o
            lse = torch.where(some, top[:, 0] + total[:, 0].log(), -math.inf)
            res["lse"][b, h, :ql] = lse
            # error of a score, then of p relative to p
            es = ((D + 8) * E32 * scale * (qq.abs() @ kk.abs().T).masked_fill(~seen, 0.0).amax(1)
                  + 2 * E32 * top[:, 0].abs() + 8 * E32)[:, None]
            tol["lse"][b, h, :ql] = (es[:, 0] + E32 * lse.abs()).nan_to_num(posinf=0.0)
            tol["o"][b, h, :ql] = 2 * es * (p @ vv.abs()) + kl * E32 * (p @ vv.abs())
            var["o"][b, h, :ql] = u ** 2 * (p ** 2 @ vv ** 2) + tiny ** 2 * (vv ** 2).sum(0)
            if dout is None:
                continue
            do = dout[b, h, :ql]
            dp = do @ vv.T
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            res["dq"][b, h, :ql] = scale * ds @ kk
            res["dk"][b, g, :kl] += scale * ds.T @ qq
            res["dv"][b, g, :kl] += p.T @ do
            e_ds = 2 * es * ds.abs() + p * ((D + 2) * E32 * (do.abs() @ vv.abs().T + (o * do).abs().sum(1, keepdim=True)))
            e_delta = u ** 2 * (o ** 2 * do ** 2).sum(1, keepdim=True)  # o as the forward pass rounded it
            tol["dq"][b, h, :ql] = scale * (e_ds + kl * E32 * ds.abs()) @ kk.abs()
            var["dq"][b, h, :ql] = scale ** 2 * (u ** 2 * ds ** 2 @ kk ** 2 + e_delta * (p @ kk) ** 2)
            tol["dk"][b, g, :kl] += scale * (e_ds + ql * E32 * ds.abs()).T @ qq.abs()
            var["dk"][b, g, :kl] += scale ** 2 * ((u ** 2 * ds ** 2).T @ qq ** 2 + (p ** 2).T @ (e_delta * qq ** 2))
            tol["dv"][b, g, :kl] += (2 * es * p).T @ do.abs() + ql * E32 * (p.T @ do.abs())
            var["dv"][b, g, :kl] += (u ** 2 * (p ** 2).T @ do ** 2) + tiny ** 2 * (do ** 2).sum(0)
    for name in tol:
        if name != "lse":
            tol[name] += 6 * var[name].sqrt() + 1.01 * u * res[name].abs() + tiny
    return res, tol


# ---- linear ------------------------------------------------------------------------------------

def act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z * torch.tanh(torch.log1p(torch.exp(-z.abs())) + z.clamp_min(0))


def act_grad(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    if name == "silu":
        return s * (1 + z * (1 - s))
    t = torch.tanh(torch.log1p(torch.exp(-z.abs())) + z.clamp_min(0))
    return t + z * (1 - t * t) * s


def linear(x, w, bias=None, residual=None, activation="none"):
    u, tiny = U[x.dtype], TINY[x.dtype]
    x, w = x.double(), w.double()
    z = x @ w.T
    size = x.abs() @ w.abs().T
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    ez = (x.shape[1] + 4) * E32 * size
    y = act(activation, z)
    # slopes are below 1.2; the activation's own evaluation costs a few units of |z|
    ey = ez if activation == "none" else 1.2 * ez + 16 * E32 * (z.abs() + y.abs())
    if residual is not None:
        y = y + residual.double()
    return ({"y": y, "z": z},
            {"y": ey + 2 * E32 * y.abs() + 1.01 * u * y.abs() + tiny, "z": ez + 1.01 * u * z.abs() + tiny})


def linear_backward(x, w, dy, z=None, dx_add=None, activation="none", dw_fp32=False):
    u, tiny = U[x.dtype], TINY[x.dtype]
    x, w, dy = x.double(), w.double(), dy.double()
    g = dy
    eg = torch.zeros_like(dy)
    if activation != "none":
        g = dy * act_grad(activation, z.double())
        eg = 32 * E32 * dy.abs() * (1 + z.double().abs().clamp_max(40))
    ug, tg = (u, tiny) if activation != "none" else (0.0, 0.0)  # dy itself is exact
    dx, dw, db = g @ w, g.T @ x, g.sum(0)
    m, n = dy.shape
    e = {"dx": (eg + n * E32 * g.abs()) @ w.abs() + 6 * (ug ** 2 * (g ** 2 @ w ** 2) + tg ** 2 * (w ** 2).sum(0)).sqrt(),
         "dw": (eg + m * E32 * g.abs()).T @ x.abs()
               + 6 * (ug ** 2 * ((g ** 2).T @ x ** 2) + tg ** 2 * (x ** 2).sum(0)).sqrt(),
         "db": (eg + (m + 4) * E32 * g.abs()).sum(0)}
    if dx_add is not None:
        dx = dx + dx_add.double()
    e["dx"] += (1.01 * u + 2 * E32) * dx.abs() + tiny
    if not dw_fp32:
        e["dw"] += 1.01 * u * dw.abs() + tiny
    return {"dx": dx, "dw": dw, "db": db}, e


# ---- layer normalisation -----------------------------------------------------------------------

def layernorm(x, gamma, beta, eps):
    u, tiny = U[x.dtype], TINY[x.dtype]
    x, gamma, beta = x.double(), gamma.double(), beta.double()
    n = x.shape[1]
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    xh = (x - mean) * rstd
    y = gamma * xh + beta
    e_mean = (n + 2) * E32 * x.abs().mean(1, keepdim=True)
    # relative error of rstd: half of the variance's (sums, and the mean's error squared)
    e_rstd = (n + 8) * E32 + (e_mean * rstd) ** 2
    e_xh = e_mean * rstd + xh.abs() * (e_rstd + 4 * E32)
    return ({"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0], "xh": xh},
            {"y": gamma.abs() * e_xh + 4 * E32 * (y.abs() + beta.abs()) + 1.01 * u * y.abs() + tiny,
             "mean": e_mean[:, 0], "rstd": (rstd * e_rstd)[:, 0], "xh": e_xh})


def layernorm_backward(x, dy, gamma, eps, dx_add=None):
    u, tiny = U[x.dtype], TINY[x.dtype]
    f, e = layernorm(x, gamma, torch.zeros_like(gamma), eps)
    xh, exh, rstd = f["xh"], e["xh"], f["rstd"][:, None]
    dy, gamma = dy.double(), gamma.double()
    rows, n = dy.shape
    g = dy * gamma
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    m1, m2 = g.abs().mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
    e2 = (n + 4) * E32 * m2 + (g.abs() * exh).mean(1, keepdim=True)
    edx = rstd * ((n + 4) * E32 * m1 + xh.abs() * e2 + exh * m2 + 4 * E32 * (g.abs() + m1 + xh.abs() * m2)) \
        + (e["rstd"] / f["rstd"])[:, None] * dx.abs()
    if dx_add is not None:
        dx = dx + dx_add.double()
    return ({"dx": dx, "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)},
            {"dx": edx + (1.01 * u + 2 * E32) * dx.abs() + tiny,
             "dgamma": (dy.abs() * (exh + (rows + 4) * E32 * xh.abs())).sum(0),
             "dbeta": (rows + 4) * E32 * dy.abs().sum(0)})
