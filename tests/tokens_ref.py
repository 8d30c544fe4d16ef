"""Operators on token tables from their definitions, in 64 bits, and how far the
kernels may be from them.

A sum of n products of 16-bit values in fp32 is off by at most n 2^-24 times the
sum of the products' magnitudes; a rounding to a type by half a step of it,
finfo(t).eps / 2 relative (and half its smallest subnormal absolute)."""
import torch

U = 2.0 ** -24  # half a step of fp32


def half(dt):
    return torch.finfo(dt).eps / 2


def scores(X, W, scale, bias):
    z = torch.matmul(X.double(), W.double().transpose(1, 2).contiguous()) * scale
    if bias is not None:  # a forbidden token, whatever its row holds
        b = bias.double().unsqueeze(1)
        z = torch.where(b == float("-inf"), b, z + b)
    return z


def score_bound(X, W, scale, bias):
    """Largest error of a score of each row, [B, M, 1]: the sum, the product with
    scale, the sum with bias (finite entries)."""
    D = X.shape[2]
    X, W = torch.nan_to_num(X.double(), 0, 0, 0), torch.nan_to_num(W.double(), 0, 0, 0)
    mag = torch.matmul(X.abs(), W.abs().transpose(1, 2).contiguous()) * abs(scale)
    e = (D + 1) * U * mag
    if bias is not None:
        b = bias.double().unsqueeze(1)
        e = torch.where(b == float("-inf"), 0.0, e + U * (mag + b.abs()))
    return e.amax(-1, keepdim=True)


def logprobs(X, W, target, scale=1.0, bias=None, k=0):
    z = scores(X, W, scale, bias)
    V = W.shape[1]
    lse = torch.logsumexp(z, -1, keepdim=True)
    none = (lse == float("-inf")).squeeze(-1)
    logp = z - lse
    p = torch.exp(logp)
    ent = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    ent = torch.where(none, 0.0, ent)
    has = (target >= 0) & (target < V)
    zt = torch.gather(z, 2, torch.where(has, target, 0).long().unsqueeze(-1)).squeeze(-1)
    lp = torch.where(has, torch.where(none, float("-inf"), zt - lse.squeeze(-1)), 0.0)
    out = [lp, ent, lse.squeeze(-1)]
    if k:
        # ties to the lowest index: a stable sort, descending
        v, i = torch.sort(z, dim=-1, descending=True, stable=True)
        v, i = v[..., :k], i[..., :k]
        gone = v == float("-inf")
        out += [torch.where(gone, -1, i).int(), torch.where(gone, float("-inf"), v - lse)]
    return out


def logprob_bound(X, W, scale, bias):
    """Of logprob, lse and top_logprob, [B, M]: a score's error twice; the roundings of
    z - m, of the logarithm and of the results; the exponentials' (a step each, times
    at most 2^6 roundings of a tree of sums and V / 256 of a running one)."""
    z = scores(X, W, scale, bias)
    V = W.shape[1]
    size = torch.where(z.isfinite() & (z.abs() < 1e30), z.abs(), 0.0).amax(-1)
    return 2 * score_bound(X, W, scale, bias).squeeze(-1) + 8 * U * (size + 16) + (96 + V / 256) * 2 * U


def grads(X, W, target, g, h=None, scale=1.0, bias=None):
    """dX, dW, and for each the bound of the error of 16-bit dz and outputs."""
    dt = X.dtype
    z = scores(X, W, scale, bias)
    V = W.shape[1]
    lse = torch.logsumexp(z, -1, keepdim=True)
    none = lse == float("-inf")
    logp = torch.where(none, float("-inf"), z - lse)
    p = torch.exp(logp)
    plogp = torch.where(p > 0, p * logp, 0.0)
    ent = -plogp.sum(-1, keepdim=True)
    has = (target >= 0) & (target < V)
    at = torch.where(has, target, 0).long().unsqueeze(-1)
    has = has & (torch.gather(z, 2, at).squeeze(-1) != float("-inf"))
    g = torch.where(has, g.double(), 0.0).unsqueeze(-1)
    h = torch.zeros_like(g) if h is None else h.double().unsqueeze(-1)
    active = ((g != 0) | (h != 0)) & ~none
    g, h = torch.where(active, g, 0.0), torch.where(active, h, 0.0)
    hot = torch.zeros_like(z).scatter_(2, at, 1.0)
    dz = g * (hot - p) - h * (plogp + p * ent)
    keep = active.expand_as(z)
    if bias is not None:
        keep = keep & (bias.unsqueeze(1) != float("-inf"))
    dz = torch.where(keep, dz, 0.0)
    # dz: p is off by the scores' and lse's errors, then the rounding to 16 bits
    dp = 4 * score_bound(X, W, scale, bias) + (128 + V / 256) * 4 * U
    mag = (g.abs() + h.abs() * (1 + logp.clamp(min=-100).abs() + ent)) * p
    e = torch.where(keep, dp * (mag + h.abs() * p) + half(dt) * (dz.abs() + dp * mag), 0.0)
    gs = torch.where(active, torch.maximum(g.abs(), h.abs()), 0.0) * 2
    # dz is stored in fp16 for either type, over gs and 2048 times larger: half its smallest step
    e = torch.where(keep, e + gs * 2.0 ** -25 / 2048, 0.0)
    Xd = torch.where(active, X.double(), 0.0)
    Wd = W.double()
    if bias is not None:
        Wd = torch.where((bias != float("-inf")).unsqueeze(-1), Wd, 0.0)
    dX = torch.matmul(dz, Wd) * scale
    dzt, et = dz.transpose(1, 2).contiguous(), e.transpose(1, 2).contiguous()
    dW = torch.matmul(dzt, Xd) * scale
    eX = torch.matmul(e + V * U * (dz.abs() + e), Wd.abs()) * abs(scale)
    eW = torch.matmul(et + X.shape[1] * U * (dzt.abs() + et), Xd.abs()) * abs(scale)
    if dt == torch.float16:
        top = gs.amax(1, keepdim=True)
        per = torch.where(gs > 0, dz.abs() / gs.clamp(min=1e-300), 0.0).sum(1).unsqueeze(-1)
        eW = eW + abs(scale) * per * top * 2.0 ** -25
        # X times a row's factor, no power of two, is rounded too: half a step of each product
        eW = eW + half(dt) * torch.matmul(dzt.abs() + et, Xd.abs()) * abs(scale)
    tiny = torch.finfo(dt).smallest_normal * half(dt) * 2
    eX = eX + half(dt) * (dX.abs() + eX) + tiny
    eW = eW + half(dt) * (dW.abs() + eW) + tiny
    return dX, dW, eX, eW


def embed(W, idx, scale):
    B, V, D = W.shape
    has = (idx >= 0) & (idx < V)
    at = torch.where(has, idx, 0).long().unsqueeze(-1).expand(-1, -1, D)
    f = torch.tensor(scale, dtype=torch.float32).item()
    rows = (torch.gather(W, 1, at).float() * f).to(W.dtype)  # one fp32 product, one rounding
    return torch.where(has.unsqueeze(-1), rows, torch.zeros((), dtype=W.dtype, device=W.device))


def embed_grad(G, idx, V, scale, into=None, dt=None):
    """The gradient in 64 bits and the bound of its error."""
    B, M, D = G.shape
    dt = dt or G.dtype
    f = torch.tensor(scale, dtype=torch.float32).item()
    has = ((idx >= 0) & (idx < V)).unsqueeze(-1)
    g = torch.where(has, G.double(), 0.0)
    at = torch.where(has.squeeze(-1), idx, 0).long().unsqueeze(-1).expand(-1, -1, D)
    s = torch.zeros((B, V, D), dtype=torch.float64, device=G.device)
    total, mag = s.scatter_add(1, at, g) * f, s.scatter_add(1, at, g.abs()) * abs(f)
    n = torch.zeros((B, V, 1), dtype=torch.float64, device=G.device).scatter_add(
        1, at[..., :1], has.double())
    err = (n + 1) * U * mag
    if into is not None:
        total = total + into.double()
        err = err + U * total.abs()
    return total, err + half(dt) * (total.abs() + err) + torch.finfo(dt).smallest_normal * half(dt)
