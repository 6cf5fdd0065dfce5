"""The operators of token models in 64 bits, from their definitions, for the tests: numpy for the generator, torch in float64 for the rest."""
import numpy as np
import torch

U = np.uint64


def kept(rows, cols, p, seed, step):
    """[rows][cols] truth values: Philox4x32 with 7 rounds on (column / 8, row, step), 16 bits a column."""
    groups, low = (cols + 7) // 8, U(0xffffffff)
    c = [np.broadcast_to(np.arange(groups, dtype=U)[None], (rows, groups)), np.broadcast_to(np.arange(rows, dtype=U)[:, None], (rows, groups)),
         np.full((rows, groups), step & 0xffffffff, U), np.full((rows, groups), step >> 32, U)]
    k0, k1 = seed & 0xffffffff, seed >> 32
    for _ in range(7):
        a, b = c[0] * U(0xD2511F53), c[2] * U(0xCD9E8D57)
        c = [(b >> U(32)) ^ c[1] ^ U(k0), b & low, (a >> U(32)) ^ c[3] ^ U(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    d = np.stack([v for w in c for v in (w & U(0xffff), w >> U(16))], -1).reshape(rows, -1)[:, :cols]
    return d >= U(limit(p))


def limit(p):
    return min(65535, int(np.rint(65536.0 * float(np.float32(p)))))


def dropout(x, p, seed, step):
    if x.numel() == 0 or limit(p) == 0:
        return x.double()
    keep = torch.from_numpy(kept(x.shape[0], x.shape[1], p, seed, step)).to(x.device)
    return torch.where(keep, x.double() * (65536.0 / (65536 - limit(p))), 0.0)


def join(y, residual, gain, eps, p=0.0, seed=0, step=0):
    x = dropout(y, p, seed, step) + (0 if residual is None else residual.double())
    rstd = (x.square().mean(1) + eps).rsqrt()
    out = x * rstd[:, None] * (1 if gain is None else gain.double())
    return x, out, rstd


def join_backward(x, rstd, gain, d_out, d_x, p=0.0, seed=0, step=0):
    x, rstd, d_out = x.double(), rstd.double()[:, None], d_out.double()
    xhat = x * rstd
    u = d_out * (1 if gain is None else gain.double())
    d_res = rstd * (u - xhat * (u * xhat).mean(1, keepdim=True)) + (0 if d_x is None else d_x.double())
    return d_res, dropout(d_res, p, seed, step), (d_out * xhat).sum(0)


def vocab(h, w, targets, weights=None):
    """loss, row_loss, lse, dh, dw; tokens without a target never touch their h."""
    there = (targets >= 0).nonzero()[:, 0]
    n, hh, ww = len(there), h.double()[there], w.double()
    z = hh @ ww.T
    top = z.amax(1) if n else z.new_zeros(0)
    lse_k = top + (z - top[:, None]).exp().sum(1).log()
    t = targets[there].long()
    loss_k = lse_k - z[torch.arange(n, device=h.device), t]
    a = weights.double()[there] if weights is not None else torch.full_like(lse_k, 1.0 / max(1, n))
    P = (z - lse_k[:, None]).exp()
    P[torch.arange(n, device=h.device), t] = torch.expm1(-loss_k)
    P = P * a[:, None]
    full = lambda v: torch.zeros((h.shape[0],) + v.shape[1:], dtype=torch.float64, device=h.device).index_copy_(0, there, v)  # noqa: E731
    return (a * loss_k).sum(), full(loss_k), full(lse_k), full(P @ ww), P.T @ hh


def off(a, b):
    """2-norm of the difference over the 2-norm of b; infinite where the finite places differ."""
    a, b = a.double().reshape(-1), b.double().reshape(-1)
    if not torch.equal(a.isfinite(), b.isfinite()) or not torch.equal(a.isnan(), b.isnan()):
        return float("inf")
    a, b = a[b.isfinite()], b[b.isfinite()]
    d, n = float((a - b).norm()), float(b.norm())
    return d / n if n else (0.0 if d == 0 else float("inf"))
