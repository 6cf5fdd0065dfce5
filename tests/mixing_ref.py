"""Rotary positions, linear attention with a decay for each head and the gated join in 64 bits, from their definitions, for the tests."""
import math

import torch


def frequencies(rot, base=10000.0, factor=1.0, context=0, low=1.0, high=32.0):
    out = []
    for i in range(rot // 2):
        theta = base ** (-2.0 * i / rot)
        w = 0.0
        if context:
            w = min(1.0, max(0.0, (context * theta / (2 * math.pi) - low) / (high - low)))
        out.append(theta * (w + (1 - w) / factor))
    return out


def rotary(x, heads, dim, rot, positions, interleaved=False, inverse=False, magnitude=1.0, **scaling):
    """positions: a list of whole numbers, one a row."""
    y = x.double().reshape(x.shape[0], heads, dim).clone()
    theta = torch.tensor(frequencies(rot, **scaling), dtype=torch.float64)
    # the angle within a turn: the product of whole numbers and frequencies, reduced in 64 bits (2^31 * 2^-53 of a radian at most)
    angle = torch.tensor(positions, dtype=torch.float64)[:, None] * theta
    if inverse:
        angle = -angle
    c, s = (f(angle).to(x.device)[:, None] * magnitude for f in (torch.cos, torch.sin))
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = y[..., lo].clone(), y[..., hi].clone()
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    return y.reshape(x.shape[0], heads * dim)


def linear(q, k, v, log_decay, lengths, scale, states=None, slots=None):
    """q [rows][heads][dim_k], k, v [rows][kv_heads][.], states [slots][heads][dim_k][dim_v] -> o (0 behind the last sequence), the states afterwards."""
    heads, share = q.shape[1], q.shape[1] // k.shape[1]
    q, k, v, lam = q.double(), k.double().repeat_interleave(share, 1), v.double().repeat_interleave(share, 1), log_decay.double()
    o = q.new_zeros(q.shape[0], heads, v.shape[2])
    after = None if states is None else states.double().clone()
    begin = 0
    for n, length in enumerate(lengths):
        slot = n if slots is None else slots[n]
        Q, K, V = (t[begin:begin + length].transpose(0, 1) for t in (q, k, v))
        old = q.new_zeros(heads, q.shape[2], v.shape[2]) if states is None or not 0 <= slot < states.shape[0] else states[slot].double()
        t = torch.arange(length, device=q.device, dtype=torch.float64)
        D = decay(lam, t[:, None] - t)
        o[begin:begin + length] = (scale * ((Q @ K.transpose(1, 2) * D) @ V + decay(lam, t + 1)[..., None] * (Q @ old))).transpose(0, 1)
        if after is not None and 0 <= slot < states.shape[0]:
            after[slot] = (K * decay(lam, length - 1 - t)[..., None]).transpose(1, 2) @ V + decay(lam, torch.tensor(float(length), device=q.device).double())[:, None, None] * old
        begin += length
    return o, after


def decay(lam, n):
    """exp(lam)^n of whole n for every head; 0 where n < 0, 1 where n = 0."""
    lam = lam.reshape(-1, *[1] * n.dim())
    return torch.where(n > 0, torch.exp(lam * n.clamp_min(1)), (n == 0).double())


def linear_backward(q, k, v, log_decay, lengths, scale, d_o, states=None, slots=None, d_states=None):
    """Gradients of sum(o d_o) + sum(states afterwards d_states) by q, k, v and the states before, by automatic differentiation."""
    leaves = [t.double().clone().requires_grad_(True) for t in (q, k, v)]
    before = None if states is None else states.double().clone().requires_grad_(True)
    with torch.enable_grad():
        o, after = linear(*leaves, log_decay, lengths, scale, before, slots)
        f = (o * d_o.double()).sum()
        if d_states is not None:
            named = list(range(len(lengths))) if slots is None else [s for s in slots if 0 <= s < states.shape[0]]
            f = f + sum((after[s] * d_states[s].double()).sum() for s in named)
        grads = torch.autograd.grad(f, leaves + ([] if before is None else [before]), allow_unused=True)
    return [torch.zeros_like(l) if g is None else g for l, g in zip(leaves + [before], grads)]


def gate(kind, g):
    return 1.0 if kind == "none" else g if kind in ("column", "plain") else torch.sigmoid(g) if kind == "sigmoid" else g * torch.sigmoid(g)


def gated(y, kind, g, residual, gain_y, gain_x, eps, group, scale, residual_scale):
    """x, out, rstd_y, rstd_x"""
    y = y.double()
    parts = y.reshape(y.shape[0], -1, group or y.shape[1])
    rstd_y = (parts.square().mean(2) + eps).rsqrt()
    u = (parts * rstd_y[..., None]).reshape(y.shape) * (1.0 if gain_y is None else gain_y.double())
    x = scale * gate(kind, None if g is None else g.double()) * u + (0 if residual is None else residual_scale * residual.double())
    rstd_x = (x.square().mean(1) + eps).rsqrt()
    return x, x * rstd_x[:, None] * (1.0 if gain_x is None else gain_x.double()), rstd_y, rstd_x


def gated_backward(y, rstd_y, kind, g, x, rstd_x, gain_y, gain_x, d_out, d_x, group, scale, residual_scale):
    """d_residual, d_y, d_gate, d_gain_y, d_gain_x from the formulas, the statistics as given."""
    y = y.double()
    one = torch.ones(y.shape[1], dtype=torch.float64, device=y.device)
    gain_y, gain_x = (one if t is None else t.double() for t in (gain_y, gain_x))
    t, d_gain_x = 0.0 if d_x is None else d_x.double(), None
    if d_out is not None:
        r = rstd_x.double().reshape(-1, 1)
        xhat, w = x.double() * r, d_out.double() * gain_x
        t = t + r * (w - xhat * (w * xhat).mean(1, keepdim=True))
        d_gain_x = (d_out.double() * xhat).sum(0)
    shape = (y.shape[0], -1, group or y.shape[1])
    ry = rstd_y.double().reshape(y.shape[0], -1, 1)
    yhat = (y.reshape(shape) * ry).reshape(y.shape)
    act, slope = 1.0, 0.0
    if kind != "none":
        leaf = g.double().clone().requires_grad_(True)
        with torch.enable_grad():
            act = gate(kind, leaf)
            slope, = torch.autograd.grad(act.sum(), leaf)
        act = act.detach()
    d_u = scale * act * t
    d_gate = scale * t * yhat * gain_y * slope
    dn = (d_u * gain_y).reshape(shape)
    n = yhat.reshape(shape)
    d_y = (ry * (dn - n * (dn * n).mean(2, keepdim=True))).reshape(y.shape)
    return residual_scale * t, d_y, d_gate.sum(0) if kind == "column" else d_gate, (d_u * yhat).sum(0), d_gain_x
