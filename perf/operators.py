"""The operators of token models that are timed for this library, each through the public binding: dropout from a
counter-based generator, the join of a residual branch with its root-mean-square norm (forward, backward, and with an 8-bit
output), and the softmax cross entropy over a vocabulary with its gradients.

Sizes are generic: rows are tokens in a minibatch (one token when an answer is produced a token at a time), columns the width of
a module, and the vocabulary that of a token model or, at the small end, the classes of the repository's own heads.
"""
import functools

import numpy as np
import torch

own = False


DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LARGEST = 8192 * 4096 * 131072          # tokens x width x vocabulary of the largest case
E4M3_MAX = 448.0
EPS = 1e-6


# ---- cases --------------------------------------------------------------------------------------

def listed():
    return [
        # classifier features of the repository's ResNets (a minibatch of 128, 64 channels), half of them dropped
        dict(name="dropout_f32_128x64", op="dropout", dtype="f32", rows=128, cols=64, p=0.5, pad=0),
        # the activations of a training minibatch: 8192 tokens of width 4096
        dict(name="dropout_bf16_8192x4096", op="dropout", dtype="bf16", rows=8192, cols=4096, p=0.1, pad=0),
        # one token being answered: latency of a single row
        dict(name="join_bf16_1x2048", op="join", mode="fwd", dtype="bf16", rows=1, cols=2048, p=0.0, pad=0),
        # training forward of a minibatch, with dropout
        dict(name="join_bf16_8192x2048", op="join", mode="fwd", dtype="bf16", rows=8192, cols=2048, p=0.1, pad=0),
        # the backward pass of the same join
        dict(name="join_bwd_bf16_8192x2048", op="join", mode="bwd", dtype="bf16", rows=8192, cols=2048, p=0.1, pad=0),
        # full precision at an odd width inside a wider tensor: nothing is aligned
        dict(name="join_bwd_f32_777x1001", op="join", mode="bwd", dtype="f32", rows=777, cols=1001, p=0.2, pad=3),
        # a prompt on its way to 8-bit products, a scale per 128 columns
        dict(name="join_q8_bf16_2048x4096", op="join", mode="q8", dtype="bf16", rows=2048, cols=4096, p=0.0, pad=0, group=128),
        # the loss of one token (scoring), nothing but the pass over the vocabulary's rows
        dict(name="vocab_bf16_t1_loss", op="vocab", dtype="bf16", tokens=1, dim=1024, vocab=32000, grads=False,
             ignored=0.0, weighted=False, pad=0),
        # the repository's own classifier head as a vocabulary: 100 classes, 64 channels, a minibatch of 256
        dict(name="vocab_f32_t256_v100", op="vocab", dtype="f32", tokens=256, dim=64, vocab=100, grads=True,
             ignored=0.0, weighted=False, pad=0),
        # a small training minibatch against a large vocabulary: weight rows are read and their gradients written
        dict(name="vocab_bf16_t64_v65536", op="vocab", dtype="bf16", tokens=64, dim=2048, vocab=65536, grads=True,
             ignored=0.0, weighted=False, pad=0),
        # a ragged minibatch, part of it without targets, sequences weighted; no size fills a tile
        dict(name="vocab_bf16_t1021_v10007", op="vocab", dtype="bf16", tokens=1021, dim=776, vocab=10007, grads=True,
             ignored=0.2, weighted=True, pad=8),
        # the largest: a full training minibatch
        dict(name="vocab_bf16_t8192_v131072", op="vocab", dtype="bf16", tokens=8192, dim=4096, vocab=131072, grads=True,
             ignored=0.05, weighted=False, pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["dropout", "join", "join", "vocab", "vocab", "vocab"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 0, 8, 3])
    p = rng.choice([0.1, 0.1, 0.2, 0.5, rng.randint(1, 90) / 100])
    if op != "vocab":
        cols = _log_int(rng, 16, 8192)
        if rng.random() < 0.6:
            cols = (cols + 7) // 8 * 8
        rows = _log_int(rng, 1, min(8192, 8192 * 4096 // cols))
        case = dict(op=op, dtype=dtype, rows=rows, cols=cols, p=p, pad=pad)
        if op == "join":
            case["mode"] = rng.choice(["fwd", "bwd", "bwd", "q8"])
            if case["mode"] == "q8":
                case["group"] = rng.choice([0, 128])
            if case["mode"] != "bwd" and rng.random() < 0.5:
                case["p"] = 0.0
        return case
    vocab, dim = _log_int(rng, 10, 131072), _log_int(rng, 16, 4096)
    if rng.random() < 0.6:
        dim = (dim + 7) // 8 * 8
    most = LARGEST // (16 if dtype == "f32" else 1)
    tokens = _log_int(rng, 1, max(1, min(8192, most // (vocab * dim))))
    return dict(op="vocab", dtype=dtype, tokens=tokens, dim=dim, vocab=vocab, grads=rng.random() < 0.7,
                ignored=rng.choice([0.0, 0.0, 0.05, 0.5]), weighted=rng.random() < 0.3, pad=pad)


def work(case):
    """Bytes: every input read once, every output written once. Flops of elementwise passes: a few per element."""
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "vocab":
        t, d, v = case["tokens"], case["dim"], case["vocab"]
        bytes_ = (t + v) * d * size + t * 4 * (3 + case["weighted"])
        if case["grads"]:
            return {"bytes": bytes_ + (t + v) * d * size, "flops": 6 * t * d * v}
        return {"bytes": bytes_, "flops": 2 * t * d * v}
    n = case["rows"] * case["cols"]
    if case["op"] == "dropout":
        return {"bytes": 2 * n * size, "flops": 2 * n}
    if case["mode"] == "fwd":
        return {"bytes": 4 * n * size + 4 * (case["rows"] + case["cols"]), "flops": 6 * n}
    if case["mode"] == "q8":
        groups = -(-case["cols"] // case["group"]) if case["group"] else 1
        return {"bytes": 3 * n * size + n + 4 * case["rows"] * groups + 4 * case["cols"], "flops": 8 * n}
    return {"bytes": 5 * n * size + 4 * (case["rows"] + 2 * case["cols"]), "flops": 12 * n}


# ---- inputs -------------------------------------------------------------------------------------

def _rows(gen, rows, cols, pad, dtype, scale=1.0):
    """[rows][cols] inside a tensor whose rows are `pad` elements longer."""
    full = torch.randn((rows, cols + pad), device="cuda", generator=gen) * scale
    return full.to(DTYPES[dtype])[:, :cols]


def _space(rows, cols, pad, dtype):
    return torch.empty((rows, cols + pad), device="cuda", dtype=DTYPES[dtype])[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, pad = case["dtype"], case["pad"]
    s = {"case": case}
    if case["op"] == "vocab":
        t, d, v = case["tokens"], case["dim"], case["vocab"]
        # normed hidden states; logits of deviation 2, and targets the model partly expects
        s["h"] = _rows(gen, t, d, pad, dtype)
        s["w"] = _rows(gen, v, d, pad, dtype, 2.0 * d ** -0.5)
        target = torch.randint(0, v, (t,), device="cuda", generator=gen)
        known = torch.rand(t, device="cuda", generator=gen) < 0.5
        s["h"][known] = (s["h"][known].float() + 0.5 * d ** 0.5 * s["w"][target[known]].float()).to(DTYPES[dtype])
        gone = torch.rand(t, device="cuda", generator=gen) < case["ignored"]
        s["target"] = torch.where(gone, -1, target).to(torch.int32)
        s["weight"] = None
        if case["weighted"]:
            s["weight"] = torch.randint(0, 4, (t,), device="cuda", generator=gen).float() / t
    else:
        rows, cols = case["rows"], case["cols"]
        s["seed"], s["step"] = seed * 0x9E3779B97F4A7C15 % 2 ** 64, seed * 0x2545F4914F6CDD1D % 2 ** 64
        if case["op"] == "dropout":
            s["x"] = _rows(gen, rows, cols, pad, dtype)
        else:
            s["gain"] = 1.0 + 0.1 * torch.randn(cols, device="cuda", generator=gen)
            if case["mode"] == "bwd":
                s["x"] = _rows(gen, rows, cols, pad, dtype, 2.0)
                s["rstd"] = (s["x"].float().square().mean(1) + EPS).rsqrt()
                s["d_out"] = _rows(gen, rows, cols, pad, dtype, 1e-2)
                s["d_x"] = _rows(gen, rows, cols, pad, dtype, 1e-2)
            else:
                s["y"] = _rows(gen, rows, cols, pad, dtype)
                s["residual"] = _rows(gen, rows, cols, pad, dtype, 2.0)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The operator's handle, its workspace and the tensors that its results go to."""
    import paper_1804_10574_amd as ddg
    case = s["case"]
    dtype, pad = case["dtype"], case["pad"]
    kind = ddg.DDG_BF16 if dtype == "bf16" else ddg.DDG_F32
    stream = torch.cuda.current_stream().cuda_stream
    f32 = functools.partial(torch.empty, device="cuda", dtype=torch.float32)
    if case["op"] == "vocab":
        t, d, v, ld = case["tokens"], case["dim"], case["vocab"], case["dim"] + pad
        s["op"] = ddg.VocabLoss(t, d, v, kind, ld_h=ld, ld_w=ld, ld_dh=ld, ld_dw=ld, stream=stream)
        s["space"] = torch.empty(s["op"].workspace_bytes(case["grads"]), device="cuda", dtype=torch.uint8)
        s["loss"], s["row_loss"], s["lse"] = f32(1), f32(t), f32(t)
        s["dh"], s["dw"] = (_space(t, d, pad, dtype), _space(v, d, pad, dtype)) if case["grads"] else (None, None)
        return
    rows, cols, ld = case["rows"], case["cols"], case["cols"] + pad
    if case["op"] == "dropout":
        s["op"] = ddg.Dropout(rows, cols, kind, p=case["p"], seed=s["seed"], ld_x=ld, ld_y=ld, stream=stream)
        s["out"] = _space(rows, cols, pad, dtype)
        return
    s["op"] = ddg.JoinNorm(rows, cols, kind, eps=EPS, p=case["p"], seed=s["seed"], ld_y=ld, ld_residual=ld, ld_x=ld,
                           ld_out=cols if case["mode"] == "q8" else ld, group=case.get("group", 0), stream=stream)
    if case["mode"] == "bwd":
        s["space"] = torch.empty(s["op"].workspace_bytes(), device="cuda", dtype=torch.uint8)
        s["d_residual"], s["d_y"], s["d_gain"] = _space(rows, cols, pad, dtype), _space(rows, cols, pad, dtype), f32(cols)
    else:
        s["x_out"], s["rstd_out"] = _space(rows, cols, pad, dtype), f32(rows)
        if case["mode"] == "q8":
            s["out"] = torch.empty((rows, cols), device="cuda", dtype=torch.float8_e4m3fn)
            s["scale"] = f32(rows, -(-cols // case["group"]) if case["group"] else 1)
        else:
            s["out"] = _space(rows, cols, pad, dtype)


# ---- one pass -----------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    case, op = s["case"], s["op"]
    if case["op"] == "vocab":
        op(s["h"], s["w"], s["target"], weights=s["weight"], loss=s["loss"], row_loss=s["row_loss"], lse=s["lse"],
           dh=s["dh"], dw=s["dw"], workspace=s["space"])
        out = {"loss": s["loss"], "row_loss": s["row_loss"], "lse": s["lse"]}
        return {**out, "dh": s["dh"], "dw": s["dw"]} if case["grads"] else out
    if case["op"] == "dropout":
        op(s["x"], s["out"], step=s["step"])
        return s["out"]
    if case["mode"] == "bwd":
        op.backward(s["x"], s["rstd"], s["gain"], s["d_out"], s["d_x"], s["d_residual"], s["d_y"], s["d_gain"],
                    workspace=s["space"], step=s["step"])
        return {"d_residual": s["d_residual"], "d_y": s["d_y"], "d_gain": s["d_gain"]}
    if case["mode"] == "q8":
        op.forward_q8(s["y"], s["residual"], s["gain"], s["out"], s["scale"], x_out=s["x_out"], rstd=s["rstd_out"], step=s["step"])
        return {"x": s["x_out"], "q": s["out"], "scale": s["scale"], "rstd": s["rstd_out"]}
    op.forward(s["y"], s["residual"], s["gain"], s["out"], x_out=s["x_out"], rstd=s["rstd_out"], step=s["step"])
    return {"x": s["x_out"], "out": s["out"], "rstd": s["rstd_out"]}


# Philox4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011): a block is a function of
# a counter (column / 8, row, step) and a key (seed), and its 128 bits are the draws of 8 neighbouring columns, 16 bits each.
ROUNDS, M0, M1, K0, K1 = 7, 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85


def _high_low(m, x):
    """Both 32-bit halves of m * x for int64 tensors of 32-bit values, whose product would pass 63 bits."""
    low, high = m * (x & 0xffff), m * (x >> 16)
    return (high + (low >> 16)) >> 16, (((high & 0xffff) << 16) + low) & 0xffffffff


def _round(state, n, seed):
    a, b, c, d = state
    h0, l0 = _high_low(M0, a)
    h1, l1 = _high_low(M1, c)
    k0, k1 = (seed + n * K0) & 0xffffffff, ((seed >> 32) + n * K1) & 0xffffffff
    return h1 ^ b ^ k0, l1, h0 ^ d ^ k1, l0


def _dropout(x, s):
    """x in 32 bits with the case's share of its elements dropped, the others scaled to keep the mean."""
    case = s["case"]
    limit = round(65536 * float(np.float32(case["p"])))
    if limit == 0:
        return x
    rows, cols = x.shape
    row = torch.arange(rows, device=x.device)[:, None].expand(rows, (cols + 7) // 8)
    group = torch.arange((cols + 7) // 8, device=x.device)[None, :].expand_as(row)
    step = torch.full_like(row, s["step"] & 0xffffffff), torch.full_like(row, s["step"] >> 32)
    words = functools.reduce(lambda st, n: _round(st, n, s["seed"]), range(ROUNDS), (group, row, *step))
    words = torch.stack(words, -1)
    draws = torch.stack((words & 0xffff, words >> 16), -1).reshape(rows, -1)[:, :cols]
    return torch.where(draws >= limit, x * (65536 / (65536 - limit)), 0.0)


def _run_plain(s):
    case = s["case"]
    to = DTYPES[case["dtype"]]
    if case["op"] == "vocab":
        return _vocab_plain(s, to)
    if case["op"] == "dropout":
        return _dropout(s["x"].float(), s).to(to)
    gain, cols = s["gain"], case["cols"]
    if case["mode"] == "bwd":
        xhat = s["x"].float() * s["rstd"][:, None]
        d_out = s["d_out"].float()
        u = d_out * gain
        d_residual = s["d_x"].float() + s["rstd"][:, None] * (u - xhat * ((u * xhat).sum(1, keepdim=True) / cols))
        return {"d_residual": d_residual.to(to), "d_y": _dropout(d_residual, s).to(to), "d_gain": (d_out * xhat).sum(0)}
    x = s["residual"].float() + _dropout(s["y"].float(), s)
    rstd = torch.rsqrt((x * x).sum(1) / cols + EPS)
    out = x * rstd[:, None] * gain
    if case["mode"] == "fwd":
        return {"x": x.to(to), "out": out.to(to), "rstd": rstd}
    group = case["group"] or cols
    wide = torch.nn.functional.pad(out, (0, -cols % group)).reshape(case["rows"], -1, group)
    scale = (wide.abs().amax(-1) / E4M3_MAX).clamp_min(2.0 ** -126)
    q = (wide / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX).reshape(case["rows"], -1)[:, :cols]
    return {"x": x.to(to), "q": q.to(torch.float8_e4m3fn), "scale": scale, "rstd": rstd}


def _vocab_plain(s, to):
    case, target = s["case"], s["target"].long()
    h, w = s["h"].float(), s["w"].float()
    z = h @ w.T
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    there = target >= 0
    column = target.clamp_min(0)[:, None]
    row_loss = torch.where(there, lse - z.gather(1, column)[:, 0], 0.0)
    share = s["weight"] if case["weighted"] else 1.0 / there.sum().clamp_min(1)
    share = torch.where(there, share, 0.0)
    out = {"loss": (row_loss * share).sum()[None], "row_loss": row_loss, "lse": torch.where(there, lse, 0.0)}
    if case["grads"]:
        p = (e / total).scatter_add(1, column, torch.full_like(column, -1.0, dtype=torch.float32)) * share[:, None]
        out.update(dh=(p @ w).to(to), dw=(p.T @ h).to(to))
    return out


# ---- the definition in 64 bits -------------------------------------------------------------------

def _kept(s):
    """Truth values [rows][cols] on the host: unsigned 64-bit products, a column of blocks at a time."""
    case = s["case"]
    u = np.uint64
    low = u(0xffffffff)
    groups, rows = (case["cols"] + 7) // 8, case["rows"]
    c = [np.tile(np.arange(groups, dtype=u), (rows, 1)), np.repeat(np.arange(rows, dtype=u)[:, None], groups, 1),
         np.full((rows, groups), s["step"] & 0xffffffff, u), np.full((rows, groups), s["step"] >> 32, u)]
    key0, key1 = s["seed"] & 0xffffffff, s["seed"] >> 32
    for _ in range(ROUNDS):
        a, b = c[0] * u(M0), c[2] * u(M1)
        c = [(b >> u(32)) ^ c[1] ^ u(key0), b & low, (a >> u(32)) ^ c[3] ^ u(key1), a & low]
        key0, key1 = (key0 + K0) % 2 ** 32, (key1 + K1) % 2 ** 32
    draws = np.empty((rows, groups, 8), u)
    for j in range(4):
        draws[:, :, 2 * j], draws[:, :, 2 * j + 1] = c[j] & u(0xffff), c[j] >> u(16)
    limit = int(np.rint(np.float64(np.float32(case["p"])) * 65536))
    return torch.from_numpy(draws.reshape(rows, -1)[:, :case["cols"]] >= u(limit)).cuda(), limit


def _dropped(x, s):
    if s["case"]["p"] == 0:
        return x
    keep, limit = _kept(s)
    return keep.double() * x * (65536.0 / (65536 - limit))


def exact(case, seed):
    s = prepare(case, seed)
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["op"] == "dropout":
        return _dropped(f["x"], s)
    if case["op"] == "vocab":
        z = f["h"] @ f["w"].T
        lse = torch.logsumexp(z, 1)
        rows = torch.arange(case["tokens"], device="cuda")
        there = s["target"] >= 0
        row_loss = torch.zeros_like(lse)
        row_loss[there] = (lse - z[rows, s["target"].long()])[there]
        share = f["weight"] * there if case["weighted"] else there.double() / max(1, int(there.sum()))
        out = {"loss": torch.dot(row_loss, share)[None], "row_loss": row_loss, "lse": lse * there}
        if case["grads"]:
            g = z.sub_(lse[:, None]).exp_()
            g[rows[there], s["target"].long()[there]] -= 1.0
            g.mul_(share[:, None])
            out.update(dh=g @ f["w"], dw=g.T @ f["h"])
        return out
    if case["mode"] == "bwd":
        n, r = f["x"], f["rstd"][:, None]
        u = f["d_out"] * f["gain"]
        d_res = f["d_x"] + r * u - r ** 3 * n * (u * n).mean(1, keepdim=True)
        return {"d_residual": d_res, "d_y": _dropped(d_res, s), "d_gain": torch.einsum("rc,rc,r->c", f["d_out"], n, f["rstd"])}
    x = f["residual"] + _dropped(f["y"], s)
    rstd = 1.0 / torch.sqrt(x.pow(2).mean(1) + EPS)
    out = x * torch.outer(rstd, f["gain"])
    if case["mode"] == "fwd":
        return {"x": x, "out": out, "rstd": rstd}
    group = case["group"] or case["cols"]
    parts = out.split(group, 1)
    scale = torch.stack([g.abs().amax(1) for g in parts], 1) / E4M3_MAX
    q = torch.cat([g / scale[:, i:i + 1] for i, g in enumerate(parts)], 1)
    return {"x": x, "q": q.float().to(torch.float8_e4m3fn), "scale": scale, "rstd": rstd}
