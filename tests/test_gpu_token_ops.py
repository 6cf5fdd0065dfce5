"""Dropout, the join of a residual branch with its norm, and the vocabulary loss against their definitions in 64 bits.

Bounds (2-norm of the difference over that of the result), from the formats: a bf16 result is rounded once, at most 2^-8 of each
element; bf16 gradients of the vocabulary loss are products of P, rounded twice, and are rounded themselves: three independent roundings whose squares
average a third of 2^-16 or less, together 2^-8, and half as much again for luck. fp32: sums of
n terms in any order differ by about sqrt(n) * 2^-24 of the norm of their terms: 1e-5 up to n = 2^14, which also covers results whose terms cancel by
a factor of three."""
import numpy as np
import pytest

from tests import token_ref as R

pytestmark = pytest.mark.gpu

ROUND = {"bf16": 2.0 ** -8, "f32": 1e-5}
GRAD = {"bf16": 1.5 * 2.0 ** -8, "f32": 1e-5}
SUMS = 1e-5
SEED, STEP = 0x9E3779B97F4A7C15, (5 << 32) + 17


def setup(dtype, seed=1):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_1804_10574_amd as ddg
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    kind = ddg.DDG_BF16 if dtype == "bf16" else ddg.DDG_F32

    def rows(n, c, pad=0, scale=1.0, shift=0):
        """[n][c] of normal values inside rows that are `pad` longer, `shift` elements into the allocation."""
        full = torch.randn(n * (c + pad) + shift, device="cuda", generator=gen) * scale
        return full.to(t)[shift:].view(n, c + pad)[:, :c]

    def space(n, c, pad=0, dt=None):
        return torch.full((n, c + pad), 7.0, device="cuda", dtype=dt or t)[:, :c]

    return torch, ddg, kind, t, gen, rows, space


def untouched(torch, view, pad):
    """The elements between the rows still hold what they held."""
    if not pad:
        return True
    return bool((view._base.view(view.shape[0], -1)[:, view.shape[1]:] == 7.0).all())


# ---- dropout -------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,p", [(1, 1, 0, 0.5), (3, 8, 0, 0.1), (7, 9, 0, 0.3), (128, 64, 0, 0.5), (65, 200, 8, 0.9), (33, 1001, 3, 0.2),
                                             (5, 40, 0, 0.0), (2, 16, 0, 0.9999999), (300, 4096, 0, 0.1), (70000, 8, 0, 0.5)])
def test_dropout(dtype, rows, cols, pad, p):
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    print(f"case dropout {dtype} {rows}x{cols}+{pad} p {p}", flush=True)
    x, y = mk(rows, cols, pad), space(rows, cols, pad)
    op = ddg.Dropout(rows, cols, kind, p=p, seed=SEED, ld_x=cols + pad, ld_y=cols + pad)
    op(x, y, step=STEP)
    want = R.dropout(x, p, SEED, STEP)
    assert torch.equal(y == 0, want == 0) or bool((x == 0).any())
    assert R.off(y, want) <= ROUND[dtype]
    assert untouched(torch, y, pad)
    again = x.clone() if not pad else None
    if again is not None:                                      # in place, and another step is another mask
        op(again, again, step=STEP)
        assert torch.equal(again, y)
        other = space(rows, cols)
        op(x, other, step=STEP + 1)
        assert rows * cols < 64 or p in (0.0, 0.9999999) or not torch.equal(other, y)


def test_dropout_share_and_what_is_dropped():
    torch, ddg, kind, t, gen, mk, space = setup("f32")
    rows, cols, p = 512, 1024, 0.25
    x = torch.full((rows, cols), float("nan"), device="cuda")
    keep = torch.from_numpy(R.kept(rows, cols, p, SEED, STEP)).cuda()
    x[keep] = 3.0
    y = space(rows, cols)
    ddg.Dropout(rows, cols, kind, p=p, seed=SEED)(x, y, step=STEP)
    assert torch.equal(y, torch.where(keep, 4.0, 0.0))         # 3 / (1 - 1/4); what is dropped is 0, NaN or not
    n = rows * cols
    assert abs(float(keep.float().mean()) - 0.75) < 5 * (0.75 * 0.25 / n) ** 0.5


# ---- the join ------------------------------------------------------------------------------------

SHAPES = [(1, 1, 0), (2, 7, 0), (1, 2048, 0), (5, 64, 0), (9, 512, 0), (4, 520, 8), (3, 1001, 3), (6, 2056, 0), (130, 4096, 0), (3, 8192, 8), (2, 8200, 0),
          (2, 32768, 0), (2, 20001, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad", SHAPES)
@pytest.mark.parametrize("p,plain", [(0.0, False), (0.3, False), (0.3, True)])
def test_join_forward(dtype, rows, cols, pad, p, plain):
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    print(f"case join {dtype} {rows}x{cols}+{pad} p {p} plain {plain}", flush=True)
    ld = cols + pad
    y, res = mk(rows, cols, pad), None if plain else mk(rows, cols, pad, 2.0)
    gain = None if plain else torch.randn(cols, device="cuda", generator=gen)
    x, out, rstd = space(rows, cols, pad), space(rows, cols, pad), space(rows, 1, dt=torch.float32)
    op = ddg.JoinNorm(rows, cols, kind, eps=1e-5, p=p, seed=SEED, ld_y=ld, ld_residual=ld, ld_x=ld, ld_out=ld)
    op.forward(y, res, gain, out, x_out=x, rstd=rstd, step=STEP)
    wx, wo, wr = R.join(y, res, gain, 1e-5, p, SEED, STEP)
    assert R.off(x, wx) <= ROUND[dtype] and R.off(out, wo) <= ROUND[dtype] and R.off(rstd, wr) <= SUMS
    assert untouched(torch, x, pad) and untouched(torch, out, pad)
    if res is not None:                                        # the stream updated in place, nothing else asked for
        out2 = space(rows, cols, pad)
        op.forward(y, res, gain, out2, x_out=res, step=STEP)
        assert torch.equal(out2, out) and torch.equal(res, x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad", SHAPES + [(3000, 96, 0), (1500, 1024, 0)])
@pytest.mark.parametrize("p,plain", [(0.0, True), (0.3, False)])
def test_join_backward(dtype, rows, cols, pad, p, plain):
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    print(f"case join backward {dtype} {rows}x{cols}+{pad} p {p} plain {plain}", flush=True)
    ld = cols + pad
    x, d_out, d_x = mk(rows, cols, pad, 2.0), mk(rows, cols, pad), None if plain else mk(rows, cols, pad)
    gain = None if plain else torch.randn(cols, device="cuda", generator=gen)
    rstd = (x.float().square().mean(1) + 1e-5).rsqrt()
    d_res, d_y, d_gain = space(rows, cols, pad), space(rows, cols, pad), space(1, cols, dt=torch.float32)
    op = ddg.JoinNorm(rows, cols, kind, p=p, seed=SEED, ld_y=ld, ld_residual=ld, ld_x=ld, ld_out=ld)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    op.backward(x, rstd, gain, d_out, d_x, d_res, d_y, d_gain, workspace=ws, step=STEP)
    wr, wy, wg = R.join_backward(x, rstd, gain, d_out, d_x, p, SEED, STEP)
    # one column: out = +-1 whatever x is, and d_residual without d_x is eps times the rest, a difference of nearly equal numbers
    if cols > 1 or not plain:
        assert R.off(d_res, wr) <= ROUND[dtype] and R.off(d_y, wy) <= ROUND[dtype]
    assert R.off(d_gain, wg) <= SUMS
    assert untouched(torch, d_res, pad) and untouched(torch, d_y, pad)
    if d_x is not None:                                        # one result at a time, and the stream's gradient in place
        only = space(rows, cols, pad)
        op.backward(x, rstd, gain, d_out, d_x, d_y=only, step=STEP)
        assert torch.equal(only, d_y)
        op.backward(x, rstd, gain, d_out, d_x, d_residual=d_x, step=STEP)
        assert torch.equal(d_x, d_res)


@pytest.mark.parametrize("rows", [0, 1])
def test_join_backward_of_few_rows_writes_the_gain(rows):
    torch, ddg, kind, t, gen, mk, space = setup("f32")
    d_gain = space(1, 40, dt=torch.float32)
    op = ddg.JoinNorm(rows, 40, kind)
    ws = torch.empty(op.workspace_bytes(), device="cuda", dtype=torch.uint8)
    x, d_out = mk(rows, 40), mk(rows, 40)
    rstd = torch.ones(rows, device="cuda")
    op.backward(x, rstd, None, d_out, d_gain=d_gain, workspace=ws)
    assert R.off(d_gain, (x.double() * d_out.double()).sum(0)) <= SUMS


def test_join_gradient_against_differences():
    """d f / d y and d f / d residual of f = sum(out * c) + sum(x * e), by central differences in 64 bits at random directions."""
    torch, ddg, kind, t, gen, mk, space = setup("f32")
    rows, cols, p, eps = 5, 77, 0.3, 1e-5
    y, res, c, e, gain = mk(rows, cols), mk(rows, cols), mk(rows, cols), mk(rows, cols), torch.randn(cols, device="cuda", generator=gen)
    x, out, rstd = space(rows, cols), space(rows, cols), space(rows, 1)
    op = ddg.JoinNorm(rows, cols, kind, eps=eps, p=p, seed=SEED)
    op.forward(y, res, gain, out, x_out=x, rstd=rstd, step=STEP)
    d_res, d_y, d_gain = space(rows, cols), space(rows, cols), space(1, cols)
    ws = torch.empty(op.workspace_bytes(), device="cuda", dtype=torch.uint8)
    op.backward(x, rstd, gain, c, e, d_res, d_y, d_gain, workspace=ws, step=STEP)

    def f(yy, rr, gg):
        xx, oo, _ = R.join(yy, rr, gg, eps, p, SEED, STEP)
        return float((oo * c.double()).sum() + (xx * e.double()).sum())

    step = 1e-5
    for which, grad in ((0, d_y), (1, d_res), (2, d_gain[0])):
        args = [y.double(), res.double(), gain.double()]
        v = torch.randn(args[which].shape, device="cuda", generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + step * v, args[which] - step * v
        slope = (f(*up) - f(*down)) / (2 * step)
        size = float(grad.double().norm() * v.norm())
        assert abs(slope - float((grad.double() * v).sum())) <= 1e-5 * size


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad", SHAPES)
@pytest.mark.parametrize("group", [0, 128])
def test_join_q8(dtype, rows, cols, pad, group):
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    print(f"case join q8 {dtype} {rows}x{cols}+{pad} group {group}", flush=True)
    ld = cols + pad
    y, res, gain = mk(rows, cols, pad), mk(rows, cols, pad), torch.randn(cols, device="cuda", generator=gen)
    y[0].zero_(); res[0].zero_()                                # a row of zeros: the least scale, zeros
    groups = -(-cols // group) if group else 1
    q = torch.full((rows, ld), 0x11, device="cuda", dtype=torch.uint8)
    scale = space(rows, groups, dt=torch.float32)
    op = ddg.JoinNorm(rows, cols, kind, eps=1e-5, p=0.0, ld_y=ld, ld_residual=ld, ld_x=ld, ld_out=ld, group=group)
    op.forward_q8(y, res, gain, q, scale)
    _, want, _ = R.join(y, res, gain, 1e-5)
    wide = torch.nn.functional.pad(want, (0, -cols % (group or cols))).view(rows, groups, -1)
    ws = (wide.abs().amax(2) / 448).clamp_min(2.0 ** -126)
    assert R.off(scale, ws) <= SUMS
    got = q[:, :cols].view(torch.float8_e4m3fn).double()
    deq = got * scale.double().repeat_interleave(group or cols, 1)[:, :cols]
    # half a step: 2^-4 of the value, and 2^-10 of the scale's unit below the normal range; the 32-bit value may lie a rounding to the side
    room = (want.abs() * 2.0 ** -4 + scale.double().repeat_interleave(group or cols, 1)[:, :cols] * 2.0 ** -10) * (1 + 1e-3)
    assert bool(((deq - want).abs() <= room).all())
    assert float(got.abs().max()) <= 448
    nearest = (want / ws.repeat_interleave(group or cols, 1)[:, :cols]).float().to(torch.float8_e4m3fn).double()
    assert float((got != nearest).double().mean()) <= 1e-3 + 1.0 / (rows * cols)
    assert not pad or bool((q[:, cols:] == 0x11).all())


def test_join_with_infinity_or_nan_keeps_to_its_row():
    torch, ddg, kind, t, gen, mk, space = setup("bf16")
    rows, cols = 6, 256
    y, res = mk(rows, cols), mk(rows, cols)
    op = ddg.JoinNorm(rows, cols, kind)
    clean, out = space(rows, cols), space(rows, cols)
    op.forward(y, res, None, clean)
    y[1, 3], res[4, 200] = float("inf"), float("nan")
    op.forward(y, res, None, out)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda"); bad[1] = bad[4] = True
    assert torch.equal(out[~bad], clean[~bad]) and bool(out[4].isnan().all()) and bool(out[1, 3].isnan())
    q, scale = torch.empty((rows, cols), device="cuda", dtype=torch.uint8), space(rows, 1, dt=torch.float32)
    op.forward_q8(y, res, None, q, scale)
    deq = q.view(torch.float8_e4m3fn).double() * scale.double()
    assert bool(deq[4].isnan().all()) and bool(deq[~bad].isfinite().all())


# ---- the vocabulary loss -------------------------------------------------------------------------

# tokens, width, vocabulary, pad: single tokens, tile edges (32, 128, 256) from both sides, odd sizes
VOCAB = [(1, 16, 10, 0), (1, 1024, 5000, 0), (2, 8, 1, 0), (3, 24, 129, 0), (31, 64, 100, 0), (32, 64, 128, 0), (33, 72, 127, 8), (64, 200, 1000, 0),
         (65, 128, 257, 0), (129, 264, 3000, 0), (256, 64, 100, 0), (300, 1000, 2999, 3), (511, 512, 8192, 0), (257, 777, 10007, 0), (1000, 136, 4096, 0)]


def vocab_case(dtype, tokens, dim, vocab, pad, gone, weighted, shift=0):
    torch, ddg, kind, t, gen, mk, space = setup(dtype, seed=tokens + vocab)
    h, w = mk(tokens, dim, pad, shift=shift), mk(vocab, dim, pad, 2.0 * dim ** -0.5, shift=shift)
    target = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
    if gone:
        target[torch.rand(tokens, device="cuda", generator=gen) < gone] = -100
    weights = torch.rand(tokens, device="cuda", generator=gen) if weighted else None
    return torch, ddg, kind, t, h, w, target, weights, space


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,dim,vocab,pad", VOCAB)
@pytest.mark.parametrize("gone,weighted", [(0.0, False), (0.4, True)])
def test_vocab_loss(dtype, tokens, dim, vocab, pad, gone, weighted):
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case(dtype, tokens, dim, vocab, pad, gone, weighted)
    print(f"case vocab {dtype} {tokens} {dim} {vocab} +{pad} gone {gone} weighted {weighted}", flush=True)
    ld = dim + pad
    op = ddg.VocabLoss(tokens, dim, vocab, kind, ld_h=ld, ld_w=ld, ld_dh=ld, ld_dw=ld)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)      # (NaN in every type)
    loss, rows, lse = space(1, 1, dt=torch.float32), space(1, tokens, dt=torch.float32), space(1, tokens, dt=torch.float32)
    dh, dw = space(tokens, dim, pad), space(vocab, dim, pad)
    op(h, w, target, weights, loss, rows, lse, dh, dw, workspace=ws)
    wl, wr, we, wdh, wdw = R.vocab(h, w, target, weights)
    assert R.off(loss, wl) <= SUMS and R.off(rows, wr) <= SUMS and R.off(lse, we) <= SUMS
    assert R.off(dh, wdh) <= GRAD[dtype] and R.off(dw, wdw) <= GRAD[dtype]
    assert bool((dh[target < 0] == 0).all())
    assert untouched(torch, dh, pad) and untouched(torch, dw, pad)
    # the loss alone has the same values, and takes no gradient's workspace
    ws2 = torch.full((op.workspace_bytes(False),), 255, device="cuda", dtype=torch.uint8)
    loss2, rows2 = space(1, 1, dt=torch.float32), space(1, tokens, dt=torch.float32)
    op(h, w, target, weights, loss2, rows2, workspace=ws2)
    assert R.off(loss2, wl) <= SUMS and R.off(rows2, wr) <= SUMS
    # one gradient at a time; bits do not depend on what else is asked for
    dw2, dh2 = space(vocab, dim, pad), space(tokens, dim, pad)
    op(h, w, target, weights, dw=dw2, workspace=ws)
    op(h, w, target, weights, dh=dh2, workspace=ws)
    assert torch.equal(dw, dw2) and torch.equal(dh, dh2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_vocab_loss_of_unaligned_operands_and_dw_in_32_bits(dtype):
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case(dtype, 40, 64, 333, 0, 0.2, False, shift=1)
    op = ddg.VocabLoss(40, 64, 333, kind, dw_f32=True)
    ws = torch.empty(op.workspace_bytes() + (333 + 40) * 64 * 4 + 512, device="cuda", dtype=torch.uint8)
    loss, dw = space(1, 1, dt=torch.float32), space(333, 64, dt=torch.float32)
    op(h, w, target, None, loss, dw=dw, workspace=ws)
    wl, _, _, _, wdw = R.vocab(h, w, target)
    assert R.off(loss, wl) <= SUMS and R.off(dw, wdw) <= GRAD[dtype]


@pytest.mark.parametrize("gradients", [True, False])
@pytest.mark.parametrize("tokens", [0, 5, 200])
def test_vocab_loss_without_any_target(tokens, gradients):
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case("bf16", tokens, 64, 300, 0, 0.0, False)
    target.fill_(-1)
    h.fill_(float("nan"))
    op = ddg.VocabLoss(tokens, 64, 300, kind)
    ws = torch.full((max(256, op.workspace_bytes()),), 255, device="cuda", dtype=torch.uint8)
    loss, rows, lse = space(1, 1, dt=torch.float32), space(1, tokens, dt=torch.float32), space(1, tokens, dt=torch.float32)
    dh, dw = (space(tokens, 64), space(300, 64)) if gradients else (None, None)
    op(h, w, target, None, loss, rows, lse, dh, dw, workspace=ws)
    assert float(loss) == 0 and bool((rows == 0).all()) and bool((lse == 0).all())
    assert not gradients or (bool((dh == 0).all()) and bool((dw == 0).all()))


def test_vocab_loss_leaves_out_what_has_no_target():
    """NaN and infinity in tokens without a target reach nothing; a target past the vocabulary is a NaN loss of its own token."""
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case("bf16", 300, 128, 2000, 0, 0.3, False)
    gone = target < 0
    op = ddg.VocabLoss(300, 128, 2000, kind)
    ws = torch.empty(op.workspace_bytes(), device="cuda", dtype=torch.uint8)
    f32 = lambda n: space(1, n, dt=torch.float32)  # noqa: E731
    loss, dh, dw = f32(1), space(300, 128), space(2000, 128)
    op(h, w, target, None, loss, None, None, dh, dw, workspace=ws)
    h[gone] = float("nan")
    h[gone.nonzero()[0]] = float("inf")
    loss2, dh2, dw2 = f32(1), space(300, 128), space(2000, 128)
    op(h, w, target, None, loss2, None, None, dh2, dw2, workspace=ws)
    assert torch.equal(loss, loss2) and torch.equal(dh, dh2) and torch.equal(dw, dw2)
    first = int((~gone).nonzero()[0])
    target[first] = 2000
    rows = f32(300)
    op(h, w, target, None, loss2, rows, workspace=ws)
    nan = rows[0].isnan()
    assert bool(loss2.isnan()) and int(nan.sum()) == 1 and bool(nan[first])


def test_vocab_loss_of_confident_tokens():
    """Logits far apart: the probability of the target is 1 to many digits; nothing overflows, and what is left of p - 1 is off by roundings of 1."""
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case("f32", 70, 64, 500, 0, 0.0, False)
    w.mul_(8.0)
    h.copy_(w[target.long()] * 0.15)
    op = ddg.VocabLoss(70, 64, 500, kind)
    ws = torch.empty(op.workspace_bytes(), device="cuda", dtype=torch.uint8)
    dh, lse = space(70, 64), space(1, 70)
    op(h, w, target, None, None, None, lse, dh, None, workspace=ws)
    _, _, we, wdh, _ = R.vocab(h, w, target)
    assert R.off(lse, we) <= SUMS
    # P = p - 1 in 32 bits, p a quotient of two rounded numbers: a few times 2^-24, times a row of w and the mean's 1/70
    assert bool(((dh.double() - wdh).norm(dim=1) <= 2.0 ** -21 / 70 * w.double().norm(dim=1).max()).all())


def test_vocab_loss_in_several_panels():
    """A vocabulary so large that the tokens take more than one turn: dw is summed over the turns."""
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case("bf16", 700, 16, 1200000, 0, 0.1, False)
    op = ddg.VocabLoss(700, 16, 1200000, kind)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    assert ws.numel() < 700 * 1200000 * 2
    loss, dh, dw = space(1, 1, dt=torch.float32), space(700, 16), space(1200000, 16)
    op(h, w, target, None, loss, None, None, dh, dw, workspace=ws)
    wl, _, _, wdh, wdw = R.vocab(h, w, target)
    assert R.off(loss, wl) <= SUMS and R.off(dh, wdh) <= GRAD["bf16"] and R.off(dw, wdw) <= GRAD["bf16"]


def test_vocab_gradient_against_differences():
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case("f32", 50, 40, 300, 0, 0.2, True)
    op = ddg.VocabLoss(50, 40, 300, kind)
    ws = torch.empty(op.workspace_bytes(), device="cuda", dtype=torch.uint8)
    dh, dw = space(50, 40), space(300, 40)
    op(h, w, target, weights, dh=dh, dw=dw, workspace=ws)
    gen = torch.Generator(device="cuda"); gen.manual_seed(3)
    step = 1e-5
    for which, grad in ((0, dh), (1, dw)):
        args = [h.double(), w.double()]
        v = torch.randn(args[which].shape, device="cuda", generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + step * v, args[which] - step * v
        slope = float(R.vocab(*up, target, weights)[0] - R.vocab(*down, target, weights)[0]) / (2 * step)
        assert abs(slope - float((grad.double() * v).sum())) <= 1e-5 * float(grad.double().norm() * v.norm())


# ---- streams and graphs --------------------------------------------------------------------------

def test_on_another_stream_and_in_a_graph():
    """One module's end (join, loss, join backward) captured on a stream of its own and replayed on new inputs: the eager bits every time."""
    torch, ddg, kind, t, gen, mk, space = setup("bf16")
    rows, cols, vocab = 96, 256, 1000
    stream = torch.cuda.Stream()
    join = ddg.JoinNorm(rows, cols, kind, p=0.1, seed=SEED, stream=stream.cuda_stream)
    head = ddg.VocabLoss(rows, cols, vocab, kind, stream=stream.cuda_stream)
    f32 = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    y, res, w, gain = mk(rows, cols), mk(rows, cols), mk(vocab, cols, scale=0.1), torch.ones(cols, device="cuda")
    target = torch.randint(-1, vocab, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    x, out, rstd, loss, dh, dw = space(rows, cols), space(rows, cols), f32(rows), f32(1), space(rows, cols), space(vocab, cols)
    d_res, d_y, d_gain = space(rows, cols), space(rows, cols), f32(cols)
    ws = torch.empty(max(join.workspace_bytes(), head.workspace_bytes()), device="cuda", dtype=torch.uint8)

    def work():
        join.forward(y, res, gain, out, x_out=x, rstd=rstd, step=STEP)
        head(out, w, target, loss=loss, dh=dh, dw=dw, workspace=ws)
        join.backward(x, rstd, gain, dh, None, d_res, d_y, d_gain, workspace=ws, step=STEP)

    results = (x, out, rstd, loss, dh, dw, d_res, d_y, d_gain)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        work()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        work()
    for turn in range(4):
        y.copy_(mk(rows, cols)); target.copy_(torch.randint(-1, vocab, (rows,), device="cuda", generator=gen, dtype=torch.int32))
        torch.cuda.synchronize()
        work()
        stream.synchronize()
        want = [v.clone() for v in results]
        for v in results:
            v.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want)), turn
        wl = R.vocab(out, w, target)[0]
        assert R.off(loss, wl) <= SUMS


# fp32 sizes whose products are taken in planes (all three, in one panel and in several), and just not
PLANES = [(1100, 520, 9000, 0, 0.3), (2000, 300, 4097, 3, 0.0), (900, 136, 150001, 0, 0.1), (256, 128, 40000, 0, 0.0), (700, 1028, 3000, 0, 0.0)]


@pytest.mark.parametrize("tokens,dim,vocab,pad,gone", PLANES)
def test_vocab_loss_of_long_fp32_products(tokens, dim, vocab, pad, gone):
    """Full precision whichever matrix instructions a size takes: the bounds of fp32 sums, with operands over 60 powers of two."""
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case("f32", tokens, dim, vocab, pad, gone, True)
    gen = torch.Generator(device="cuda"); gen.manual_seed(7)
    powers = torch.randint(-30, 31, (dim,), device="cuda", generator=gen).float()
    h.mul_(torch.exp2(powers)); w.mul_(torch.exp2(-powers))
    ld = dim + pad
    op = ddg.VocabLoss(tokens, dim, vocab, kind, ld_h=ld, ld_w=ld, ld_dh=ld, ld_dw=ld)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    loss, lse, dh, dw = space(1, 1), space(1, tokens), space(tokens, dim, pad), space(vocab, dim, pad)
    op(h, w, target, weights, loss, None, lse, dh, dw, workspace=ws)
    wl, _, we, wdh, wdw = R.vocab(h, w, target, weights)
    assert R.off(loss, wl) <= SUMS and R.off(lse, we) <= SUMS
    scale = torch.exp2(powers).double()
    assert R.off(dh.double() * scale, wdh * scale) <= GRAD["f32"] and R.off(dw.double() / scale, wdw / scale) <= GRAD["f32"]
    assert untouched(torch, dh, pad) and untouched(torch, dw, pad)
    again = space(vocab, dim, pad)
    op(h, w, target, weights, dw=again, workspace=ws)
    assert torch.equal(again, dw)


@pytest.mark.parametrize("tokens", [1, 2, 3, 7, 16, 17, 64])
def test_loss_of_few_tokens_alone(tokens):
    """The one-launch join of maxima and sums and the launches that more tokens take."""
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case("bf16", tokens, 72, 9001, 0, 0.3, True)
    target[0] = 9000
    op = ddg.VocabLoss(tokens, 72, 9001, kind)
    ws = torch.full((op.workspace_bytes(False),), 255, device="cuda", dtype=torch.uint8)
    for a in (weights, None):
        loss, rows, lse = space(1, 1, dt=torch.float32), space(1, tokens, dt=torch.float32), space(1, tokens, dt=torch.float32)
        op(h, w, target, a, loss, rows, lse, workspace=ws)
        wl, wr, we, _, _ = R.vocab(h, w, target, a)
        assert R.off(loss, wl) <= SUMS and R.off(rows, wr) <= SUMS and R.off(lse, we) <= SUMS


# ---- far apart -----------------------------------------------------------------------------------

def test_rows_beyond_32_bits():
    """Rows 2 and 4 MiB apart in tensors of 4.6 and 9 GB: offsets that pass 2^32 bytes and 2^31 elements, in every operand."""
    torch, ddg, kind, t, gen, mk, space = setup("bf16")
    rows, cols, ld = 2200, 72, 1 << 20
    far = lambda n, step: torch.empty(n * step, device="cuda", dtype=t).view(n, step)[:, :cols]  # noqa: E731
    x, y = far(rows, ld), far(rows, 2 * ld)
    x.copy_(mk(rows, cols))
    ddg.Dropout(rows, cols, kind, p=0.3, seed=SEED, ld_x=ld, ld_y=2 * ld)(x, y, step=STEP)
    assert R.off(y, R.dropout(x, 0.3, SEED, STEP)) <= ROUND["bf16"]
    out = space(rows, cols)
    ddg.JoinNorm(rows, cols, kind, eps=1e-5, ld_y=ld, ld_residual=2 * ld).forward(x, y, None, out)
    assert R.off(out, R.join(x, y, None, 1e-5)[1]) <= ROUND["bf16"]
    # as the vocabulary's rows, and their gradients'
    tokens = 300
    h, target = mk(tokens, cols), torch.randint(0, rows, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
    op = ddg.VocabLoss(tokens, cols, rows, kind, ld_w=ld, ld_dw=2 * ld)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    loss, dh = space(1, 1, dt=torch.float32), space(tokens, cols)
    op(h, x, target, None, loss, dh=dh, dw=y, workspace=ws)
    wl, _, _, wdh, wdw = R.vocab(h, x, target)
    assert R.off(loss, wl) <= SUMS and R.off(dh, wdh) <= GRAD["bf16"] and R.off(y, wdw) <= GRAD["bf16"]


@pytest.mark.parametrize("dtype,dim,vocab", [("bf16", 24, 900001), ("f32", 512, 160000)])
def test_vocab_loss_in_several_panels_with_dw_in_32_bits(dtype, dim, vocab):
    """Also in planes (fp32, 512 wide): dw is summed over the turns in place."""
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case(dtype, 900, dim, vocab, 0, 0.1, False)
    op = ddg.VocabLoss(900, dim, vocab, kind, dw_f32=True)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    loss, dh, dw = space(1, 1, dt=torch.float32), space(900, dim), space(vocab, dim, dt=torch.float32)
    op(h, w, target, None, loss, None, None, dh, dw, workspace=ws)
    wl, _, _, wdh, wdw = R.vocab(h, w, target)
    assert R.off(loss, wl) <= SUMS and R.off(dh, wdh) <= GRAD[dtype] and R.off(dw, wdw) <= GRAD[dtype]


# sizes at which neither product of the gradients fills the chip: one launch has both, in small, middle and large tiles, with and without parts
TOGETHER = [(1021, 777, 10007, 0), (500, 1000, 8000, 8), (700, 130, 20000, 3), (4100, 260, 1000, 0), (300, 1100, 5001, 0), (1500, 700, 15000, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,dim,vocab,pad", TOGETHER)
@pytest.mark.parametrize("gone,dw_f32", [(0.0, False), (0.6, True)])
def test_vocab_gradients_together(dtype, tokens, dim, vocab, pad, gone, dw_f32):
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case(dtype, tokens, dim, vocab, pad, gone, gone > 0)
    ld = dim + pad
    op = ddg.VocabLoss(tokens, dim, vocab, kind, ld_h=ld, ld_w=ld, ld_dh=ld, ld_dw=ld, dw_f32=dw_f32)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    wide = torch.float32 if dw_f32 else t
    loss, dh, dw = space(1, 1, dt=torch.float32), space(tokens, dim, pad), space(vocab, dim, pad, dt=wide)
    op(h, w, target, weights, loss, None, None, dh, dw, workspace=ws)
    wl, _, _, wdh, wdw = R.vocab(h, w, target, weights)
    assert R.off(loss, wl) <= SUMS and R.off(dh, wdh) <= GRAD[dtype] and R.off(dw, wdw) <= GRAD[dtype]
    assert untouched(torch, dh, pad) and untouched(torch, dw, pad)
    ws.fill_(255)
    again = [space(1, 1, dt=torch.float32), space(tokens, dim, pad), space(vocab, dim, pad, dt=wide)]
    op(h, w, target, weights, again[0], None, None, again[1], again[2], workspace=ws)
    assert torch.equal(loss, again[0]) and torch.equal(dh, again[1]) and torch.equal(dw, again[2])


@pytest.mark.parametrize("dtype,vocab,dim,dw_f32", [("bf16", 33000, 1032, False), ("bf16", 33001, 1030, False), ("bf16", 17000, 1001, True), ("f32", 9000, 2000, False)])
def test_vocab_large_dw(dtype, vocab, dim, dw_f32):
    """dw of 64 MiB and more (few tokens, a launch of its own), in 16-byte pieces and not, read back by another kernel."""
    torch, ddg, kind, t, h, w, target, weights, space = vocab_case(dtype, 40, dim, vocab, 0, 0.2, True)
    op = ddg.VocabLoss(40, dim, vocab, kind, dw_f32=dw_f32)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    loss, dh, dw = space(1, 1, dt=torch.float32), space(40, dim), space(vocab, dim, dt=torch.float32 if dw_f32 else t)
    for _ in range(2):
        op(h, w, target, weights, loss, None, None, dh, dw, workspace=ws)
    wl, _, _, wdh, wdw = R.vocab(h, w, target, weights)
    assert R.off(loss, wl) <= SUMS and R.off(dh, wdh) <= GRAD[dtype] and R.off(dw, wdw) <= GRAD[dtype]
