"""The vocabulary loss at sizes that take every kind of launch (the host's tests assert which), against its definition in 64 bits.

Bounds: as in the other tests of this operator; sums of n terms in fp32 are off by sqrt(n) * 2^-24, which passes 1e-5 from n = 2^14.8 on."""
import pytest

from tests import test_gpu_token_ops as ops
from tests import token_ref as R
from tests.vocab_plan import KINDS, PLANES

pytestmark = pytest.mark.gpu


def grad(dtype, n):
    return ops.GRAD["bf16"] if dtype == "bf16" else max(ops.GRAD["f32"], n ** 0.5 * 2.0 ** -24)


def check(dtype, tokens, dim, vocab, gone, weighted, powers=0):
    """powers: columns of h and w are multiplied by up to 2^+-powers and its reciprocal, which leaves the logits alone, and the gradients' columns are taken back."""
    torch, ddg, kind, t, h, w, target, weights, space = ops.vocab_case(dtype, tokens, dim, vocab, 0, gone, weighted)
    print(f"case vocab {dtype} {tokens} {dim} {vocab} gone {gone} weighted {weighted}", flush=True)
    scale = torch.exp2(torch.randint(-powers, powers + 1, (dim,), device="cuda", generator=torch.Generator("cuda").manual_seed(7)).float())
    h.mul_(scale)
    w.div_(scale)
    op = ddg.VocabLoss(tokens, dim, vocab, kind)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    f32 = lambda n: space(1, n, dt=torch.float32)  # noqa: E731
    loss, rows, lse, dh, dw = f32(1), f32(tokens), f32(tokens), space(tokens, dim), space(vocab, dim)
    op(h, w, target, weights, loss, rows, lse, dh, dw, workspace=ws)
    wl, wr, we, wdh, wdw = R.vocab(h, w, target, weights)
    assert R.off(loss, wl) <= ops.SUMS and R.off(rows, wr) <= ops.SUMS and R.off(lse, we) <= ops.SUMS
    scale = scale.double()
    assert R.off(dh * scale, wdh * scale) <= grad(dtype, vocab) and R.off(dw / scale, wdw / scale) <= grad(dtype, tokens)
    assert bool((dh[target < 0] == 0).all())


@pytest.mark.parametrize("dtype,size", sorted({(k[0], s) for k in KINDS for s in k[2:]}))
@pytest.mark.parametrize("gone,weighted", [(0.0, False), (0.4, True)])
def test_every_kind_of_launch(dtype, size, gone, weighted):
    check(dtype, *size, gone, weighted)


@pytest.mark.parametrize("size", [s for s, _ in PLANES])
def test_planes_over_60_powers_of_two(size):
    check("f32", *size, 0.3, True, powers=30)


@pytest.mark.parametrize("dtype,tokens,dim,vocab", [("bf16", 700, 16, 1200000), ("f32", 900, 512, 160000)])
@pytest.mark.parametrize("gone", [0.9, 1.0])
@pytest.mark.parametrize("dw_f32", [False, True])
def test_turns_that_no_token_is_left_for(dtype, tokens, dim, vocab, gone, dw_f32):
    """Tokens with a target fill a part of the first turn, or none: the later ones add nothing."""
    torch, ddg, kind, t, h, w, target, weights, space = ops.vocab_case(dtype, tokens, dim, vocab, 0, gone, False)
    if gone == 1:
        target.fill_(-1)
    op = ddg.VocabLoss(tokens, dim, vocab, kind, dw_f32=dw_f32)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    loss, dh, dw = space(1, 1, dt=torch.float32), space(tokens, dim), space(vocab, dim, dt=torch.float32 if dw_f32 else t)
    op(h, w, target, None, loss, None, None, dh, dw, workspace=ws)
    wl, _, _, wdh, wdw = R.vocab(h, w, target)
    assert R.off(loss, wl) <= ops.SUMS and R.off(dh, wdh) <= grad(dtype, vocab) and R.off(dw, wdw) <= grad(dtype, tokens)
