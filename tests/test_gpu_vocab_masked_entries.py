"""Entries of the vocabulary that are masked through a column of w (whose h is 1), in runs longer than a tile's columns: by infinity or by the lowest finite value they have
the probability 0 that they have by -30000, exactly, so everything has the same bits; and it is the definition's in 64 bits (bounds as in the other tests of this operator)."""
import pytest

from tests import test_gpu_token_ops as ops
from tests import token_ref as R

pytestmark = pytest.mark.gpu


def masked_case(dtype, tokens, dim, vocab, level):
    """Column 0 of h is 1, of w `level`; returns a function that masks a run of two thirds of the vocabulary, which no target is in, and computes everything."""
    torch, ddg, kind, t, h, w, target, weights, space = ops.vocab_case(dtype, tokens, dim, vocab, 0, 0.1, False)
    lo, hi = vocab // 6, vocab // 6 + 2 * vocab // 3
    h[:, 0], w[:, 0] = 1.0, level
    inside = (target >= lo) & (target < hi)
    target[inside] = hi + target[inside] % (vocab - hi)
    op = ddg.VocabLoss(tokens, dim, vocab, kind)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    f32 = lambda n: space(1, n, dt=torch.float32)  # noqa: E731

    def call(mask):
        w[lo:hi, 0] = torch.finfo(t).min if mask == "lowest" else mask
        out = f32(1), f32(tokens), f32(tokens), space(tokens, dim), space(vocab, dim)
        op(h, w, target, None, *out, workspace=ws)
        return out

    return torch, call, h, w, target


def against_definition(dtype, h, w, target, loss, rows, lse, dh, dw):
    wl, wr, we, wdh, wdw = R.vocab(h, w, target)
    assert R.off(loss, wl) <= ops.SUMS and R.off(rows, wr) <= ops.SUMS and R.off(lse, we) <= ops.SUMS
    assert R.off(dh[:, 1:], wdh[:, 1:]) <= ops.GRAD[dtype] and R.off(dw, wdw) <= ops.GRAD[dtype]


# one tile and several, waves whose columns are all masked, every kind of launch; fp32 on the direct path
INFINITE = [("f32", 20, 64, 100), ("f32", 33, 64, 250), ("f32", 200, 128, 2000), ("bf16", 20, 64, 100), ("bf16", 33, 64, 250), ("bf16", 200, 128, 2000),
            ("bf16", 1021, 776, 10007), ("bf16", 40000, 512, 250)]


@pytest.mark.parametrize("dtype,tokens,dim,vocab", INFINITE)
@pytest.mark.parametrize("level", [0.0, -200.0, 200.0])
def test_entries_masked_by_infinity(dtype, tokens, dim, vocab, level):
    torch, call, h, w, target = masked_case(dtype, tokens, dim, vocab, level)
    finite = call(-30000.0)
    got = call(float("-inf"))
    loss, rows, lse, dh, dw = got
    assert all(torch.equal(a, b) for a, b in zip((loss, rows, lse, dh[:, 1:], dw), (finite[0], finite[1], finite[2], finite[3][:, 1:], finite[4])))
    assert bool(dh[target >= 0, 0].isnan().all())           # a probability of 0 times an entry of -infinity
    if level == 0:
        against_definition(dtype, h, w, target, *got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,dim,vocab", [(20, 64, 100), (200, 128, 2000), (1021, 776, 10007), (40000, 1024, 256)])      # (fp32: the last two in planes)
@pytest.mark.parametrize("level", [0.0, -200.0])
def test_entries_masked_by_the_lowest_value(dtype, tokens, dim, vocab, level):
    torch, call, h, w, target = masked_case(dtype, tokens, dim, vocab, level)
    finite = call(-30000.0)
    got = call("lowest")
    assert all(torch.equal(a, b) for a, b in zip(got, finite))
    if level == 0:
        against_definition(dtype, h, w, target, *got)
