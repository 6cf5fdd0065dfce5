"""A target past the vocabulary: the loss is NaN, and so is everything that the token reaches, wherever past the vocabulary it is and whichever launches the sizes take."""
import pytest

from tests import test_gpu_token_ops as ops

pytestmark = pytest.mark.gpu

# one tile, several; entries that are whole 16-byte pieces and not; fp32 products in planes (the last)
SIZES = [(20, 64, 100), (20, 64, 104), (200, 128, 2000), (200, 128, 2003), (1500, 700, 15001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,dim,vocab", SIZES)
@pytest.mark.parametrize("past", [0, 1, 5, 70, 1 << 20, None])
def test_target_past_the_vocabulary(dtype, tokens, dim, vocab, past):
    weighted = past in (1, 70)
    torch, ddg, kind, t, h, w, target, weights, space = ops.vocab_case(dtype, tokens, dim, vocab, 0, 0.2, weighted)
    op = ddg.VocabLoss(tokens, dim, vocab, kind)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    f32 = lambda n: space(1, n, dt=torch.float32)  # noqa: E731

    def call():
        out = f32(1), f32(tokens), f32(tokens), space(tokens, dim), space(vocab, dim)
        op(h, w, target, weights, *out, workspace=ws)
        return out

    bad = int((target >= 0).nonzero()[3])
    loss, rows, lse, dh, dw = call()
    target[bad] = 2 ** 31 - 1 if past is None else vocab + past
    loss2, rows2, lse2, dh2, dw2 = call()
    others = torch.arange(tokens, device="cuda") != bad
    assert torch.equal(rows2[0][others], rows[0][others]) and torch.equal(lse2, lse) and torch.equal(dh2[others], dh[others])
    assert bool(loss2.isnan()) and bool(rows2[0][bad].isnan())
    assert bool(dh2[bad].isnan().all()) and bool(dw2.isnan().all())
    assert bool(dw.isfinite().all()) and bool(dh.isfinite().all())
