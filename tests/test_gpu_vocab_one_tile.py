"""The vocabulary loss of many tokens over a vocabulary that one tile of the products holds (characters, bytes), against its definition in 64 bits.

Bounds as in the other tests of this operator; a sum over n tokens in 32 bits is off by sqrt(n) * 2^-24 of the norm of its terms, 1.6e-5 at 65536 tokens, which gives
dw 2e-5 in fp32."""
import pytest

from tests import test_gpu_token_ops as ops
from tests import token_ref as R
from tests.vocab_plan import ONE_TILE

pytestmark = pytest.mark.gpu

DW = {"bf16": ops.GRAD["bf16"], "f32": 2e-5}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,dim,vocab", ONE_TILE)
@pytest.mark.parametrize("gone,weighted", [(0.0, False), (0.3, True)])
def test_vocab_loss_of_many_tokens_over_one_tile(dtype, tokens, dim, vocab, gone, weighted):
    torch, ddg, kind, t, h, w, target, weights, space = ops.vocab_case(dtype, tokens, dim, vocab, 0, gone, weighted)
    print(f"case vocab {dtype} {tokens} {dim} {vocab} gone {gone} weighted {weighted}", flush=True)
    op = ddg.VocabLoss(tokens, dim, vocab, kind)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)      # (NaN in every type)
    f32 = lambda n: space(1, n, dt=torch.float32)  # noqa: E731
    loss, rows, lse, dh, dw = f32(1), f32(tokens), f32(tokens), space(tokens, dim), space(vocab, dim)
    op(h, w, target, weights, loss, rows, lse, dh, dw, workspace=ws)
    wl, wr, we, wdh, wdw = R.vocab(h, w, target, weights)
    assert R.off(loss, wl) <= ops.SUMS and R.off(rows, wr) <= ops.SUMS and R.off(lse, we) <= ops.SUMS
    assert R.off(dh, wdh) <= ops.GRAD[dtype] and R.off(dw, wdw) <= DW[dtype]
    for only in (dict(dh=space(tokens, dim)), dict(dw=space(vocab, dim))):      # one gradient at a time: the same bits
        ws.fill_(255)
        op(h, w, target, weights, workspace=ws, **only)
        assert torch.equal(*only.values(), dh if "dh" in only else dw)
