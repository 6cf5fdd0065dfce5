"""The vocabulary loss of operands off 16 bytes in a workspace of the size that the query gives for them, against its definition in 64 bits."""
import pytest

from tests import test_gpu_token_ops as ops
from tests import token_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,dim,vocab", [(5, 64, 333), (40, 64, 333), (300, 512, 3000)])
def test_vocab_loss_of_operands_off_16_bytes(dtype, tokens, dim, vocab):
    torch, ddg, kind, t, h, w, target, weights, space = ops.vocab_case(dtype, tokens, dim, vocab, 0, 0.2, True, shift=1)
    assert h.data_ptr() % 16 and w.data_ptr() % 16
    op = ddg.VocabLoss(tokens, dim, vocab, kind, unaligned=True)
    loss, dh, dw = space(1, 1, dt=torch.float32), space(tokens, dim), space(vocab, dim)
    op(h, w, target, weights, loss, dh=dh, dw=dw, workspace=torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8))
    wl, _, _, wdh, wdw = R.vocab(h, w, target, weights)
    assert R.off(loss, wl) <= ops.SUMS and R.off(dh, wdh) <= ops.GRAD[dtype] and R.off(dw, wdw) <= ops.GRAD[dtype]
    alone = space(1, 1, dt=torch.float32)
    op(h, w, target, weights, alone, workspace=torch.full((op.workspace_bytes(False),), 255, device="cuda", dtype=torch.uint8))
    assert R.off(alone, wl) <= ops.SUMS
