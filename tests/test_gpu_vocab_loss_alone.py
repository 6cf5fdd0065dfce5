"""The vocabulary loss without gradients of many tokens (scoring): one tile, in planes, in several turns, against its definition in 64 bits.

Bounds as in the other tests of this operator: a log-sum over n entries is off by sqrt(n) * 2^-24 at most, 6.5e-5 at 1.2 million, of values of 14 and more: less than 1e-5 of them."""
import pytest

from tests import test_gpu_token_ops as ops
from tests import token_ref as R
from tests.vocab_plan import LOSS_ALONE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,size", [(d, s) for d, s, _ in LOSS_ALONE])
@pytest.mark.parametrize("gone,weighted", [(0.0, False), (0.3, True)])
def test_loss_of_many_tokens_alone(dtype, size, gone, weighted):
    torch, ddg, kind, t, h, w, target, weights, space = ops.vocab_case(dtype, *size, 0, gone, weighted)
    tokens, dim, vocab = size
    print(f"case vocab {dtype} {size} gone {gone} weighted {weighted}", flush=True)
    op = ddg.VocabLoss(tokens, dim, vocab, kind)
    ws = torch.full((op.workspace_bytes(False),), 255, device="cuda", dtype=torch.uint8)
    loss, rows, lse = (space(1, n, dt=torch.float32) for n in (1, tokens, tokens))
    op(h, w, target, weights, loss, rows, lse, workspace=ws)
    there, wide = target >= 0, w.double()
    we, wr = torch.zeros(tokens, device="cuda", dtype=torch.float64), torch.zeros(tokens, device="cuda", dtype=torch.float64)
    for i in range(0, tokens, 1000):
        z = h[i:i + 1000].double() @ wide.T
        we[i:i + 1000] = z.logsumexp(1)
        wr[i:i + 1000] = we[i:i + 1000] - z.gather(1, target[i:i + 1000].long().clamp_min(0)[:, None])[:, 0]
    we, wr = we * there, wr * there
    wl = (wr * weights.double()).sum() if weighted else wr.sum() / there.sum()
    assert R.off(loss, wl) <= ops.SUMS and R.off(rows, wr) <= ops.SUMS and R.off(lse, we) <= ops.SUMS
