"""The 8-bit output of the join against the 32-bit output of the same operands: q = out / scale, the quotient of 32 bits, rounded to nearest even."""
import pytest

from tests import test_gpu_token_ops as ops
from tests import token_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,pad", [(2048, 4096, 0), (3000, 1001, 3), (40, 20000, 0), (4001, 130, 0)])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_q8_is_the_quotient_rounded(rows, cols, pad, group, p):
    """Millions of quotients, of which some lie a rounding away from a tie. What else a call gives is the 32-bit join's, dropout among it."""
    torch, ddg, kind, t, gen, mk, space = ops.setup("f32")
    ld = cols + pad
    y, res, gain = mk(rows, cols, pad), mk(rows, cols, pad, 2.0), torch.randn(cols, device="cuda", generator=gen)
    y[0].zero_(); res[0].zero_()                                # a row of zeros: the least scale, zeros
    y[1].mul_(2.0 ** 12); res[1].mul_(2.0 ** -12)
    gain[:min(cols, 128)] *= 2.0 ** 10                          # groups far apart
    op = ddg.JoinNorm(rows, cols, kind, eps=1e-5, p=p, seed=ops.SEED, ld_y=ld, ld_residual=ld, ld_x=ld, ld_out=ld, group=group)
    f32 = lambda *s: space(*s, dt=torch.float32)  # noqa: E731
    x, out, rstd = space(rows, cols, pad), space(rows, cols, pad), f32(rows, 1)
    op.forward(y, res, gain, out, x_out=x, rstd=rstd, step=ops.STEP)
    groups = -(-cols // group) if group else 1
    x8, rstd8, scale = space(rows, cols, pad), f32(rows, 1), f32(rows, groups)
    q = torch.full((rows, ld), 0x11, device="cuda", dtype=torch.uint8)
    op.forward_q8(y, res, gain, q, scale, x_out=x8, rstd=rstd8, step=ops.STEP)
    assert torch.equal(x8, x) and torch.equal(rstd8, rstd)
    assert R.off(x, R.join(y, res, gain, 1e-5, p, ops.SEED, ops.STEP)[0]) <= ops.ROUND["f32"]
    wide = torch.nn.functional.pad(out, (0, -cols % (group or cols))).view(rows, groups, -1)
    top = wide.abs().amax(2).double() / 448                      # (a 32-bit product with 1 / 448: two roundings)
    assert bool(((scale.double() - top.clamp_min(2.0 ** -126)).abs() <= 2.0 ** -23 * top).all())
    quotient = (wide.double() / scale.double()[:, :, None]).float()      # (64 bits hold enough that the second rounding is that of the quotient itself)
    want = quotient.clamp(-448, 448).view(rows, -1)[:, :cols].to(torch.float8_e4m3fn)
    assert torch.equal(q[:, :cols], want.view(torch.uint8))
    assert not pad or bool((q[:, cols:] == 0x11).all())
