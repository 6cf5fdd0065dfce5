"""What rotary positions, linear attention and the gated join refuse, before any device work, the frequencies of the rotary table and the sizes of workspaces
(dry runs: no GPU)."""
import math

import numpy as np
import pytest

import paper_1804_10574_amd as ddg
from tests import mixing_ref as R
from tests.test_token_ops_host import INVALID, SHAPE, Space, refused

A, B, C_, D, E, F, G, H, I, J, K, L = (4096 + i * (1 << 28) for i in range(12))      # addresses that nothing reads
BF16, F32 = ddg.DDG_BF16, ddg.DDG_F32


# ---- rotary positions ----------------------------------------------------------------------------

def rot(rows=4, heads=2, dim=64, dtype=BF16, **kw):
    return ddg.Rotary(rows, heads, dim, dtype, dry_run=True, **kw)


def test_rotary_refusals():
    rot()(A, B, C_, positions=D)
    rot()(A, A, C_)                                            # in place
    rot(rows=0)(None, None, None)
    for args in ((None, B, C_), (A, None, C_), (A, B, None)):
        refused(INVALID, "null", rot(), *args)
    refused(INVALID, "dtype", rot(dtype=5), A, B, C_)
    refused(SHAPE, "rows", rot(rows=-1), A, B, C_)
    refused(SHAPE, "columns", rot(heads=0), A, B, C_)
    for dim in (0, -2, 1026):
        refused(SHAPE, "a head has", rot(dim=dim), A, B, C_)
    for r in (3, 66, -2):
        refused(SHAPE, "rot", rot(rot=r), A, B, C_)
    refused(SHAPE, "rot", rot(dim=63), A, B, C_)               # (the whole head by default: odd)
    rot(dim=63, rot=62)(A, B, C_)
    refused(SHAPE, "too long", rot(heads=1 << 21, dim=1024), A, B, C_)
    for ld in ("ld_x", "ld_y"):
        refused(SHAPE, ld, rot(**{ld: 127}), A, B, C_)
        refused(SHAPE, ld, rot(**{ld: (1 << 30) + 1}), A, B, C_)
    nan, inf = float("nan"), float("inf")
    for name, values in (("base", (1.0, 0.0, nan, inf)), ("factor", (0.5, nan, inf)), ("context", (-1.0, nan, inf)), ("magnitude", (0.0, -1.0, nan, inf))):
        for v in values:
            refused(INVALID, name, rot(**{name: v}), A, B, C_)
            refused(INVALID, name, rot(**{name: v}).table)
    for low, high in ((2.0, 2.0), (-1.0, 3.0), (5.0, 1.0), (nan, 2.0), (1.0, inf)):
        refused(INVALID, "low", rot(context=4096, low=low, high=high), A, B, C_)
    refused(INVALID, "overlaps", rot(), A, A + 2, C_)
    refused(INVALID, "overlaps", rot(ld_x=128, ld_y=130), A, A, C_)
    refused(INVALID, "y overlaps table", rot(), A, B, B)
    refused(INVALID, "y overlaps positions", rot(), A, B, C_, positions=B)
    refused(INVALID, "aligned", rot(), A, B, C_ + 4)
    refused(INVALID, "aligned", rot(), A + 1, B, C_)
    refused(INVALID, "int32", rot(), A, B, C_, positions=np.zeros(4, np.int64))
    refused(INVALID, "on the device", rot(), A, B, rot().table())
    rot(ld_x=256, ld_y=256)(A, A + 256, C_)                    # queries beside keys


@pytest.mark.parametrize("kw", [dict(), dict(factor=8.0), dict(factor=8.0, context=4096), dict(factor=2.5, context=8192, low=2.0, high=16.0, base=500000.0), dict(rot=2)])
def test_rotary_table(kw):
    """Frequencies in turns: the reference's are good to a few 2^-53 of their value (2^-49 allowed), the table's to half a step, 2^-65 of a turn, 2 pi 2^-65 in
    radians; and by parts between the two ends."""
    op = rot(dim=128, **kw)
    table = op.table()
    want = R.frequencies(kw.get("rot", 128), **{k: v for k, v in kw.items() if k != "rot"})
    assert table.dtype == np.uint64 and len(table) == len(want)
    for t, w in zip(table, want):
        assert abs(int(t) / 2.0 ** 64 * 2 * math.pi - w) <= w * 2.0 ** -49 + 2 * math.pi * 2.0 ** -65
    if kw.get("context"):
        plain = R.frequencies(128, base=kw.get("base", 10000.0))
        ratio = [w / p for w, p in zip(want, plain)]
        assert ratio[0] == 1.0 and abs(ratio[-1] * kw["factor"] - 1) < 1e-12 and any(1 / kw["factor"] + 1e-6 < r < 1 for r in ratio)


@pytest.mark.parametrize("first", [(1 << 48) + 1, -(1 << 48) - 1, (1 << 62), -(1 << 63)])
def test_rotary_refuses_positions_that_the_table_does_not_reach(first):
    """A step of the table times the position has to stay a small part of a turn, and the sum with positions and rows inside 64 bits."""
    refused(INVALID, "first", rot(), A, B, C_, first=first)
    edge = (1 << 48) if first > 0 else -(1 << 48)
    rot()(A, B, C_, first=edge)
    rot()(A, B, C_, positions=D, first=edge)


@pytest.mark.parametrize("dim,kw", [(128, dict()), (1024, dict(base=1.0001, factor=40.0, context=8192, low=0.0, high=0.5)), (80, dict(base=500000.0, factor=2.5)),
                                    (90, dict(base=10.0, factor=1.7, context=4096, low=2.0, high=16.0)), (2, dict())])
def test_rotary_table_is_within_four_steps(dim, kw):
    """Frequencies in 64 digits, low <= high / 2. The table's are formed with 64 bits, 2^-64 relative for each rounding, of at most 0.16 of a turn, 0.16 steps: the power is good to 2^-63 and its
    exponent's rounding is less than another (3), the turn's constant, the quotient and the product (3), the share that is kept: four operations on values up to twice its range (8), and its
    complement, quotient and sum (3): 17 * 0.16 = 2.7, and half a step for the rounding to whole ones."""
    from decimal import Decimal as N, localcontext
    with localcontext() as c:
        c.prec = 64
        pi = N("3.14159265358979323846264338327950288419716939937510582097494459")
        table = rot(dim=dim, **kw).table()
        factor, context, low, high = (N(kw.get(k, v)) for k, v in (("factor", 1.0), ("context", 0), ("low", 1.0), ("high", 32.0)))
        for i, got in enumerate(table):
            theta = (N(kw.get("base", 10000.0)).ln() * -2 * i / dim).exp()
            w = min(N(1), max(N(0), (context * theta / (2 * pi) - low) / (high - low))) if context else N(0)
            assert abs(N(int(got)) - theta * (w + (1 - w) / factor) / (2 * pi) * 2 ** 64) <= 4


# ---- linear attention ----------------------------------------------------------------------------

def lin(rows=64, heads=4, dim_k=32, dim_v=48, dtype=BF16, **kw):
    return ddg.LinearAttention(rows, heads, dim_k, dim_v, dtype, dry_run=True, **kw)


def test_linear_refusals():
    ok = (A, B, C_, D, E)
    lin().forward(*ok)
    lin().forward(*ok, state_in=F, state_out=F)                # in place
    lin(sequences=3).forward(*ok, starts=G)
    lin(rows=0, sequences=2).forward(None, None, None, D, None, state_in=F, state_out=G)
    for miss in range(5):
        args = list(ok)
        args[miss] = None
        refused(INVALID, "null", lin().forward, *args)
    refused(INVALID, "dtype", lin(dtype=4).forward, *ok)
    refused(SHAPE, "rows", lin(rows=-1).forward, *ok)
    refused(SHAPE, "at most", lin(rows=(1 << 23) + 1).forward, *ok)
    refused(SHAPE, "columns", lin(heads=0).forward, *ok)
    refused(SHAPE, "share", lin(kv_heads=3).forward, *ok)
    refused(SHAPE, "share", lin(kv_heads=-1).forward, *ok)
    refused(SHAPE, "share", lin(kv_heads=8).forward, *ok)
    for dims in (dict(dim_k=0), dict(dim_v=0), dict(dim_k=257), dict(dim_v=-4), dict(dim_v=300)):
        refused(SHAPE, "columns", lin(scale=1.0, **dims).forward, *ok)
    refused(SHAPE, "sequences", lin(sequences=0).forward, *ok)
    refused(SHAPE, "slots", lin(slots=-1).forward, *ok)
    refused(SHAPE, "equal sequences", lin(sequences=3).forward, *ok)
    refused(SHAPE, "slots is null", lin(sequences=4, slots=3).forward, *ok, state_in=F)
    lin(sequences=4, slots=3).forward(*ok, state_in=F, slots=G)
    lin(sequences=4, slots=3).forward(*ok)                     # (no states: nothing to place)
    for v in (float("nan"), float("inf")):
        refused(INVALID, "scale", lin(scale=v).forward, *ok)
    for ld in ("ld_q", "ld_k", "ld_v", "ld_o"):
        refused(SHAPE, ld, lin(**{ld: 100}).forward, *ok)
        refused(SHAPE, ld, lin(**{ld: (1 << 30) + 1}).forward, *ok)
    refused(INVALID, "o overlaps q", lin().forward, A, B, C_, D, A)
    refused(INVALID, "o overlaps log_decay", lin().forward, A, B, C_, D, D)
    refused(INVALID, "state_out overlaps state_in", lin().forward, *ok, state_in=F, state_out=F + 4)
    refused(INVALID, "state_out overlaps starts", lin().forward, *ok, starts=G, state_out=G)
    refused(INVALID, "aligned", lin().forward, A + 1, B, C_, D, E)
    refused(INVALID, "aligned", lin().forward, *ok, state_in=F + 2)
    refused(INVALID, "int32", lin().forward, *ok, starts=np.zeros(2, np.int64))
    refused(INVALID, "int32", lin().forward, *ok, slots=np.zeros(1, np.float32))
    refused(SHAPE, "more than a launch holds", lin(rows=1 << 22, sequences=1 << 22, heads=64).forward, *ok)
    wide = 4 * (32 + 32 + 48)                                  # queries, keys and values side by side
    lin(ld_q=wide, ld_k=wide, ld_v=wide).forward(A, A + 256, A + 512, D, E)


def test_linear_workspace():
    short = lin(rows=192)
    assert short.workspace_bytes() == 0 and short.workspace_bytes(True) == 0
    long = lin(rows=1 << 16)
    need, both = long.workspace_bytes(), long.workspace_bytes(True)
    assert need > 0 and both > 0 and need % 256 == 0 and both % 256 == 0
    args = (A, B, C_, D, E)
    long.forward(*args, workspace=Space(need))
    refused(INVALID, "workspace of", long.forward, *args)
    refused(INVALID, "workspace of", long.forward, *args, workspace=Space(min(need, 4096)))
    refused(INVALID, "256-byte", long.forward, *args, workspace=Space(need, (1 << 40) + 16))
    refused(INVALID, "overlaps", long.forward, A, B, C_, D, 1 << 40, workspace=Space(need))
    assert lin(dim_k=300, scale=1.0).workspace_bytes() == 0
    shared = lin(rows=100, kv_heads=2)
    assert shared.workspace_bytes() == 0 and shared.workspace_bytes(True) >= 100 * 4 * (32 + 48) * 4
    refused(INVALID, "workspace of", shared.backward, A, B, C_, D, E, F, G, H)
    shared.backward(A, B, C_, D, E, F, G, H, workspace=Space(shared.workspace_bytes(True)))
    assert max(need, both) < 3.1 * 4 * 32 * 48 * 4 * (1 << 16) / 192 + 4096   # pieces: at most one per 192 rows


@pytest.mark.parametrize("dtype,shortest", [(BF16, 192), (F32, 64)])
@pytest.mark.parametrize("rows,sequences", [(8192, 64), (65536, 512), (4096, 4096), (100000, 65536), (8192, 1), (1000, 5000)])
def test_linear_workspace_does_not_grow_with_sequences(dtype, shortest, rows, sequences):
    """Only sequences longer than a segment need states between segments: there are at most two for every segment of the rows, however many sequences."""
    op = lin(rows=rows, heads=8, dim_k=64, dim_v=96, dtype=dtype, sequences=sequences)
    state = 8 * 64 * 96 * 4
    most = max(2 * rows // shortest, 2) * state + 255
    assert op.workspace_bytes() <= most and op.workspace_bytes(True) <= 3 * most
    need = op.workspace_bytes()
    op.forward(A, B, C_, D, E, starts=G, workspace=Space(need, 1 << 45))


def test_linear_backward_refusals():
    op = lin()
    ok = (A, B, C_, D, E)
    op.backward(*ok, F, G, H)
    op.backward(*ok, dv=H)
    op.backward(*ok, d_state_in=H, d_state_out=I)
    refused(INVALID, "nothing", op.backward, *ok)
    for miss in range(5):
        args = list(ok)
        args[miss] = None
        refused(INVALID, "null", op.backward, *args, dq=F)
    refused(INVALID, "dq overlaps q", op.backward, *ok, dq=A)
    refused(INVALID, "dk overlaps dv", op.backward, *ok, dk=F, dv=F)
    refused(INVALID, "d_state_in overlaps d_state_out", op.backward, *ok, d_state_in=H, d_state_out=H)
    refused(SHAPE, "equal sequences", lin(sequences=5).backward, *ok, dq=F)
    refused(SHAPE, "slots is null", lin(sequences=2, slots=1).backward, *ok, d_state_in=F)


def test_linear_step_refusals():
    op = lin(rows=8)
    op.step(A, B, C_, D, E, state_in=F, state_out=F)
    op.step(A, B, C_, D, E)                                    # no state: the row alone
    lin(rows=0).step(None, None, None, D, None)
    refused(INVALID, "null", op.step, A, B, C_, None, E)
    refused(INVALID, "null", op.step, A, B, C_, D, None)
    refused(SHAPE, "slots is null", lin(rows=8, slots=7).step, A, B, C_, D, E, state_in=F)
    lin(rows=8, slots=7).step(A, B, C_, D, E, state_in=F, slots=G)
    refused(INVALID, "overlaps", op.step, A, B, C_, D, E, state_in=F, state_out=F + 64)
    refused(INVALID, "o overlaps v", op.step, A, B, C_, D, C_)
    refused(INVALID, "int32", op.step, A, B, C_, D, E, slots=np.zeros(8, np.int64))
    refused(SHAPE, "more than a launch holds", lin(rows=1 << 20, heads=64).step, A, B, C_, D, E)
    refused(SHAPE, "rows", lin(rows=-3).step, A, B, C_, D, E)


# ---- the gated join ------------------------------------------------------------------------------

def gated(rows=4, cols=64, dtype=BF16, gate="silu", **kw):
    return ddg.GatedJoin(rows, cols, dtype, gate=gate, dry_run=True, **kw)


def test_gated_refusals():
    ok = (A, B, C_, D, E)
    gated().forward(*ok, x_out=F, out=G, rstd_y=H, rstd_x=I)
    gated().forward(*ok, out=G)
    gated().forward(A, B, None, None, None, x_out=F)
    gated().forward(*ok, x_out=C_)                             # the stream in place
    gated().forward(*ok, x_out=A)
    gated(gate="none").forward(A, None, C_, D, E, out=G)
    gated(rows=0).forward(None, None, None, None, None, out=G)
    refused(INVALID, "nothing", gated().forward, *ok)
    refused(INVALID, "null", gated().forward, None, B, C_, D, E, out=G)
    refused(INVALID, "null", gated().forward, A, None, C_, D, E, out=G)
    refused(INVALID, "gate must", gated, gate="tanh")
    bad = gated()
    bad.desc.gate = 9
    refused(INVALID, "gate must", bad.forward, *ok, out=G)
    refused(INVALID, "eps", gated(eps=0.0).forward, *ok, out=G)
    refused(INVALID, "eps", gated(eps=float("nan")).forward, *ok, out=G)
    refused(INVALID, "finite", gated(scale=float("inf")).forward, *ok, out=G)
    refused(INVALID, "finite", gated(residual_scale=float("nan")).forward, *ok, out=G)
    for cols, group in ((64, 12), (64, 4), (64, 128), (96, 64), (2048, 1024), (64, -8)):
        refused(SHAPE, "group", gated(cols=cols, group=group).forward, *ok, out=G)
    gated(cols=96, group=32).forward(*ok, out=G)
    refused(SHAPE, "at most 8192", gated(cols=8193).forward, *ok, out=G)
    for ld in ("ld_y", "ld_gate", "ld_residual", "ld_x", "ld_out"):
        refused(SHAPE, ld, gated(**{ld: 60}).forward, *ok, out=G)
    refused(INVALID, "out overlaps gate", gated().forward, *ok, out=B)
    refused(INVALID, "x_out overlaps gate", gated().forward, *ok, x_out=B)
    refused(INVALID, "out overlaps y", gated().forward, *ok, out=A)
    refused(INVALID, "x_out overlaps residual", gated(ld_x=72).forward, *ok, x_out=C_)
    refused(INVALID, "rstd_y overlaps rstd_x", gated(group=8).forward, *ok, rstd_y=H, rstd_x=H + 16)
    refused(INVALID, "gate must be aligned", gated(gate="column").forward, A, B + 2, C_, D, E, out=G)
    gated(gate="plain").forward(A, B + 2, C_, D, E, out=G)


def test_gated_backward_refusals():
    op = gated()
    n = op.workspace_bytes()
    space = Space(n)
    ok = (A, B, C_, D, E, F, G)                                # y, rstd_y, gate, x, rstd_x, gain_y, gain_x
    op.backward(*ok, d_out=H, d_x=I, d_residual=J, d_y=K, d_gate=L, d_gain_y=4096 + (12 << 28), d_gain_x=4096 + (13 << 28), workspace=space)
    op.backward(A, B, C_, None, None, F, G, d_x=I, d_y=K)      # no norm after the join: x is not needed
    op.backward(*ok, d_out=H, d_x=I, d_residual=I)             # in place
    refused(INVALID, "nothing", op.backward, *ok, d_out=H)
    refused(INVALID, "both null", op.backward, *ok, d_y=K)
    refused(INVALID, "null", op.backward, None, B, C_, D, E, F, G, d_out=H, d_y=K)
    refused(INVALID, "null", op.backward, A, None, C_, D, E, F, G, d_out=H, d_y=K)
    refused(INVALID, "null", op.backward, A, B, None, D, E, F, G, d_out=H, d_y=K)
    refused(INVALID, "rstd_x", op.backward, A, B, C_, D, None, F, G, d_out=H, d_y=K)
    refused(INVALID, "x and", op.backward, A, B, C_, None, E, F, G, d_out=H, d_y=K)
    refused(INVALID, "no gate", gated(gate="none").backward, *ok, d_out=H, d_gate=L)
    refused(INVALID, "workspace", op.backward, *ok, d_out=H, d_gain_y=K)
    refused(INVALID, "workspace", op.backward, *ok, d_out=H, d_gain_x=K, workspace=Space(n - 1))
    refused(INVALID, "16-byte", op.backward, *ok, d_out=H, d_gain_x=K, workspace=Space(n, (1 << 40) + 8))
    op.backward(*ok, d_out=H, d_gate=K)                        # (a gate of rows is no sum)
    refused(INVALID, "workspace", gated(gate="column").backward, *ok, d_out=H, d_gate=K)
    assert gated(gate="column").workspace_bytes() == n // 2 * 3 and gated(cols=20000).workspace_bytes() == 0
    refused(INVALID, "overlaps", op.backward, *ok, d_out=H, d_residual=J, d_y=J)
    refused(INVALID, "overlaps", op.backward, *ok, d_out=H, d_y=A)
    refused(INVALID, "overlaps", op.backward, *ok, d_out=H, d_gate=C_)


def test_sizes_that_no_index_holds_are_refused():
    big = (1 << 30) + 1
    refused(SHAPE, "at most", rot(rows=big), A, 1 << 45, C_)
    refused(SHAPE, "at most", gated(rows=big, cols=8).forward, A, B, None, None, None, out=1 << 50)
    refused(SHAPE, "ld_gate", gated(ld_gate=big).forward, A, B, C_, D, E, out=G)
    refused(SHAPE, "too many heads", lin(heads=1 << 23).forward, A, B, C_, D, E)


class OnDevice:
    """What the binding asks of a tensor on the device: no GPU is needed to refuse one."""

    is_cuda = True

    def __init__(self, count, size, dtype="torch.int64", contiguous=True):
        self.count, self.size, self.dtype, self.contiguous = count, size, dtype, contiguous

    def data_ptr(self):
        return C_

    def numel(self):
        return self.count

    def element_size(self):
        return self.size

    def is_contiguous(self):
        return self.contiguous

    def stride(self):
        return (1 if self.contiguous else 2,)


def test_rotary_table_on_the_host_or_of_another_kind_is_refused():
    import torch
    op = rot()                                                 # heads of 64: 32 words
    for host in (torch.from_numpy(op.table().view("int64")), op.table(), op.table().view("int64")):
        refused(INVALID, "on the device", op, A, B, host)
    op(A, B, OnDevice(32, 8))
    op(A, B, OnDevice(40, 8, "torch.float64"))                 # (any 8-byte type, longer than needed)
    for other in (OnDevice(32, 4, "torch.float32"), OnDevice(64, 4, "torch.int32"), OnDevice(32, 8, contiguous=False), OnDevice(31, 8)):
        refused(INVALID, "table must be 32 words", op, A, B, other)
    refused(INVALID, "table must be 10 words", rot(rot=20), A, B, OnDevice(9, 8))
    rot(rot=20)(A, B, OnDevice(10, 8))


def test_whole_numbers_on_the_host_or_too_few_are_refused():
    import torch
    few, int32 = OnDevice(3, 4, "torch.int32"), OnDevice(5, 4, "torch.int32")
    for host in (torch.zeros(8, dtype=torch.int32), np.zeros(8, np.int32)):
        refused(INVALID, "positions must be on the device", rot(), A, B, C_, positions=host)
        refused(INVALID, "starts must be on the device", lin(sequences=2).forward, A, B, C_, D, E, starts=host)
        refused(INVALID, "slots must be on the device", lin(sequences=2).forward, A, B, C_, D, E, slots=host)
        refused(INVALID, "starts must be on the device", lin(sequences=2).backward, A, B, C_, D, E, dq=F, starts=host)
        refused(INVALID, "slots must be on the device", lin(sequences=2).backward, A, B, C_, D, E, dq=F, slots=host)
        refused(INVALID, "slots must be on the device", lin(rows=4).step, A, B, C_, D, E, slots=host)
    rot(rows=5)(A, B, D, positions=int32)
    refused(INVALID, "positions must be 4 or more", rot(), A, B, D, positions=few)
    lin(sequences=4).forward(A, B, F, D, E, starts=int32)
    refused(INVALID, "starts must be 4 or more", lin(sequences=3).forward, A, B, F, D, E, starts=few)
    refused(INVALID, "starts must be 4 or more", lin(sequences=3).backward, A, B, F, D, E, dq=G, starts=few)
    refused(INVALID, "slots must be 4 or more", lin(sequences=4).forward, A, B, F, D, E, slots=few)
    refused(INVALID, "slots must be 4 or more", lin(sequences=4).backward, A, B, F, D, E, dq=G, slots=few)
    lin(rows=5, sequences=1).step(A, B, F, D, E, slots=int32)
    refused(INVALID, "slots must be 6 or more", lin(rows=6, sequences=1).step, A, B, F, D, E, slots=int32)
    refused(INVALID, "int32", lin(sequences=2).forward, A, B, F, D, E, starts=OnDevice(5, 8))
    refused(INVALID, "int32", rot(), A, B, D, positions=OnDevice(5, 4, "torch.int32", contiguous=False))
