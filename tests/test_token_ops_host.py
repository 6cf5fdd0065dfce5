"""What the operators of token models refuse, before any device work, and the sizes of their workspaces (dry runs: no GPU)."""
import pytest

import paper_1804_10574_amd as ddg

A, B, C_, D, E, F, G, H = (4096 + i * (1 << 28) for i in range(8))      # addresses that nothing reads
INVALID, SHAPE = 1, 2


def refused(status, text, call, *args, **kw):
    with pytest.raises(ddg.DDGError) as e:
        call(*args, **kw)
    assert e.value.status == status and text in str(e.value), str(e.value)


def drop(rows=4, cols=64, dtype=ddg.DDG_BF16, p=0.5, **kw):
    return ddg.Dropout(rows, cols, dtype, p=p, dry_run=True, **kw)


def test_dropout_refusals():
    drop()(A, B)
    drop()(A, A)                                             # in place
    drop(rows=0)(None, None)
    refused(INVALID, "null", drop(), None, B)
    refused(INVALID, "null", drop(), A, None)
    refused(INVALID, "dtype", drop(dtype=7), A, B)
    refused(SHAPE, "rows", drop(rows=-1), A, B)
    refused(SHAPE, "columns", drop(cols=0), A, B)
    for p in (-0.1, 1.0, 1.5, float("nan")):
        refused(INVALID, "p must", drop(p=p), A, B)
    refused(SHAPE, "ld_x", drop(ld_x=63), A, B)
    refused(SHAPE, "ld_y", drop(ld_y=-64), A, B)
    refused(INVALID, "aligned", drop(), A + 1, B)
    refused(INVALID, "overlaps", drop(), A, A + 2)
    refused(INVALID, "overlaps", drop(ld_x=64, ld_y=72), A, A)
    drop(ld_x=128, ld_y=128)(A, A + 128)                     # the two halves of one tensor's rows
    refused(INVALID, "overlaps", drop(ld_x=128, ld_y=128), A, A + 126)
    drop(ld_x=128, ld_y=128)(A + 128, A)


def join(rows=4, cols=64, dtype=ddg.DDG_BF16, **kw):
    return ddg.JoinNorm(rows, cols, dtype, dry_run=True, **kw)


def test_join_refusals():
    ok = dict(x_out=D, rstd=E)
    join().forward(A, B, C_, F, **ok)
    join().forward(A, None, None, F)
    join().forward(A, B, C_, F, x_out=B)                     # the stream in place
    join().forward(A, B, C_, F, x_out=A)
    join(rows=0).forward(None, None, None, None)
    refused(INVALID, "null", join().forward, None, B, C_, F)
    refused(INVALID, "null", join().forward, A, B, C_, None)
    refused(INVALID, "eps", join(eps=0.0).forward, A, B, C_, F)
    refused(INVALID, "eps", join(eps=float("nan")).forward, A, B, C_, F)
    refused(INVALID, "p must", join(p=1.0).forward, A, B, C_, F)
    refused(INVALID, "group", join(group=64).forward, A, B, C_, F)
    refused(SHAPE, "at most 32768", join(cols=32769).forward, A, B, C_, F)
    for ld in ("ld_y", "ld_residual", "ld_x", "ld_out"):
        refused(SHAPE, ld, join(**{ld: 60}).forward, A, B, C_, F)
    refused(INVALID, "out overlaps y", join().forward, A, B, C_, A)
    refused(INVALID, "x_out overlaps residual", join(ld_x=72).forward, A, B, C_, F, x_out=B)
    refused(INVALID, "out overlaps rstd", join().forward, A, B, C_, F, rstd=F)
    refused(INVALID, "gain must be aligned", join().forward, A, B, C_ + 2, F)
    join().forward_q8(A, B, C_, F, E)
    refused(INVALID, "null", join().forward_q8, A, B, C_, F, None)
    refused(INVALID, "null", join().forward_q8, A, B, C_, None, E)
    refused(INVALID, "q overlaps scale", join().forward_q8, A, B, C_, F, F + 4)


def test_join_backward_refusals():
    op = join()
    n = op.workspace_bytes()
    assert n >= 64 * 4
    import numpy as np
    space = np.empty(n + 64, np.uint8)
    space = space[-space.ctypes.data % 16:][:n]
    op.backward(A, B, C_, D, E, F, G, H, workspace=space)
    op.backward(A, B, None, D, d_y=G)
    op.backward(A, B, C_, D, E, d_residual=E)                # in place
    refused(INVALID, "nothing", op.backward, A, B, C_, D, E)
    for miss in range(3):
        args = [A, B, C_, D]
        args[(0, 1, 3)[miss]] = None
        refused(INVALID, "null", op.backward, *args, d_y=G)
    refused(INVALID, "workspace", op.backward, A, B, C_, D, d_gain=H)
    refused(INVALID, "workspace", op.backward, A, B, C_, D, d_gain=H, workspace=space[:-1])
    refused(INVALID, "overlaps", op.backward, A, B, C_, D, d_residual=F, d_y=F)
    refused(INVALID, "overlaps", op.backward, A, B, C_, D, d_residual=A)
    refused(INVALID, "overlaps", op.backward, A, B, C_, D, d_gain=C_, workspace=space)
    assert join(cols=40000).workspace_bytes() == 0


def loss(tokens=8, dim=64, vocab=100, dtype=ddg.DDG_BF16, **kw):
    return ddg.VocabLoss(tokens, dim, vocab, dtype, dry_run=True, **kw)


class Space:                                                 # a workspace that nothing touches
    def __init__(self, n, at=1 << 40):
        self.nbytes, self.at = n, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.nbytes

    def element_size(self):
        return 1


def test_vocab_refusals():
    op = loss()
    full, alone = Space(op.workspace_bytes()), Space(op.workspace_bytes(False))
    assert alone.nbytes < full.nbytes
    op(A, B, C_, D, E, F, G, H, 4096 + (8 << 28), workspace=full)
    op(A, B, C_, loss=E, workspace=alone)
    refused(INVALID, "null", op, None, B, C_, loss=E, workspace=alone)
    refused(INVALID, "null", op, A, None, C_, loss=E, workspace=alone)
    refused(INVALID, "null", op, A, B, None, loss=E, workspace=alone)
    refused(INVALID, "nothing", op, A, B, C_, workspace=alone)
    refused(INVALID, "workspace", op, A, B, C_, loss=E)
    refused(INVALID, "workspace", op, A, B, C_, dh=H, workspace=alone)
    refused(INVALID, "256-byte", op, A, B, C_, loss=E, workspace=Space(alone.nbytes, (1 << 40) + 128))
    refused(INVALID, "overlaps", op, A, B, C_, dh=A, workspace=full)
    refused(INVALID, "overlaps", op, A, B, C_, dw=B, workspace=full)
    refused(INVALID, "loss overlaps row_loss", op, A, B, C_, loss=E, row_loss=E, workspace=alone)
    refused(INVALID, "overlaps workspace", op, A, B, C_, loss=1 << 40, workspace=alone)
    refused(INVALID, "dtype", loss(dtype=3), A, B, C_, loss=E, workspace=alone)
    refused(SHAPE, "vocab", loss(vocab=0), A, B, C_, loss=E, workspace=alone)
    refused(SHAPE, "columns", loss(dim=0), A, B, C_, loss=E, workspace=alone)
    refused(SHAPE, "rows", loss(tokens=-1), A, B, C_, loss=E, workspace=alone)
    for ld in ("ld_h", "ld_w", "ld_dh", "ld_dw"):
        refused(SHAPE, ld, loss(**{ld: 63}), A, B, C_, loss=E, workspace=alone)
    refused(SHAPE, "at most", loss(vocab=1 << 22), A, B, C_, loss=E, workspace=alone)
    assert loss(vocab=1 << 22).workspace_bytes() == 0
    loss(tokens=0)(None, B, None, loss=E, workspace=Space(max(256, loss(tokens=0).workspace_bytes())))
    # a pointer off its 16 bytes needs room for a copy, which the call names
    refused(INVALID, "needs a workspace of", op, A, B + 2, C_, loss=E, workspace=alone)


def test_vocab_workspace_is_bounded():
    """What is kept of the probabilities does not grow with the tokens beyond 1 GiB."""
    dims = dict(dim=1024, vocab=131072)
    size = [loss(tokens=t, **dims).workspace_bytes() for t in (1024, 4096, 65536, 262144)]
    own = [t * (1024 * 2 + 20) for t in (1024, 4096, 65536, 262144)]                 # gathered hidden states and words of the tokens
    rest = [s - o for s, o in zip(size, own)]
    assert rest[0] < rest[1] < 2.1 * 2 ** 30 and rest[3] < rest[1] + 131072 * 1024 * 4 + (1 << 28)
    assert loss(tokens=4096, **dims).workspace_bytes() < 4096 * 131072 * 4


def test_sizes_that_no_index_holds_are_refused():
    big = (1 << 30) + 1
    refused(SHAPE, "at most", drop(rows=big, cols=1), A, 1 << 45)
    refused(SHAPE, "at most", join(rows=big, cols=1).forward, A, 1 << 45, None, 1 << 46)
    refused(SHAPE, "at most", loss(tokens=big), A, B, C_, loss=E, workspace=Space(1 << 60))
    for ld in ("ld_x", "ld_y"):
        refused(SHAPE, ld, drop(**{ld: big}), A, 1 << 45)
    refused(SHAPE, "ld_dw", loss(ld_dw=1 << 62), A, B, C_, loss=E, workspace=Space(1 << 60))
    drop(rows=1 << 30, cols=1, ld_x=1 << 30, ld_y=1 << 30)(4096, 1 << 62)


def test_more_tokens_than_a_launch_holds_are_refused():
    refused(SHAPE, "tokens", loss(tokens=(1 << 23) + 1), A, B, C_, loss=E, workspace=Space(1 << 60))
    assert loss(tokens=(1 << 23) + 1).workspace_bytes() == 0
    assert loss(tokens=1 << 23).workspace_bytes() > 0
