"""What the workspace query of the vocabulary loss covers (dry runs: no GPU)."""
import itertools

import pytest

import paper_1804_10574_amd as ddg
from tests.test_token_ops_host import A, B, C_, D, E, INVALID, Space, refused


@pytest.mark.parametrize("dtype", [ddg.DDG_F32, ddg.DDG_BF16])
@pytest.mark.parametrize("tokens,dim,vocab", [(1, 64, 100), (64, 128, 5000), (65, 64, 257), (1500, 704, 15000), (40000, 1024, 256), (300, 72, 3000)])
@pytest.mark.parametrize("gradients", [True, False])
def test_room_for_operands_off_16_bytes(dtype, tokens, dim, vocab, gradients):
    """With `unaligned` the query's size is enough wherever h and w lie; without it, for 16-byte pointers, and no larger."""
    def op(unaligned):
        return ddg.VocabLoss(tokens, dim, vocab, dtype, dry_run=True, unaligned=unaligned)

    room, tight = Space(op(True).workspace_bytes(gradients)), Space(op(False).workspace_bytes(gradients))
    size = 4 if dtype == ddg.DDG_F32 else 2
    results = dict(loss=E, dh=D if gradients else None)
    assert tight.nbytes <= room.nbytes <= tight.nbytes + (tokens + vocab) * dim * size + 512
    for off_h, off_w in itertools.product((0, 4, 8), repeat=2):
        op(True)(A + off_h, B + off_w, C_, workspace=room, **results)
    op(False)(A, B, C_, workspace=tight, **results)
    if tight.nbytes < room.nbytes:
        refused(INVALID, "needs a workspace of", op(False), A + 4, B + 4, C_, workspace=tight, **results)


def test_targets_of_another_type_are_refused():
    """torch's and numpy's whole numbers are 64 bits unless asked otherwise: read as 32 they would be other targets."""
    import numpy as np
    import torch
    op = ddg.VocabLoss(8, 64, 100, ddg.DDG_BF16, dry_run=True)
    space = Space(op.workspace_bytes(False))
    for good in (torch.zeros(8, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32), np.zeros(8, np.int32), C_):
        op(A, B, good, loss=E, workspace=space)
    for bad in (torch.zeros(8, dtype=torch.int64), torch.zeros(8), torch.zeros(8, dtype=torch.int16), np.zeros(8, np.int64), np.zeros(8, np.uint32)):
        refused(INVALID, "targets must be int32", op, A, B, bad, loss=E, workspace=space)
    for bad in (torch.zeros(16, dtype=torch.int32)[::2], torch.zeros(2, 5, dtype=torch.int32)[:, 1:], np.zeros(16, np.int32)[::2]):
        refused(INVALID, "targets must be int32, next to each other", op, A, B, bad, loss=E, workspace=space)
