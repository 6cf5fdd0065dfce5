"""What vocab_plan() may choose, whatever the sizes, and which path the sizes of the GPU tests take (on the host, no GPU)."""
import itertools
import random

import pytest

from tests.vocab_plan import DEEP, FEW, HALF, KINDS, LARGE, LOSS_ALONE, MEDIUM, ONE_TILE, PLANES, ROWS, SHORT, SMALL, kinds, vocab_plan

PANEL_BYTES = (1 << 30) + (1 << 24)


def check(dtype, tokens, dim, vocab, grads, dw_f32):
    p = vocab_plan(dtype, tokens, dim, vocab, grads, dw_f32)
    size = 2 if dtype == "bf16" else 4
    where = (dtype, tokens, dim, vocab, grads, dw_f32)
    # the planes of P are written by the pass over its rows, which a vocabulary of one finished tile does without
    assert not (p.planes and p.whole and grads), where
    assert not (p.planes and dtype == "bf16") and (not p.planes or p.pack_h and p.pack_w), where
    assert not p.whole or vocab <= ROWS[p.cfg_z], where
    # tiles that have a kernel: fp32 has the largest in planes only, and those no other
    if dtype == "f32":
        assert (p.cfg_z == LARGE) == p.planes, where
    assert p.cfg_z in (LARGE, MEDIUM, SMALL, HALF, FEW, DEEP), where
    if grads:
        assert p.cfg_dh in (LARGE, MEDIUM, SMALL, HALF, FEW) and p.cfg_dw in (LARGE, MEDIUM, SHORT, SMALL), where
        assert not p.pair or (p.cfg_dh == p.cfg_dw and p.cfg_dh in (LARGE, MEDIUM, SMALL) and p.panels == 1), where
        assert dtype == "bf16" or (p.cfg_dh == LARGE) == (p.cfg_dw == LARGE) == p.planes, where
        assert p.splits_dw == 1 or p.panels == 1, where
        assert p.acc == (p.panels > 1 and dtype == "bf16" and not dw_f32), where
    # panels cover the tokens, columns of statistics the vocabulary
    assert p.panels >= 1 and p.panel * p.panels >= tokens > p.panel * (p.panels - 1) or tokens == 0, where
    assert p.stats * p.stat_cols >= vocab and p.ld_p >= vocab + 64 and p.dim_p >= dim, where
    assert p.panel <= 256 or not grads or p.panel * p.ld_p * (10 if p.planes else size) <= PANEL_BYTES, where
    # the parts of the workspace, in order, each with room for what goes there
    wide = (dim + 3) // 4 * 4
    need = [(p.o_scalar, 256), (p.o_row, tokens * 16), (p.o_zt, tokens * 4), (p.o_stat, p.panel * p.stats * 8)]
    if grads:
        need += [(p.o_p, p.panel * p.ld_p * size)] + ([(p.o_planes, p.panel * p.ld_p * 6)] if p.planes else [])
        need += [(p.o_part, p.splits * p.panel * wide * 4 if p.splits > 1 else 0), (p.o_part_dw, p.splits_dw * vocab * wide * 4 if p.splits_dw > 1 else 0)]
        need += [(p.o_acc, vocab * wide * 4)] if p.acc else []
    need += [(p.o_h, tokens * p.dim_p * (6 if p.planes else size))] if p.pack_h else []
    need += [(p.o_w, vocab * p.dim_p * (6 if p.planes else size))] if p.pack_w else []
    for (at, n), (after, _) in zip(need, need[1:] + [(p.bytes, 0)]):
        assert at % 256 == 0 and at + n <= after < at + n + 256, where
    assert 1 <= p.splits <= 64 and 1 <= p.splits_dw <= 64 and p.stat_cols in (32, 64, 128), where


SIZES = [1, 2, 31, 64, 65, 193, 256, 257, 1021, 4096, 10007, 40000, 65536, 131072]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("grads,dw_f32", [(True, False), (True, True), (False, False)])
def test_every_plan_holds_together(dtype, grads, dw_f32):
    for tokens, vocab in itertools.product([0] + SIZES, SIZES):
        for dim in (1, 16, 100, 512, 777, 1024, 4096):
            check(dtype, tokens, dim, vocab, grads, dw_f32)
    rng = random.Random(5)
    for _ in range(20000):
        tokens, dim, vocab = (round(most ** rng.random()) for most in (1 << 23, 1 << 14, 1 << 20))
        check(dtype, tokens, dim, vocab, grads, dw_f32)


@pytest.mark.parametrize("tokens,dim,vocab", ONE_TILE)
def test_long_products_over_one_tile_are_in_planes(tokens, dim, vocab):
    p = vocab_plan("f32", tokens, dim, vocab)
    assert p.planes and not p.whole and p.cfg_z == LARGE
    assert vocab_plan("bf16", tokens, dim, vocab).whole


@pytest.mark.parametrize("dtype,kind,sizes", [(k[0], k[1], k[2:]) for k in KINDS])
def test_sizes_take_the_launches_that_they_are_listed_for(dtype, kind, sizes):
    assert all(kind in kinds(vocab_plan(dtype, *s)) for s in sizes)
    assert sorted(s[1] % 8 == 0 for s in sizes) == [False, True]


def test_every_kind_of_launch_is_listed():
    """Of 100000 plans up to the sizes of a training minibatch none has launches that KINDS lacks."""
    listed, rng = {k[:2] for k in KINDS}, random.Random(11)
    for _ in range(50000):
        size = [round(low * (most / low) ** rng.random()) for low, most in ((20, 20000), (16, 8192), (20, 200000))]
        for dtype in ("f32", "bf16"):
            p = vocab_plan(dtype, *size)
            missing = {(dtype, k) for k in kinds(p)} - listed
            assert not missing, (size, missing)


@pytest.mark.parametrize("size,expected", PLANES)
def test_sizes_of_the_planes(size, expected):
    p = vocab_plan("f32", *size)
    assert {k: getattr(p, k) for k in expected} == expected and p.planes == expected.get("planes", True)


@pytest.mark.parametrize("dtype,size,expected", LOSS_ALONE)
def test_sizes_of_the_loss_alone(dtype, size, expected):
    p = vocab_plan(dtype, *size, grads=False)
    assert {k: getattr(p, k) for k in expected} == expected


def test_sizes_of_gradients_in_one_launch():
    """What the tests of gradients in one launch are for: all of their sizes take one, and each type all three tiles, with parts and without."""
    from tests.test_gpu_token_ops import TOGETHER
    for dtype in ("f32", "bf16"):
        plans = [vocab_plan(dtype, *t[:3]) for t in TOGETHER]
        assert all(p.pair for p in plans) and {p.cfg_dh for p in plans} >= ({LARGE, SMALL, MEDIUM})
        assert {p.splits > 1 for p in plans} == {False, True}
