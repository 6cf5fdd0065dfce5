"""Rotary positions, linear attention with a decay for each head, and the gated join against their definitions in 64 bits.

Bounds (2-norm of the difference over that of the result), from the formats: a bf16 result is rounded once, at most 2^-8 of each element. Linear attention of bf16
operands keeps 16 bits of the products of two rows and of the state as operands: 2^-16 each of the terms, 2^-12 together where they are eight times the result. fp32, and states whatever the operands: sums of n terms in any
order differ by about sqrt(n) 2^-24 of the norm of their terms, 1e-5 up to n = 2^14. Cosines and sines in fp32 are good to 2^-23, products and sum to 2^-24 each: 2^-21."""
import math

import pytest

from tests import mixing_ref as R
from tests.test_gpu_token_ops import setup, untouched
from tests.token_ref import off

pytestmark = pytest.mark.gpu

ROUND = {"bf16": 2.0 ** -8, "f32": 1e-5}
TURN = {"bf16": 2.0 ** -8, "f32": 2.0 ** -21}
MIX = {"bf16": 2.0 ** -8 + 2.0 ** -12, "f32": 1e-5}
SUMS = 1e-5


# ---- rotary positions ----------------------------------------------------------------------------

# rows, heads, columns, turned, pad
TURNED = [(1, 1, 2, 2, 0), (1, 20, 64, 64, 0), (3, 2, 16, 16, 0), (5, 3, 64, 32, 0), (7, 2, 63, 20, 1), (33, 4, 128, 128, 8), (130, 5, 72, 36, 3), (9, 1, 1024, 1024, 0),
          (6, 3, 40, 2, 0), (2, 2, 80, 78, 5), (5000, 3, 64, 64, 0), (20000, 2, 16, 8, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,heads,dim,rot,pad", TURNED)
@pytest.mark.parametrize("interleaved,inverse", [(False, False), (True, False), (False, True), (True, True)])
def test_rotary(dtype, rows, heads, dim, rot, pad, interleaved, inverse):
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    print(f"case rotary {dtype} {rows} {heads}x{dim} rot {rot} +{pad} {interleaved} {inverse}", flush=True)
    ld = heads * dim + pad
    x, y = mk(rows, heads * dim, pad), space(rows, heads * dim, pad)
    kw = dict(factor=4.0, context=2048) if inverse else {}
    op = ddg.Rotary(rows, heads, dim, kind, rot=rot, interleaved=interleaved, magnitude=1.25, ld_x=ld, ld_y=ld, **kw)
    table = torch.from_numpy(op.table().view("int64")).cuda()
    positions = torch.randint(-5, 100000, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    op(x, y, table, positions=positions, first=3, inverse=inverse)
    want = R.rotary(x, heads, dim, rot, [p + 3 for p in positions.tolist()], interleaved, inverse, 1.25, **kw)
    assert off(y, want) <= TURN[dtype]
    still = y.reshape(rows, heads, dim)[..., rot:] if not pad else None
    assert still is None or torch.equal(still, x.reshape(rows, heads, dim)[..., rot:])
    assert untouched(torch, y, pad)
    op(x, x, table, positions=positions, first=3, inverse=inverse)        # in place
    assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rotary_far_positions(dtype):
    """The largest positions, backwards too: the reference's angles are good to 2^31 * 2^-53 of a radian there."""
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    positions = [0, 1, -1, 1 << 20, -(1 << 20) - 1, (1 << 31) - 1, -(1 << 31), 123456789]
    x, y = mk(len(positions), 128), space(len(positions), 128)
    op = ddg.Rotary(len(positions), 2, 64, kind)
    table = torch.from_numpy(op.table().view("int64")).cuda()
    op(x, y, table, positions=torch.tensor(positions, device="cuda", dtype=torch.int32))
    # (the reference's frequencies are good to 2^-52 of their value: at 2^31 radians, 2^-21 of the angle)
    assert off(y, R.rotary(x, 2, 64, 64, positions)) <= TURN[dtype] + 2.0 ** -21
    assert torch.equal(y[0], x[0])                                         # position 0
    far = (1 << 40) + 7                                                    # the first position alone has 64 bits
    op(x, y, table, first=far)
    near = space(len(positions), 128)
    op(x, near, table, first=far - 4)
    assert torch.equal(near.isfinite(), y.isfinite()) and not torch.equal(near, y)


def turned_by_whole_numbers(torch, x, heads, dim, table, positions, inverse):
    """Halves of x turned by position times the table's own fractions of a turn, modulo 2^64, formed exactly on the host."""
    part = [[p * f % (1 << 64) / 2.0 ** 64 for f in table] for p in positions]
    angle = (-2.0 if inverse else 2.0) * math.pi * torch.tensor(part, dtype=torch.float64, device=x.device)[:, None]
    a, b = x.double().reshape(len(positions), heads, 2, dim // 2).unbind(2)
    return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1).reshape(x.shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first,given", [((1 << 40) + 7, False), (-(1 << 40) - 9, False), ((1 << 33) + 1, True), (-(1 << 35) + 3, True), ((1 << 48), False), (-(1 << 48), True),
                                         ((1 << 31) - 2, False), (-(1 << 31) - 2, True)])
def test_rotary_positions_past_32_bits(dtype, first, given):
    """Every angle of first, and of first + positions, against whole numbers: what fp32 makes of an eighth of a turn (2^-28 of a turn, 2^-25 radians) is within TURN."""
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    print(f"case rotary {dtype} first {first} positions {given}", flush=True)
    offsets = [0, 1, -1, (1 << 31) - 1, -(1 << 31), 65537, -12345678] if given else list(range(7))
    rows, heads, dim = len(offsets), 2, 64
    x = mk(rows, heads * dim)
    op = ddg.Rotary(rows, heads, dim, kind)
    host = op.table()
    table = torch.from_numpy(host.view("int64")).cuda()
    positions = torch.tensor(offsets, device="cuda", dtype=torch.int32) if given else None
    for inverse in (False, True):
        y = space(rows, heads * dim)
        op(x, y, table, positions=positions, first=first, inverse=inverse)
        want = turned_by_whole_numbers(torch, x, heads, dim, [int(f) for f in host], [first + p for p in offsets], inverse)
        for r in range(rows):
            assert off(y[r], want[r]) <= TURN[dtype], (r, offsets[r])


def test_rotary_rows_of_two_launches():
    """More rows than a launch takes (2^23): the second launch's positions go on where the first one's end, given or not."""
    torch, ddg, kind, t, gen, mk, space = setup("bf16")
    cut, dim = 1 << 23, 2
    rows, first = cut + 1000, (1 << 40) - 5
    x, y = mk(rows, dim), space(rows, dim)
    op, tail = ddg.Rotary(rows, 1, dim, kind), ddg.Rotary(1000, 1, dim, kind)
    host = op.table()
    table = torch.from_numpy(host.view("int64")).cuda()
    positions = torch.arange(rows, device="cuda", dtype=torch.int32) * 3 - 7
    for p in (None, positions):
        op(x, y, table, positions=p, first=first)
        alone = space(1000, dim)
        tail(x[cut:], alone, table, positions=None if p is None else p[cut:], first=first if p is not None else first + cut)
        assert torch.equal(y[cut:], alone)
        at = list(range(cut - 3, cut + 3)) + [0, 1, rows - 1]
        want = turned_by_whole_numbers(torch, x[at], 1, dim, [int(host[0])], [first + (r if p is None else int(p[r])) for r in at], False)
        assert off(y[at], want) <= TURN["bf16"]


def test_rotary_keeps_scores_relative():
    """Scores of turned queries and keys depend on the distance alone, and the inverse takes a turn back."""
    torch, ddg, kind, t, gen, mk, space = setup("f32")
    rows, dim = 64, 128
    x = mk(1, dim).expand(rows, dim).contiguous()
    y, z = space(rows, dim), space(rows, dim)
    op = ddg.Rotary(rows, 1, dim, kind)
    table = torch.from_numpy(op.table().view("int64")).cuda()
    op(x, y, table, first=1 << 20)
    s = y.double() @ y.double().T
    for d in (1, 7, 30):
        diag = torch.diagonal(s, d)
        assert float((diag - diag[0]).abs().max()) <= 2.0 ** -19 * float(s[0, 0])
    op(y, z, table, first=1 << 20, inverse=True)
    assert off(z, x) <= 2.0 ** -20


# ---- linear attention ----------------------------------------------------------------------------

def mixing(dtype, lengths, heads, kv_heads, dim_k, dim_v, pad=0, behind=0, seed=1, states=False, slots=None):
    torch, ddg, kind, t, gen, mk, space = setup(dtype, seed)
    rows = sum(lengths) + behind

    class Case:
        pass

    c = Case()
    c.torch, c.ddg, c.rows, c.lengths, c.heads, c.kv_heads, c.dim_k, c.dim_v, c.space, c.pad = torch, ddg, rows, lengths, heads, kv_heads, dim_k, dim_v, space, pad
    c.q, c.k, c.v, c.d_o = mk(rows, heads * dim_k, pad), mk(rows, kv_heads * dim_k, pad), mk(rows, kv_heads * dim_v, pad), mk(rows, heads * dim_v, pad)
    # heads that see all, that forget slowly and fast, and one that sees its own row only
    c.lam = torch.tensor([(0.0, -1e-3, -0.05, -0.7, -3.0, float("-inf"), -0.01)[i % 7] for i in range(heads)], device="cuda")
    c.count = max(slots) + 2 if slots else len(lengths)
    c.slots_list = slots
    c.slots = torch.tensor(slots, device="cuda", dtype=torch.int32) if slots else None
    c.starts = torch.tensor([0] + list(lengths), device="cuda").cumsum(0).to(torch.int32)
    c.scale = dim_k ** -0.5
    shape = (c.count, heads, dim_k, dim_v)
    c.states = torch.randn(shape, device="cuda", generator=gen) if states else None
    c.d_states = torch.randn(shape, device="cuda", generator=gen) if states else None
    c.op = ddg.LinearAttention(rows, heads, dim_k, dim_v, kind, sequences=len(lengths), kv_heads=kv_heads, slots=c.count, ld_q=heads * dim_k + pad,
                               ld_k=kv_heads * dim_k + pad, ld_v=kv_heads * dim_v + pad, ld_o=heads * dim_v + pad)
    c.ws = lambda backward=False: torch.full((c.op.workspace_bytes(backward) + 256,), 255, device="cuda", dtype=torch.uint8)      # (NaN in every type)
    c.wide = lambda x, h, d: x[:sum(lengths)].reshape(sum(lengths), h, d)
    return c


def reference(c):
    o, after = R.linear(c.wide(c.q, c.heads, c.dim_k), c.wide(c.k, c.kv_heads, c.dim_k), c.wide(c.v, c.kv_heads, c.dim_v), c.lam, c.lengths, c.scale, c.states, c.slots_list)
    return o.reshape(-1, c.heads * c.dim_v), after


# lengths, heads, heads of keys, columns of keys and values, pad
MIXED = [([1], 1, 1, 1, 1, 0), ([2], 1, 1, 16, 16, 0), ([63], 2, 2, 64, 64, 0), ([64], 2, 1, 64, 64, 0), ([65], 3, 1, 32, 64, 8), ([128], 1, 1, 128, 128, 0),
         ([1, 64, 0, 129, 7], 4, 2, 64, 128, 0), ([0, 0, 3], 2, 2, 40, 72, 3), ([200], 2, 2, 96, 200, 0), ([70, 190], 6, 3, 72, 40, 1), ([130], 1, 1, 256, 256, 0),
         ([100], 7, 7, 8, 136, 0), ([17, 90], 2, 1, 130, 60, 0), ([33], 5, 5, 3, 129, 2), ([4] * 300, 2, 2, 16, 24, 0), ([700], 2, 2, 64, 64, 0),
         ([3000], 2, 1, 64, 128, 0), ([1700, 5, 0, 900], 3, 3, 128, 64, 8), ([2500, 400], 1, 1, 33, 70, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim_k,dim_v,pad", MIXED)
@pytest.mark.parametrize("states", [False, True])
def test_linear_forward(dtype, lengths, heads, kv_heads, dim_k, dim_v, pad, states):
    slots = [(5 * i) % (len(lengths) * 5 - 1) if i != 1 else -1 for i in range(len(lengths))] if states and len(lengths) < 9 else None
    c = mixing(dtype, lengths, heads, kv_heads, dim_k, dim_v, pad, behind=3, states=states, slots=slots)
    print(f"case linear {dtype} {lengths[:6]} {heads}/{kv_heads} {dim_k} {dim_v} +{pad} states {states}", flush=True)
    torch = c.torch
    for x in (c.q, c.k, c.v):
        x[sum(lengths):] = float("nan")                        # behind the last sequence
    o = c.space(c.rows, heads * dim_v, pad)
    after = torch.full_like(c.states, 7.0) if states else None
    c.op.forward(c.q, c.k, c.v, c.lam, o, starts=c.starts, slots=c.slots, state_in=c.states, state_out=after, workspace=c.ws())
    want, want_after = reference(c)
    n = sum(lengths)
    assert off(o[:n], want) <= MIX[dtype]
    assert bool((o[n:] == 7.0).all()) and untouched(torch, o, pad)
    if states:
        used = [s for s in (slots or range(len(lengths))) if s >= 0]
        rest = [s for s in range(c.count) if s not in used]
        assert off(after[used], want_after[used]) <= SUMS
        assert bool((after[rest] == 7.0).all())
        again, o2 = c.states.clone(), c.space(c.rows, heads * dim_v, pad)          # in place, and nothing depends on the order of workgroups
        c.op.forward(c.q, c.k, c.v, c.lam, o2, starts=c.starts, slots=c.slots, state_in=again, state_out=again, workspace=c.ws())
        assert torch.equal(again[used], after[used]) and torch.equal(again[rest], c.states[rest]) and torch.equal(o2, o)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,heads,kv_heads,dim_k,dim_v,pad", MIXED)
@pytest.mark.parametrize("states", [False, True])
def test_linear_backward(dtype, lengths, heads, kv_heads, dim_k, dim_v, pad, states):
    slots = [(5 * i) % (len(lengths) * 5 - 1) if i != 1 else -1 for i in range(len(lengths))] if states and len(lengths) < 9 else None
    c = mixing(dtype, lengths, heads, kv_heads, dim_k, dim_v, pad, behind=2, states=states, slots=slots, seed=2)
    print(f"case linear backward {dtype} {lengths[:6]} {heads}/{kv_heads} {dim_k} {dim_v} +{pad} states {states}", flush=True)
    torch = c.torch
    n = sum(lengths)
    for x in (c.q, c.k, c.v, c.d_o):
        x[n:] = float("nan")
    dq, dk, dv = (c.space(c.rows, h * d, pad) for h, d in ((heads, dim_k), (kv_heads, dim_k), (kv_heads, dim_v)))
    ds = torch.full_like(c.states, 7.0) if states else None
    kw = dict(starts=c.starts, slots=c.slots, state_in=c.states, d_state_out=c.d_states)
    c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, dq, dk, dv, d_state_in=ds, workspace=c.ws(True), **kw)
    wq, wk, wv, ws = R.linear_backward(c.wide(c.q, heads, dim_k), c.wide(c.k, kv_heads, dim_k), c.wide(c.v, kv_heads, dim_v), c.lam, lengths, c.scale,
                                       c.wide(c.d_o, heads, dim_v), c.states, slots, c.d_states) if states else (
        *R.linear_backward(c.wide(c.q, heads, dim_k), c.wide(c.k, kv_heads, dim_k), c.wide(c.v, kv_heads, dim_v), c.lam, lengths, c.scale, c.wide(c.d_o, heads, dim_v)), None)
    for name, got, want in (("dq", dq, wq), ("dk", dk, wk), ("dv", dv, wv)):
        assert off(got[:n], want.reshape(n, -1)) <= MIX[dtype], name
        assert bool((got[n:] == 7.0).all()) and untouched(torch, got, pad), name
    if states:
        used = [s for s in (slots or range(len(lengths))) if s >= 0]
        rest = [s for s in range(c.count) if s not in used]
        assert off(ds[used], ws[used]) <= SUMS and bool((ds[rest] == 7.0).all())
    for which in ("dq", "dk", "dv"):                           # one at a time: the same bits
        one = c.space(*dict(dq=(c.rows, heads * dim_k), dk=(c.rows, kv_heads * dim_k), dv=(c.rows, kv_heads * dim_v))[which], pad)
        c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, **{which: one}, workspace=c.ws(True), **kw)
        assert off(one[:n], dict(dq=dq, dk=dk, dv=dv)[which][:n]) <= MIX[dtype]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", [[90], [800, 0, 70], [1, 2]])
@pytest.mark.parametrize("heads,kv_heads,dim_k,dim_v,pad", [(4, 2, 64, 96, 0), (2, 2, 96, 24, 8), (4, 1, 33, 60, 3), (2, 2, 128, 128, 0), (3, 3, 40, 72, 1)])
def test_linear_gradient_of_the_first_state_alone(dtype, lengths, heads, kv_heads, dim_k, dim_v, pad):
    """The walk has no results but the state: of heads that share keys or not, whole and cut, aligned or not. And the same as beside the other gradients."""
    c = mixing(dtype, lengths, heads, kv_heads, dim_k, dim_v, pad, behind=2, states=True, seed=5)
    print(f"case d_state_in alone {dtype} {lengths} {heads}/{kv_heads} {dim_k} {dim_v} +{pad}", flush=True)
    torch, n = c.torch, sum(lengths)
    for x in (c.q, c.k, c.v, c.d_o):
        x[n:] = float("nan")
    kw = dict(starts=c.starts, state_in=c.states, d_state_out=c.d_states, workspace=c.ws(True))
    alone, beside = torch.full_like(c.states, 7.0), torch.full_like(c.states, 7.0)
    c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, d_state_in=alone, **kw)
    *_, want = R.linear_backward(c.wide(c.q, heads, dim_k), c.wide(c.k, kv_heads, dim_k), c.wide(c.v, kv_heads, dim_v), c.lam, lengths, c.scale, c.wide(c.d_o, heads, dim_v),
                                 c.states, None, c.d_states)
    assert off(alone, want) <= SUMS
    dq, dk, dv = (c.space(c.rows, h * d, pad) for h, d in ((heads, dim_k), (kv_heads, dim_k), (kv_heads, dim_v)))
    c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, dq, dk, dv, d_state_in=beside, **kw)
    assert off(alone, beside) <= SUMS
    c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, d_state_in=beside, **dict(kw, state_in=None, d_state_out=None))      # (linear in d_o and d_state_out; does not read state_in)
    zero = torch.zeros_like(c.states)
    *_, want = R.linear_backward(c.wide(c.q, heads, dim_k), c.wide(c.k, kv_heads, dim_k), c.wide(c.v, kv_heads, dim_v), c.lam, lengths, c.scale, c.wide(c.d_o, heads, dim_v),
                                 zero, None, zero)
    assert off(beside, want) <= SUMS


@pytest.mark.parametrize("dtype,states", [("f32", True), ("f32", False), ("bf16", False)])
@pytest.mark.parametrize("lengths", [[150], [700, 0, 30]])
@pytest.mark.parametrize("heads,kv_heads,dim,pad", [(2, 2, 64, 0), (4, 2, 32, 8), (2, 1, 72, 3), (1, 1, 128, 0)])
def test_linear_gradients_one_at_a_time_have_the_same_bits(dtype, states, lengths, heads, kv_heads, dim, pad):
    """fp32, and bf16 where no state is asked for: the same launches, so the same order of sums (bf16 with d_state_in keeps more of the weighted rows, for all gradients of the call).
    Forward: o with and without the state, in fp32."""
    c = mixing(dtype, lengths, heads, kv_heads, dim, dim, pad, states=states, seed=6)
    torch = c.torch
    shapes = dict(dq=heads * dim, dk=kv_heads * dim, dv=kv_heads * dim)
    kw = dict(starts=c.starts, state_in=c.states, d_state_out=c.d_states, workspace=c.ws(True))
    every = {w: c.space(c.rows, n, pad) for w, n in shapes.items()}
    ds = torch.full_like(c.states, 7.0) if states else None
    c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, **every, d_state_in=ds, **kw)
    for which, n in shapes.items():
        one = c.space(c.rows, n, pad)
        c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, **{which: one}, **kw)
        assert torch.equal(one, every[which]), which
    if states:
        o, p, after = c.space(c.rows, heads * dim, pad), c.space(c.rows, heads * dim, pad), torch.empty_like(c.states)
        c.op.forward(c.q, c.k, c.v, c.lam, o, starts=c.starts, state_in=c.states, state_out=after, workspace=c.ws())
        c.op.forward(c.q, c.k, c.v, c.lam, p, starts=c.starts, state_in=c.states, workspace=c.ws())
        assert torch.equal(o, p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim_k,dim_v,pad", [(64, 96, 0), (96, 24, 8), (128, 256, 0), (250, 60, 1), (16, 192, 0), (32, 48, 0), (30, 34, 5), (128, 64, 1)])
@pytest.mark.parametrize("lengths", [[90], [800, 0, 70]])
def test_linear_gradients_of_keys_and_values_of_unlike_width(dtype, lengths, dim_k, dim_v, pad):
    test_linear_backward(dtype, lengths, 4, 2, dim_k, dim_v, pad, True)


# more sequences than segments, so that states between segments are numbered by rows; long ones next to each other, between short and empty ones, and a row more than whole segments
MANY = [1] * 150 + [500, 0, 401] + [0] * 40 + [2] * 100 + [193, 64, 65, 129, 0, 385] + [1] * 200


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,dim_k,dim_v,pad", [(2, 1, 16, 24, 0), (3, 3, 64, 100, 8)])
def test_linear_many_short_sequences_and_a_few_long(dtype, heads, kv_heads, dim_k, dim_v, pad):
    test_linear_forward(dtype, MANY, heads, kv_heads, dim_k, dim_v, pad, True)
    test_linear_backward(dtype, MANY, heads, kv_heads, dim_k, dim_v, pad, True)
    c = mixing(dtype, MANY, heads, kv_heads, dim_k, dim_v, pad, states=True)
    o, dq = c.space(c.rows, heads * dim_v, pad), c.space(c.rows, heads * dim_k, pad)
    for backward in (False, True):
        need, ws = c.op.workspace_bytes(backward), c.ws(backward)
        if backward:
            c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, dq=dq, starts=c.starts, state_in=c.states, d_state_out=c.d_states, workspace=ws[:need])
        else:
            c.op.forward(c.q, c.k, c.v, c.lam, o, starts=c.starts, state_in=c.states, workspace=ws[:need])
        assert need and bool((ws[need:] == 255).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count", [63, 64, 65, 4097])
def test_linear_finds_its_sequence_among_many(dtype, count):
    """Sequences are searched 64 at a time: one, two and three trips; long ones first, last and at the borders of a trip, empty ones between."""
    lengths = [(0, 1, 1, 2)[i % 4] for i in range(count)]
    for n, length in ((0, 401), (1, 0), (62, 130), (63, 65), (64, 200), (65, 64), (2048, 129), (4095, 330), (4096, 140)):
        if n < count:
            lengths[n] = length
    lengths[-1] = 270
    c = mixing(dtype, lengths, 1, 1, 16, 24, behind=1, states=True)
    o, after = c.space(c.rows, 24), c.torch.full_like(c.states, 7.0)
    c.op.forward(c.q, c.k, c.v, c.lam - 0.02, o, starts=c.starts, state_in=c.states, state_out=after, workspace=c.ws())
    c.lam = c.lam - 0.02
    want, want_after = reference(c)
    assert off(o[:-1], want) <= MIX[dtype] and bool((o[-1] == 7.0).all())
    assert off(after[:count], want_after[:count]) <= SUMS


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_equal_sequences_need_no_starts(dtype):
    c = mixing(dtype, [150, 150, 150], 2, 2, 64, 64, states=True)
    torch = c.torch
    o, p = c.space(450, 128), c.space(450, 128)
    a, b = torch.empty_like(c.states), torch.empty_like(c.states)
    c.op.forward(c.q, c.k, c.v, c.lam, o, state_in=c.states, state_out=a, workspace=c.ws())
    c.op.forward(c.q, c.k, c.v, c.lam, p, starts=c.starts, state_in=c.states, state_out=b, workspace=c.ws())
    assert torch.equal(o, p) and torch.equal(a, b)


def test_linear_starts_out_of_range_stay_inside():
    """Starts that the host cannot check: whatever lies outside the rows is taken as their bound, a sequence that ends before it begins is empty."""
    c = mixing("f32", [100, 0, 60], 2, 2, 16, 16)
    torch = c.torch
    o = c.space(160, 32)
    for starts, lengths in (([-50, 100, 100, 1 << 30], [100, 0, 60]), ([0, 100, 90, 160], None), ([160, 0, 0, 0], None)):
        o.fill_(7.0)
        c.op.forward(c.q, c.k, c.v, c.lam, o, starts=torch.tensor(starts, device="cuda", dtype=torch.int32), workspace=c.ws())
        if lengths:
            assert off(o, reference(c)[0]) <= SUMS
    assert bool((o == 7.0).all())
    c = mixing("f32", [700, 300], 1, 1, 16, 16)                # more than a segment, the starts falling
    o, guard = c.space(1000, 16), c.ws()
    c.op.forward(c.q, c.k, c.v, c.lam, o, starts=torch.tensor([1000, 40, 0], device="cuda", dtype=torch.int32), workspace=guard)
    assert bool((o == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,heads,kv_heads,dim_k,dim_v,pad", [(1, 1, 1, 1, 1, 0), (1, 8, 8, 64, 64, 0), (5, 4, 2, 128, 128, 8), (33, 3, 1, 40, 72, 3), (7, 2, 2, 256, 256, 0),
                                                                 (4, 2, 2, 100, 130, 0), (3, 1, 1, 256, 6, 1), (200, 2, 2, 32, 200, 0)])
@pytest.mark.parametrize("empty", [False, True])
def test_linear_step(dtype, rows, heads, kv_heads, dim_k, dim_v, pad, empty):
    slots = [3 * i + 1 for i in range(rows)] if empty else None
    if empty:
        slots[rows // 2] = -1 if rows > 1 else 1
    c = mixing(dtype, [1] * rows, heads, kv_heads, dim_k, dim_v, pad, states=True, slots=slots)
    print(f"case step {dtype} {rows} {heads}/{kv_heads} {dim_k} {dim_v} +{pad} {empty}", flush=True)
    torch = c.torch
    o, after = c.space(rows, heads * dim_v, pad), torch.full_like(c.states, 7.0)
    c.op.step(c.q, c.k, c.v, c.lam, o, slots=c.slots, state_in=c.states, state_out=after)
    want, want_after = reference(c)
    used = [s for s in (slots or range(rows)) if s >= 0]
    rest = [s for s in range(c.count) if s not in used]
    assert off(o, want) <= ROUND[dtype] and untouched(torch, o, pad)
    assert off(after[used], want_after[used]) <= SUMS and bool((after[rest] == 7.0).all())
    o2, own = c.space(rows, heads * dim_v, pad), c.states.clone()
    c.op.step(c.q, c.k, c.v, c.lam, o2, slots=c.slots, state_in=own, state_out=own)
    assert torch.equal(o2, o) and torch.equal(own[used], after[used]) and torch.equal(own[rest], c.states[rest])
    bare = c.space(rows, heads * dim_v, pad)                   # no state: the row alone
    c.op.step(c.q, c.k, c.v, c.lam, bare)
    c.states = None
    assert off(bare, reference(c)[0]) <= ROUND[dtype]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_prompt_then_tokens_is_one_sequence(dtype):
    """A prompt in two pieces and four tokens one by one against the whole in 64 bits; states go from call to call."""
    c = mixing(dtype, [340], 3, 1, 64, 96, states=False)
    torch, ddg, kind = c.torch, c.ddg, c.ddg.DDG_BF16 if dtype == "bf16" else c.ddg.DDG_F32
    state = torch.zeros((1, 3, 64, 96), device="cuda")
    o = c.space(340, 3 * 96)
    at = 0
    for n in (200, 136, 1, 1, 1, 1):
        op = ddg.LinearAttention(n, 3, 64, 96, kind, kv_heads=1)
        part = [x[at:at + n] for x in (c.q, c.k, c.v)]
        if n > 1:
            ws = torch.empty(op.workspace_bytes() + 1, device="cuda", dtype=torch.uint8)
            op.forward(*part, c.lam, o[at:at + n], state_in=state, state_out=state, workspace=ws)
        else:
            op.step(*part, c.lam, o[at:at + n], state_in=state, state_out=state)
        at += n
    c.states = torch.zeros_like(state)
    want, after = reference(c)
    assert off(o, want) <= MIX[dtype] and off(state, after) <= SUMS


def test_linear_gradients_against_differences():
    """Central differences of f = sum(o d_o) + sum(state_out G) in 64 bits at random directions, ragged, shared keys, through the states."""
    c = mixing("f32", [70, 1, 40], 4, 2, 24, 20, states=True)
    torch = c.torch
    dq, dk, dv = c.space(c.rows, 96), c.space(c.rows, 48), c.space(c.rows, 40)
    ds = torch.empty_like(c.states)
    c.op.backward(c.q, c.k, c.v, c.lam, c.d_o, dq, dk, dv, starts=c.starts, state_in=c.states, d_state_out=c.d_states, d_state_in=ds, workspace=c.ws(True))
    args = [c.q.double(), c.k.double(), c.v.double(), c.states.double()]

    def f(q, k, v, s):
        o, after = R.linear(c.wide(q, 4, 24), c.wide(k, 2, 24), c.wide(v, 2, 20), c.lam, c.lengths, c.scale, s)
        return float((o.reshape(c.rows, -1) * c.d_o.double()).sum() + (after * c.d_states.double()).sum())

    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    for which, grad in enumerate((dq, dk, dv, ds)):
        d = torch.randn(args[which].shape, device="cuda", generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + 1e-5 * d, args[which] - 1e-5 * d
        slope = (f(*up) - f(*down)) / 2e-5
        assert abs(slope - float((grad.double() * d).sum())) <= 1e-5 * float(grad.double().norm() * d.norm())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_nan_keeps_to_its_sequence_and_head(dtype):
    """NaN in keys reaches later rows of its own sequence and heads only; in queries its own row; an infinity in values its own column of these rows."""
    c = mixing(dtype, [100, 200, 50], 4, 2, 64, 64, states=True)
    torch = c.torch
    clean, o = c.space(350, 256), c.space(350, 256)
    run = lambda out: c.op.forward(c.q, c.k, c.v, c.lam, out, starts=c.starts, state_in=c.states, workspace=c.ws())  # noqa: E731
    run(clean)
    c.k[150, 3] = float("nan")                                 # row 50 of sequence 1, heads 0 and 1
    run(o)
    same = torch.ones(350, 4, dtype=torch.bool, device="cuda")
    same[150:300, :2] = False
    assert torch.equal(o.view(350, 4, 64)[same], clean.view(350, 4, 64)[same]) and bool(o.view(350, 4, 64)[150, 0].isnan().all())
    c.k[150, 3] = 0.5
    run(clean)
    c.q[120, 64 + 2] = float("inf")                            # head 1 alone
    run(o)
    same[:] = True
    same[120, 1] = False
    assert torch.equal(o.view(350, 4, 64)[same], clean.view(350, 4, 64)[same]) and not bool(o.view(350, 4, 64)[120, 1].isfinite().any())
    c.q[120, 64 + 2] = 0.5
    run(clean)
    c.v[170, 64 + 5] = float("inf")                            # row 70 of sequence 1, heads 2 and 3, one column
    run(o)
    same[:] = True
    same[164:300, 2:] = False                                  # (its chunk of 64 rows takes another order of sums)
    assert torch.equal(o.view(350, 4, 64)[same], clean.view(350, 4, 64)[same]) and not bool(o.view(350, 4, 64)[170, 2, 5].isfinite())
    assert off(o.view(350, 4, 64)[164:170], clean.view(350, 4, 64)[164:170]) <= MIX[dtype]
    other = [j for j in range(64) if j != 5]
    same[228:] = True
    assert torch.equal(o.view(350, 4, 64)[same][:, other], clean.view(350, 4, 64)[same][:, other])
    assert off(o.view(350, 4, 64)[:, :, other], clean.view(350, 4, 64)[:, :, other]) <= MIX[dtype]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("row", [0, 15, 16, 40, 63, 64, 100])
def test_linear_gradients_of_rows_before_and_after_a_nan(dtype, row):
    """NaN in d_o of a row reaches dq of that row alone, dk and dv of it and of rows before it; NaN in v dq of it and of later rows, and dk of its row alone."""
    c = mixing(dtype, [130], 1, 1, 64, 64)
    torch = c.torch

    def run():
        dq, dk, dv = c.space(130, 64), c.space(130, 64), c.space(130, 64)
        c.op.backward(c.q, c.k, c.v, c.lam - 0.01, c.d_o, dq, dk, dv, workspace=c.ws(True))
        return dq, dk, dv

    bad = lambda t: [i for i in range(130) if not bool(t[i].isfinite().all())]  # noqa: E731
    keep = c.d_o[row].clone()
    c.d_o[row] = float("nan")
    dq, dk, dv = run()
    assert bad(dq) == [row] and bad(dk) == list(range(row + 1)) and bad(dv) == list(range(row + 1))
    c.d_o[row] = keep
    c.v[row] = float("inf")
    dq, dk, dv = run()
    assert bad(dq) == list(range(row, 130)) and bad(dk) == [row] and bad(dv) == []


def test_linear_rows_beyond_32_bits():
    """Rows 2^27 elements apart: offsets pass 2^31 elements and 2^32 bytes."""
    torch, ddg, kind, t, gen, mk, space = setup("bf16")
    ld, rows, heads, dim = 1 << 27, 40, 2, 64
    full = torch.zeros(rows * ld, device="cuda", dtype=torch.bfloat16).view(rows, ld)
    cols = heads * dim
    near = mk(rows, 3 * cols)
    full[:, -4 * cols:-cols] = near
    q, k, v, o = (full[:, ld - (4 - i) * cols:][:, :cols] for i in range(4))
    lam = torch.tensor([-0.01, -0.3], device="cuda")
    ddg.LinearAttention(rows, heads, dim, dim, kind, ld_q=ld, ld_k=ld, ld_v=ld, ld_o=ld).forward(q, k, v, lam, o)
    want, _ = R.linear(*(near[:, i * cols:(i + 1) * cols].reshape(rows, heads, dim) for i in range(3)), lam, [rows], dim ** -0.5)
    assert off(o, want.reshape(rows, cols)) <= MIX["bf16"]
    y = torch.empty((rows, cols), device="cuda", dtype=torch.bfloat16)
    op = ddg.Rotary(rows, heads, dim, kind, ld_x=ld)
    op(q, y, torch.from_numpy(op.table().view("int64")).cuda())
    assert off(y, R.rotary(near[:, :cols].contiguous(), heads, dim, dim, list(range(rows)))) <= TURN["bf16"]
    out = torch.empty((rows, cols), device="cuda", dtype=torch.bfloat16)
    ddg.GatedJoin(rows, cols, kind, gate="silu", ld_y=ld, ld_gate=ld, ld_residual=ld).forward(q, k, v, None, None, out=out)
    near = near.double()
    assert off(out, R.gated(near[:, :cols], "silu", near[:, cols:2 * cols], near[:, 2 * cols:], None, None, 1e-6, 0, 1.0, 1.0)[1]) <= ROUND["bf16"]


# ---- the gated join ------------------------------------------------------------------------------

# rows, columns, group, pad
GATED = [(1, 1, 0, 0), (2, 7, 0, 0), (1, 2048, 128, 0), (5, 64, 8, 0), (9, 512, 512, 0), (4, 520, 8, 8), (3, 1001, 0, 3), (6, 2048, 256, 0), (130, 4096, 64, 0), (3, 8192, 32, 8),
         (2, 8192, 0, 0), (700, 8192, 128, 0), (2, 8001, 0, 1), (600, 4104, 8, 0), (11, 320, 16, 5)]


def gated_case(dtype, rows, cols, pad, gate, plain):
    torch, ddg, kind, t, gen, mk, space = setup(dtype, rows + cols)
    gain = lambda: None if plain else torch.randn(cols, device="cuda", generator=gen)  # noqa: E731
    g = None if gate == "none" else torch.randn(cols, device="cuda", generator=gen) if gate == "column" else mk(rows, cols, pad, 2.0)
    return torch, ddg, kind, mk, space, g, gain(), gain()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,group,pad", GATED)
@pytest.mark.parametrize("gate,plain", [("none", True), ("column", False), ("plain", False), ("sigmoid", False), ("silu", False)])
def test_gated_forward(dtype, rows, cols, group, pad, gate, plain):
    torch, ddg, kind, mk, space, g, gain_y, gain_x = gated_case(dtype, rows, cols, pad, gate, plain)
    print(f"case gated {dtype} {rows}x{cols}+{pad} group {group} {gate}", flush=True)
    ld, parts = cols + pad, cols // group if group else 1
    y, res = mk(rows, cols, pad, 3.0), None if plain else mk(rows, cols, pad, 2.0)
    x, out = space(rows, cols, pad), space(rows, cols, pad)
    ry, rx = space(rows, parts, dt=torch.float32), space(rows, 1, dt=torch.float32)
    op = ddg.GatedJoin(rows, cols, kind, eps=1e-5, gate=gate, group=group, scale=0.7, residual_scale=0.9, ld_y=ld, ld_gate=ld, ld_residual=ld, ld_x=ld, ld_out=ld)
    op.forward(y, g, res, gain_y, gain_x, x_out=x, out=out, rstd_y=ry, rstd_x=rx)
    wx, wo, wy, wr = R.gated(y, gate, g, res, gain_y, gain_x, 1e-5, group, 0.7, 0.9)
    assert off(x, wx) <= ROUND[dtype] and off(out, wo) <= ROUND[dtype] and off(ry, wy) <= SUMS and off(rx, wr) <= SUMS
    assert untouched(torch, x, pad) and untouched(torch, out, pad)
    only = space(rows, cols, pad)
    op.forward(y, g, res, gain_y, gain_x, out=only)
    assert torch.equal(only, out)
    op.forward(y, g, res, gain_y, gain_x, x_out=only)
    assert torch.equal(only, x)
    target = y if res is None else res                         # the stream in place
    op.forward(y, g, res, gain_y, gain_x, x_out=target)
    assert torch.equal(target, x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,group,pad", GATED + [(3000, 96, 32, 0), (1500, 1024, 0, 0)])
@pytest.mark.parametrize("gate,plain", [("none", True), ("column", False), ("plain", False), ("sigmoid", False), ("silu", False)])
def test_gated_backward(dtype, rows, cols, group, pad, gate, plain):
    torch, ddg, kind, mk, space, g, gain_y, gain_x = gated_case(dtype, rows, cols, pad, gate, plain)
    print(f"case gated backward {dtype} {rows}x{cols}+{pad} group {group} {gate}", flush=True)
    ld, parts = cols + pad, cols // group if group else 1
    y, x, d_out, d_x = mk(rows, cols, pad, 3.0), mk(rows, cols, pad, 2.0), mk(rows, cols, pad), None if plain else mk(rows, cols, pad)
    ry = (y.float().reshape(rows, parts, -1).square().mean(2) + 1e-5).rsqrt()
    rx = (x.float().square().mean(1) + 1e-5).rsqrt()
    op = ddg.GatedJoin(rows, cols, kind, eps=1e-5, gate=gate, group=group, scale=0.7, residual_scale=0.9, ld_y=ld, ld_gate=ld, ld_residual=ld, ld_x=ld, ld_out=ld)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    d_res, d_y = space(rows, cols, pad), space(rows, cols, pad)
    d_gate = None if gate == "none" else space(1, cols, dt=torch.float32) if gate == "column" else space(rows, cols, pad)
    dgy, dgx = space(1, cols, dt=torch.float32), space(1, cols, dt=torch.float32)
    op.backward(y, ry, g, x, rx, gain_y, gain_x, d_out=d_out, d_x=d_x, d_residual=d_res, d_y=d_y, d_gate=d_gate, d_gain_y=dgy, d_gain_x=dgx, workspace=ws)
    wr, wy, wg, wgy, wgx = R.gated_backward(y, ry, gate, g, x, rx, gain_y, gain_x, d_out, d_x, group, 0.7, 0.9)
    # one column: its norm is +-1 whatever it is, and a gradient through it is eps times the rest, a difference of nearly equal numbers
    if cols > 1:
        assert off(d_res, wr) <= ROUND[dtype] and off(d_y, wy) <= ROUND[dtype]
        assert d_gate is None or off(d_gate, wg) <= (SUMS if gate == "column" else ROUND[dtype])
        assert off(dgy, wgy) <= SUMS and off(dgx, wgx) <= SUMS
    assert untouched(torch, d_res, pad) and untouched(torch, d_y, pad) and (d_gate is None or gate == "column" or untouched(torch, d_gate, pad))
    one = space(rows, cols, pad)                               # one result at a time: the same bits
    op.backward(y, ry, g, x, rx, gain_y, gain_x, d_out=d_out, d_x=d_x, d_y=one)
    assert torch.equal(one, d_y)
    sums = space(1, cols, dt=torch.float32)
    op.backward(y, ry, g, x, rx, gain_y, gain_x, d_out=d_out, d_x=d_x, d_gain_y=sums, workspace=ws)
    assert torch.equal(sums, dgy)
    if d_x is not None:                                        # no norm behind the join; and the stream's gradient in place
        op.backward(y, ry, g, None, None, gain_y, None, d_x=d_x, d_y=one)
        assert cols == 1 or off(one, R.gated_backward(y, ry, gate, g, None, None, gain_y, None, None, d_x, group, 0.7, 0.9)[1]) <= ROUND[dtype]
        op.backward(y, ry, g, x, rx, gain_y, gain_x, d_out=d_out, d_x=d_x, d_residual=d_x)
        assert torch.equal(d_x, d_res)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["sigmoid", "silu"])
def test_gated_by_gates_that_are_all_but_open_or_closed(dtype, gate):
    """Each element within its own roundings: a gate's distance from 0 or 1 is no difference of rounded numbers."""
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    rows, cols = 7, 96
    y, d_x = mk(rows, cols), mk(rows, cols)
    g = torch.linspace(-24, 24, rows * cols, device="cuda").reshape(rows, cols).to(y.dtype)
    ry = torch.ones((rows, 1), device="cuda")
    op = ddg.GatedJoin(rows, cols, kind, gate=gate)
    d_gate, x = space(rows, cols), space(rows, cols)
    op.backward(y, ry, g, None, None, None, None, d_x=d_x, d_gate=d_gate)
    v, u, a = g.double(), y.double(), d_x.double()
    sig, rest = 1 / (1 + torch.exp(-v)), 1 / (1 + torch.exp(v))
    want = a * u * (sig * rest if gate == "sigmoid" else sig * (1 + v * rest))
    size = (a * u).abs() * (sig * rest if gate == "sigmoid" else sig * (1 + v.abs() * rest))       # of the terms
    # e is off by 2^-23 (2 + |g|) of itself with bf16 rows, |g| <= 24, by a step (2^-23) with fp32; nine more roundings of half a step or a step (1 / x): 36 and 10 steps
    steps = 10 if dtype == "f32" else 36
    assert bool(((d_gate.double() - want).abs() <= (0 if dtype == "f32" else 2.0 ** -8) * want.abs() + steps * 2.0 ** -23 * size).all())
    # forward: x = act(g) y rstd; the sum of 96 squares in 14 roundings of half a step, of which the root keeps half, and the rest of rstd in six
    op.forward(y, g, None, None, None, x_out=x)
    want = (sig if gate == "sigmoid" else v * sig) * u * ((u * u).mean(1, keepdim=True) + 1e-6).rsqrt()
    assert bool(((x.double() - want).abs() <= ((0 if dtype == "f32" else 2.0 ** -8) + (steps + 14) * 2.0 ** -23) * want.abs()).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["none", "column", "plain", "sigmoid", "silu"])
def test_gated_gradients_of_one_column(dtype, gate):
    """The norm of one column is its sign: a gradient through it is what is left of nearly equal terms, so each result is bounded by roundings of its terms, 2^-24 each (gates: 10 steps of
    2^-23 with fp32, 36 with bf16 rows, as above), and by its own one."""
    torch, ddg, kind, mk, space, g, gain_y, gain_x = gated_case(dtype, 37, 1, 0, gate, False)
    rows = 37
    y, x, d_out, d_x = mk(rows, 1, 0, 3.0), mk(rows, 1, 0, 2.0), mk(rows, 1), mk(rows, 1)
    ry, rx = (y.float().square().mean(1) + 1e-5).rsqrt().reshape(rows, 1), (x.float().square().mean(1) + 1e-5).rsqrt()
    op = ddg.GatedJoin(rows, 1, kind, eps=1e-5, gate=gate, scale=0.7, residual_scale=0.9)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    d_res, d_y, dgy, dgx = space(rows, 1), space(rows, 1), space(1, 1, dt=torch.float32), space(1, 1, dt=torch.float32)
    d_gate = None if gate == "none" else space(1, 1, dt=torch.float32) if gate == "column" else space(rows, 1)
    op.backward(y, ry, g, x, rx, gain_y, gain_x, d_out=d_out, d_x=d_x, d_residual=d_res, d_y=d_y, d_gate=d_gate, d_gain_y=dgy, d_gain_x=dgx, workspace=ws)
    wr, wy, wg, wgy, wgx = R.gated_backward(y, ry, gate, g, x, rx, gain_y, gain_x, d_out, d_x, 0, 0.7, 0.9)
    a, r, n = d_out.double(), rx.double().reshape(rows, 1), y.double() * ry.double()
    xhat, w = x.double() * r, (d_out.double() * gain_x.double()).abs()
    t = d_x.double().abs() + r * (w + xhat * xhat * w)                     # sizes of t's terms; ten roundings on the way
    half, turn = 2.0 ** -24, 0.0 if dtype == "f32" else 2.0 ** -8
    if gate == "none":
        act = slope = torch.ones_like(t)
    else:
        act, v = R.gate(gate, g.double()), g.double()
        s, rest = 1 / (1 + torch.exp(-v)), 1 / (1 + torch.exp(v))
        slope = torch.ones_like(act) if gate in ("column", "plain") else s * rest if gate == "sigmoid" else s * (1 + v.abs() * rest)
    gates = 0 if gate in ("none", "column", "plain") else 2 * (10 if dtype == "f32" else 36)
    u = 0.7 * act.abs() * t
    fits = lambda got, want, size, steps: bool(((got.double() - want).abs() <= half * steps * size + (turn + half) * want.abs()).all())  # noqa: E731
    assert fits(d_res, wr, 0.9 * t, 12)
    assert fits(d_y, wy, ry.double() * gain_y.double().abs() * u * (1 + n * n), 20 + gates)
    sums = 37                                                                # (a sum of 37 terms in any order: a rounding of it for each)
    assert fits(dgy, wgy, (u * n.abs()).sum(0), 16 + gates + sums) and fits(dgx, wgx, (a * xhat).abs().sum(0), 4 + sums)
    size = 0.7 * t * (n * gain_y.double()).abs() * slope.abs()
    if gate == "column":
        assert fits(d_gate.reshape(1), wg.reshape(1), size.sum(0), 18 + sums)
    elif gate != "none":
        assert fits(d_gate, wg, size, 18 + gates)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,group,pad", [(1, 64, 8, 0), (33, 1024, 64, 0), (7, 520, 8, 3), (300, 2048, 128, 0), (5, 192, 64, 5), (4, 4104, 8, 0), (9, 1001, 0, 1), (600, 96, 32, 0)])
@pytest.mark.parametrize("gate", ["none", "column", "plain", "sigmoid", "silu"])
def test_gated_norm_without_a_join(dtype, rows, cols, group, pad, gate):
    """The norm behind a block and its gate alone, as before a projection: no residual and no next norm; backward from the gradient of its result."""
    torch, ddg, kind, mk, space, g, gain_y, _ = gated_case(dtype, rows, cols, pad, gate, False)
    print(f"case gated norm alone {dtype} {rows}x{cols}+{pad} group {group} {gate}", flush=True)
    ld, parts = cols + pad, cols // group if group else 1
    y, d = mk(rows, cols, pad, 3.0), mk(rows, cols, pad)
    x, ry = space(rows, cols, pad), space(rows, parts, dt=torch.float32)
    op = ddg.GatedJoin(rows, cols, kind, eps=1e-5, gate=gate, group=group, ld_y=ld, ld_gate=ld, ld_x=ld)
    op.forward(y, g, None, gain_y, None, x_out=x, rstd_y=ry)
    wx, _, wry, _ = R.gated(y, gate, g, None, gain_y, None, 1e-5, group, 1.0, 1.0)
    assert off(x, wx) <= ROUND[dtype] and off(ry, wry) <= SUMS and untouched(torch, x, pad)
    d_y, dgy = space(rows, cols, pad), space(1, cols, dt=torch.float32)
    d_gate = None if gate == "none" else space(1, cols, dt=torch.float32) if gate == "column" else space(rows, cols, pad)
    ws = torch.full((op.workspace_bytes(),), 255, device="cuda", dtype=torch.uint8)
    op.backward(y, ry, g, None, None, gain_y, None, d_x=d, d_y=d_y, d_gate=d_gate, d_gain_y=dgy, workspace=ws)
    _, wy, wg, wgy, _ = R.gated_backward(y, ry, gate, g, None, None, gain_y, None, None, d, group, 1.0, 1.0)
    assert off(d_y, wy) <= ROUND[dtype] and off(dgy, wgy) <= SUMS and untouched(torch, d_y, pad)
    assert d_gate is None or off(d_gate, wg) <= (SUMS if gate == "column" else ROUND[dtype])
    leaf = [y.double(), gain_y.double()] + ([] if g is None else [g.double()])
    for t in leaf:
        t.requires_grad_(True)
    with torch.enable_grad():
        out = R.gated(leaf[0], gate, leaf[2] if g is not None else None, None, leaf[1], None, 1e-5, group, 1.0, 1.0)[0]
        grads = torch.autograd.grad((out * d.double()).sum(), leaf)           # the formulas by automatic differentiation, statistics and all
    for got, want in zip((d_y, dgy, d_gate), grads):
        assert off(got.reshape(want.shape), want) <= (ROUND[dtype] if got.dtype != torch.float32 else SUMS)


@pytest.mark.parametrize("rows", [0, 1])
def test_gated_backward_of_few_rows_writes_the_sums(rows):
    torch, ddg, kind, t, gen, mk, space = setup("f32")
    op = ddg.GatedJoin(rows, 40, kind, gate="column")
    ws = torch.empty(op.workspace_bytes(), device="cuda", dtype=torch.uint8)
    y, d_x, g, ry = mk(rows, 40), mk(rows, 40), mk(1, 40)[0], torch.ones((rows, 1), device="cuda")
    sums = [space(1, 40, dt=torch.float32) for _ in range(3)]
    op.backward(y, ry, g, None, None, None, None, d_x=d_x, d_gate=sums[0], d_gain_y=sums[1], d_gain_x=sums[2], workspace=ws)
    p = (y.double() * d_x.double()).sum(0)
    assert off(sums[0], p) <= SUMS and off(sums[1], p * g.double()) <= SUMS and bool((sums[2] == 0).all())


@pytest.mark.parametrize("gate,group", [("silu", 8), ("sigmoid", 0), ("column", 0), ("plain", 8)])
def test_gated_gradients_against_differences(gate, group):
    """Central differences of f = sum(out c) + sum(x e) in 64 bits by each operand, the statistics those of the operands."""
    torch, ddg, kind, t, gen, mk, space = setup("f32")
    rows, cols, eps = 5, 72, 1e-5
    y, res, c, e = mk(rows, cols), mk(rows, cols), mk(rows, cols), mk(rows, cols)
    g = mk(1, cols)[0].contiguous() if gate == "column" else mk(rows, cols)
    gain_y, gain_x = (torch.randn(cols, device="cuda", generator=gen) for _ in range(2))
    op = ddg.GatedJoin(rows, cols, kind, eps=eps, gate=gate, group=group, scale=0.7, residual_scale=0.9)
    x, out, ry, rx = space(rows, cols), space(rows, cols), space(rows, cols // group if group else 1), space(rows, 1)
    op.forward(y, g, res, gain_y, gain_x, x_out=x, out=out, rstd_y=ry, rstd_x=rx)
    grads = [space(rows, cols), torch.empty_like(g), space(rows, cols), space(1, cols), space(1, cols)]
    ws = torch.empty(op.workspace_bytes(), device="cuda", dtype=torch.uint8)
    op.backward(y, ry, g, x, rx, gain_y, gain_x, d_out=c, d_x=e, d_y=grads[0], d_gate=grads[1], d_residual=grads[2], d_gain_y=grads[3], d_gain_x=grads[4], workspace=ws)
    args = [v.double() for v in (y, g, res, gain_y, gain_x)]

    def f(y, g, res, gain_y, gain_x):
        x, out, _, _ = R.gated(y, gate, g, res, gain_y, gain_x, eps, group, 0.7, 0.9)
        return float((out * c.double()).sum() + (x * e.double()).sum())

    for which, grad in enumerate(grads):
        v = torch.randn(args[which].shape, device="cuda", generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + 1e-5 * v, args[which] - 1e-5 * v
        slope = (f(*up) - f(*down)) / 2e-5
        grad = grad.double().reshape(v.shape)
        assert abs(slope - float((grad * v).sum())) <= 1e-5 * float(grad.norm() * v.norm())


def test_gated_with_infinity_or_nan_keeps_to_its_row():
    torch, ddg, kind, t, gen, mk, space = setup("bf16")
    rows, cols = 6, 256
    y, res, g = mk(rows, cols), mk(rows, cols), mk(rows, cols)
    op = ddg.GatedJoin(rows, cols, kind, gate="silu", group=64)
    clean, out, x = space(rows, cols), space(rows, cols), space(rows, cols)
    op.forward(y, g, res, None, None, out=clean)
    y[1, 3], res[4, 200], g[5, 7] = float("inf"), float("nan"), -100.0
    op.forward(y, g, res, None, None, out=out, x_out=x)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda"); bad[1] = bad[4] = bad[5] = True
    assert torch.equal(out[~bad], clean[~bad]) and bool(out[4].isnan().all()) and bool(x[1, 64:].isfinite().all()) and bool(x[1, 3].isnan())
    assert bool(out[5].isfinite().all())                       # a gate that is shut


# ---- together ------------------------------------------------------------------------------------

def block(torch, ddg, kind, dtype, rows, heads, dim, sequences, stream, inputs, ws):
    """A mixing block: rotary positions of queries and keys, linear attention, norm per head with its gate and the next norm; forward and backward. -> results"""
    cols = heads * dim
    q, k, v, g, res, lam, gain_y, gain_x, table, c, e = inputs
    like = torch.empty_like
    turn = ddg.Rotary(rows, heads, dim, kind, stream=stream)
    mix = ddg.LinearAttention(rows, heads, dim, dim, kind, sequences=sequences, stream=stream)
    join = ddg.GatedJoin(rows, cols, kind, gate="silu", group=dim, stream=stream)
    tq, tk, o, x, out = like(q), like(k), like(v), like(v), like(v)
    ry, rx = torch.empty((rows, heads), device="cuda"), torch.empty(rows, device="cuda")
    turn(q, tq, table)
    turn(k, tk, table)
    mix.forward(tq, tk, v, lam, o, workspace=ws)
    join.forward(o, g, res, gain_y, gain_x, x_out=x, out=out, rstd_y=ry, rstd_x=rx)
    d_o, d_g, d_res, dgy, dgx = like(o), like(g), like(res), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    join.backward(o, ry, g, x, rx, gain_y, gain_x, d_out=c, d_x=e, d_residual=d_res, d_y=d_o, d_gate=d_g, d_gain_y=dgy, d_gain_x=dgx, workspace=ws)
    dtq, dtk, dv, dq, dk = like(q), like(k), like(v), like(q), like(k)
    mix.backward(tq, tk, v, lam, d_o, dtq, dtk, dv, workspace=ws)
    turn(dtq, dq, table, inverse=True)
    turn(dtk, dk, table, inverse=True)
    return x, out, dq, dk, dv, d_g, d_res, dgy, dgx


def block_case(dtype, rows, heads, dim, sequences):
    torch, ddg, kind, t, gen, mk, space = setup(dtype)
    cols = heads * dim
    tensors = [mk(rows, cols) for _ in range(5)]
    lam = -torch.rand(heads, device="cuda", generator=gen) * 0.2
    gains = [1 + 0.1 * torch.randn(cols, device="cuda", generator=gen) for _ in range(2)]
    table = torch.from_numpy(ddg.Rotary(rows, heads, dim, kind).table().view("int64")).cuda()
    need = max(ddg.LinearAttention(rows, heads, dim, dim, kind, sequences=sequences).workspace_bytes(True), ddg.GatedJoin(rows, cols, kind).workspace_bytes())
    ws = torch.full((need,), 255, device="cuda", dtype=torch.uint8)
    return torch, ddg, kind, [*tensors, lam, *gains, table, mk(rows, cols), mk(rows, cols)], ws


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_block_of_all_of_them(dtype):
    """The block against the same block in 64 bits, differentiated automatically. Every step's bf16 result is an operand of the next one: six roundings of 2^-8 lie on the
    longest way (turned queries, products, o, d_y, dq before its turn, dq), with independent signs, and each gradient amplifies them by its own condition, of a few: 2^-4 is
    far below what a wrong term would give, which is of order 1."""
    rows, heads, dim, sequences = 600, 2, 64, 2
    torch, ddg, kind, inputs, ws = block_case(dtype, rows, heads, dim, sequences)
    got = block(torch, ddg, kind, dtype, rows, heads, dim, sequences, None, inputs, ws)
    q, k, v, g, res, lam, gain_y, gain_x, table, c, e = inputs
    leaves = [t.double().requires_grad_(True) for t in (q, k, v, g, res, gain_y, gain_x)]
    theta = torch.tensor(R.frequencies(dim), device="cuda", dtype=torch.float64)
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * theta
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def turned(t):
        a, b = t.reshape(rows, heads, 2, dim // 2).unbind(2)
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)

    o, _ = R.linear(turned(leaves[0]), turned(leaves[1]), leaves[2].reshape(rows, heads, dim), lam, [rows // 2] * 2, dim ** -0.5)
    y = o.reshape(rows, -1, dim)
    u = (y * (y.square().mean(2, keepdim=True) + 1e-6).rsqrt()).reshape(rows, -1) * leaves[5]
    x = leaves[4] + leaves[3] * torch.sigmoid(leaves[3]) * u
    out = x * (x.square().mean(1, keepdim=True) + 1e-6).rsqrt() * leaves[6]
    grads = torch.autograd.grad((out * c.double()).sum() + (x * e.double()).sum(), leaves)
    bound = 2.0 ** -4 if dtype == "bf16" else 1e-4
    for a, b in zip(got, [x, out, *grads]):
        assert off(a, b.detach()) <= bound


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_block_in_a_graph(dtype):
    """Captured on a stream of its own and replayed with other inputs, eager work and waits between: every replay has the eager bits. A second graph shares the workspace."""
    rows, heads, dim, sequences = 1400, 2, 64, 1
    torch, ddg, kind, inputs, ws = block_case(dtype, rows, heads, dim, sequences)
    first = block(torch, ddg, kind, dtype, rows, heads, dim, sequences, None, inputs, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            results = block(torch, ddg, kind, dtype, rows, heads, dim, sequences, torch.cuda.current_stream().cuda_stream, inputs, ws)
        graphs.append((graph, results))
    for turn in range(4):
        for graph, results in graphs:
            graph.replay()
            torch.cuda.synchronize()
            eager = block(torch, ddg, kind, dtype, rows, heads, dim, sequences, None, inputs, ws)
            assert all(torch.equal(a, b) for a, b in zip(results, eager))
        assert turn or all(torch.equal(a, b) for a, b in zip(eager, first))
        for t in inputs[:5]:
            t.add_(0.25)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ragged_prompts_and_tokens_in_a_graph(dtype):
    """A captured pass over ragged prompts, their gradients and a row of every sequence, replayed with other starts, slots and positions in the same tensors: the eager bits every time."""
    torch, ddg, kind, t, gen, mk, space = setup(dtype, 4)
    rows, heads, kv_heads, dim, count, pool = 900, 4, 2, 64, 6, 9
    q, k, v, d_o = mk(rows, heads * dim), mk(rows, kv_heads * dim), mk(rows, kv_heads * dim), mk(rows, heads * dim)
    lam = torch.tensor([-0.01, -0.2, 0.0, -1.0], device="cuda")
    begin = torch.randn((pool, heads, dim, dim), device="cuda", generator=gen)
    starts, slots = (torch.zeros(n, device="cuda", dtype=torch.int32) for n in (count + 1, count))
    positions = torch.zeros(rows, device="cuda", dtype=torch.int32)
    table = torch.from_numpy(ddg.Rotary(rows, heads, dim, kind).table().view("int64")).cuda()
    need = ddg.LinearAttention(rows, heads, dim, dim, kind, sequences=count, kv_heads=kv_heads, slots=pool).workspace_bytes(True)
    ws = torch.full((need,), 255, device="cuda", dtype=torch.uint8)

    def run(stream):
        mix = ddg.LinearAttention(rows, heads, dim, dim, kind, sequences=count, kv_heads=kv_heads, slots=pool, stream=stream)
        one = ddg.LinearAttention(count, heads, dim, dim, kind, kv_heads=kv_heads, slots=pool, stream=stream)
        o, tq, states = torch.zeros_like(d_o), torch.empty_like(q), torch.empty_like(begin)
        dq, dk, dv, ds, token = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(begin), torch.empty((count, heads * dim), device="cuda", dtype=t)
        states.copy_(begin)
        ddg.Rotary(rows, heads, dim, kind, stream=stream)(q, tq, table, positions=positions)
        mix.forward(tq, k, v, lam, o, starts=starts, slots=slots, state_in=states, state_out=states, workspace=ws)
        mix.backward(tq, k, v, lam, d_o, dq, dk, dv, starts=starts, slots=slots, state_in=begin, d_state_in=ds, workspace=ws)
        one.step(q[:count], k[:count], v[:count], lam, token, slots=slots, state_in=states, state_out=states)
        return o, dq, dk, dv, ds, states, token

    turns = [([0, 300, 300, 310, 700, 701, 900], [3, 0, 8, 1, -1, 5]), ([5, 6, 7, 8, 9, 10, 11], [0, 1, 2, 3, 4, 5]), ([0, 0, 0, 900, 900, 900, 900], [8, 7, 6, 5, 4, 3]),
             ([100, 228, 420, 613, 614, 615, 890], [2, 9, 4, 6, 8, 0])]

    def put(turn):
        starts.copy_(torch.tensor(turns[turn][0], dtype=torch.int32))
        slots.copy_(torch.tensor(turns[turn][1], dtype=torch.int32))
        positions.copy_(torch.arange(rows, dtype=torch.int32) * (turn + 1) - 7)

    put(0)
    run(None)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        results = run(torch.cuda.current_stream().cuda_stream)
    for turn in (0, 1, 2, 3, 0):
        put(turn)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = run(None)
        assert all(torch.equal(a, b) for a, b in zip(results, eager)), turn
        begins, named = turns[turn]
        lengths = [b - a for a, b in zip(begins, begins[1:])]
        where = slice(begins[0], begins[-1])
        wide = lambda x, h: x[where].reshape(-1, h, dim)  # noqa: E731
        turned = R.rotary(q, heads, dim, dim, positions.tolist()).to(t)
        want, _ = R.linear(wide(turned, heads), wide(k, kv_heads), wide(v, kv_heads), lam, lengths, dim ** -0.5, begin, named)
        bound = MIX[dtype] if dtype == "f32" else 2 * MIX[dtype]                # (the turned row that is compared with is rounded from 64 bits: some round the other way)
        assert off(results[0][where], want.reshape(-1, heads * dim)) <= bound
        assert bool((results[0][:begins[0]] == 0).all()) and bool((results[0][begins[-1]:] == 0).all())
