"""Plans of rotary positions, and the calls that are refused before a GPU is touched."""
import ctypes as C
import math
import threading

import pytest
import torch

from paper_2605_11335_amd import binding as B


def test_plan_has_the_angles_of_the_definition():
    r = B.cf_rope_plan(128, [22, 21, 20], [10000.0, 256.0, 1.0])
    assert (r.head_dim, r.n_axes, r.n_pairs) == (128, 3, 63)
    p = 0
    for axis, (pairs, theta) in enumerate(((22, 10000.0), (21, 256.0), (20, 1.0))):
        for j in range(pairs):
            assert r.axis[p] == axis
            # the reference is a double: half a step of a value below 1 / 2 pi < 2^-2 is 2^-55, of pow and of the division one each
            assert abs(r.turn[p] * 2.0 ** -64 - theta ** (-j / pairs) / (2 * math.pi)) <= 4 * 2.0 ** -55
            p += 1
    assert r.turn[63] == 0 and r.axis[63] == 0


@pytest.mark.parametrize("args", [(96, [4]), (128, [65]), (128, []), (64, [6] * 5), (64, [0]), (64, [20, 13]), (64, [8], 0.5), (64, [8], math.inf),
                                  (64, [8], math.nan), (64, [8], [1e4, 1e4]), (64, [-1])])
def test_plans_that_are_refused(args):
    with pytest.raises(B.ChunkflowError) as e:
        B.cf_rope_plan(*args)
    assert e.value.code == B.CF_ERR_ARG and str(e.value)


HERE = 1 << 20          # a made-up aligned address: these calls are refused before anything is read


def operand(x=HERE, y=HERE * 64, x_row=256, x_head=128, y_row=256, y_head=128, heads=2):
    return B.cf_rope_operand(x, y, x_row, x_head, y_row, y_head, heads, 0)


def apply_code(*ops, rope=None, pos=HERE * 128, n=5, n_ops=None, dtype=B.CF_BF16):
    rope = B.cf_rope_plan(128, [64]) if rope is None else rope
    arr = (B.cf_rope_operand * 2)(*ops)
    return B.lib().cf_rope_apply(C.byref(rope), pos, n, arr, len(ops) if n_ops is None else n_ops, dtype, 0, None)


@pytest.mark.parametrize("what", [
    dict(ops=[operand()], dtype=2), dict(ops=[operand()], n=-1), dict(ops=[operand()], pos=None), dict(ops=[operand()], pos=HERE + 2),
    dict(ops=[operand()], n_ops=0), dict(ops=[operand()], n_ops=3), dict(ops=[operand()], rope=B.cf_rope()),
    dict(ops=[operand(x=None)]), dict(ops=[operand(y=None)]), dict(ops=[operand(heads=0)]),
    dict(ops=[operand(x=HERE + 8)]), dict(ops=[operand(y=HERE * 64 + 2)]), dict(ops=[operand(x_row=257)]), dict(ops=[operand(x_head=-128)]),
    dict(ops=[operand(y_head=64)]), dict(ops=[operand(y_row=128)]), dict(ops=[operand(y_row=0)]),          # outputs over one another
    dict(ops=[operand(y=HERE + 256)]), dict(ops=[operand(y=HERE, y_row=512)]),                             # half over the input
    dict(ops=[operand(), operand(x=HERE * 2)]),                                                            # one output for both
    dict(ops=[operand(), operand(x=HERE * 64, y=HERE * 90)]),                                              # an output over the other's input
    dict(ops=[operand(x=HERE * 64, x_row=384, y_row=384), operand(x=HERE * 64 + 256, y=HERE * 64 + 256, x_row=384, y_row=384)])])      # columns that meet
def test_rotations_that_are_refused(what):
    ops = what.pop("ops")
    assert apply_code(*ops, **what) == B.CF_ERR_ARG
    assert b"rope_apply" in B.lib().cf_last_error(None)


def test_no_rows_are_no_work():
    assert apply_code(operand(), n=0) == B.CF_OK
    rope = B.cf_rope_plan(64, [32])
    assert B.lib().cf_rope_tables(C.byref(rope), None, 0, None, None, None) == B.CF_OK


@pytest.mark.parametrize("args", [(None, HERE, HERE * 2), (HERE, None, HERE * 2), (HERE, HERE * 2, None), (HERE, HERE * 2 + 4, HERE * 3), (HERE + 1, HERE * 2, HERE * 3),
                                  (HERE, HERE * 2, HERE * 2 + 64), (HERE, HERE, HERE * 3)])
def test_tables_that_are_refused(args):
    rope = B.cf_rope_plan(64, [32])
    assert B.lib().cf_rope_tables(C.byref(rope), args[0], 10, args[1], args[2], None) == B.CF_ERR_ARG
    assert b"rope_tables" in B.lib().cf_last_error(None)


@pytest.mark.parametrize("hd,n", [(64, 2 ** 24 * 32), (128, 2 ** 24 * 16), (128, 2 ** 31 - 1), (128, 2 ** 40)])
def test_more_rows_than_a_launch_has_room_for(hd, n):
    rope = B.cf_rope_plan(hd, [32])
    assert B.lib().cf_rope_tables(C.byref(rope), HERE, n, HERE << 30, HERE << 31, None) == B.CF_ERR_ARG and b" rows" in B.lib().cf_last_error(None)
    for rows in (n, 2 ** 24):
        assert apply_code(operand(), rope=rope, n=rows) == B.CF_ERR_ARG and b" rows" in B.lib().cf_last_error(None)


def test_the_binding_refuses_tensors_that_do_not_fit():
    rope = B.cf_rope_plan(64, [16, 16])
    pos, q = torch.zeros(6, 2, dtype=torch.int32), torch.zeros(6, 3, 64)
    t = lambda *s, d=torch.float32: torch.zeros(*s, dtype=d)       # noqa: E731
    for bad in (lambda: B.cf_rope_tables(rope, pos.long(), t(6, 32), t(6, 32)), lambda: B.cf_rope_tables(rope, pos, t(6, 64), t(6, 32)),
                lambda: B.cf_rope_tables(rope, pos[:, :1], t(6, 32), t(6, 32)), lambda: B.cf_rope_tables(rope, pos, t(6, 32), t(6, 32)),
                lambda: B.cf_rope_apply(rope, pos, q, q.half()), lambda: B.cf_rope_apply(rope, pos, q.half(), q.half()), lambda: B.cf_rope_apply(rope, pos, q, q, q),
                lambda: B.cf_rope_apply(rope, pos[:5], q, q), lambda: B.cf_rope_apply(rope, pos, t(6, 3, 128)[..., ::2], q),
                lambda: B.cf_rope_apply(rope, pos, q, t(6, 2, 64)), lambda: B.cf_rope_apply(rope, pos, q, q, t(6, 3, 32), t(6, 3, 32)),
                lambda: B.cf_rope_apply(rope, pos, q, q)):        # all of them on the CPU, the last otherwise in order
        with pytest.raises(B.ChunkflowError) as e:
            bad()
        assert e.value.code == B.CF_ERR_ARG


def test_errors_without_a_context_belong_to_their_thread():
    assert apply_code(operand(x=None)) == B.CF_ERR_ARG
    mine = B.lib().cf_last_error(None)
    seen = []

    def other():
        with pytest.raises(B.ChunkflowError):
            B.cf_rope_plan(96, [4])
        seen.append(B.lib().cf_last_error(None))

    t = threading.Thread(target=other)
    t.start()
    t.join()
    assert B.lib().cf_last_error(None) == mine and b"head_dim 96" in seen[0]
