"""Calls on a paged 8-bit cache that are refused before a GPU is touched."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2605_11335_amd import binding as B
from tests.kvutil import E4M3, power

HERE = 1 << 20          # a made-up aligned address: these calls are refused before anything is read


def cache(**kw):
    f = dict(k=HERE, v=HERE * 2, scales=HERE * 3, table=HERE * 4, n_pages=10, page_tokens=64, heads=4, head_dim=128, n_seqs=3, table_width=5)
    f.update(kw)
    return B.cf_kv_cache(**f)


def new(**kw):
    f = dict(k=HERE * 5, v=HERE * 6, k_row=512, k_head=128, v_row=512, v_head=128, cu=HERE * 7, lens=HERE * 8, n_tokens=9, dtype=B.CF_BF16)
    f.update(kw)
    return B.cf_kv_new(**f)


def query(**kw):
    f = dict(q=HERE * 5, o=HERE * 6, q_row=1024, q_head=128, o_row=1024, o_head=128, cu=HERE * 7, lens=HERE * 8, n_tokens=9, heads=8, max_q=0, causal=0, scale=0.1)
    f.update(kw)
    return B.cf_kv_query(**f)


BAD_CACHES = [dict(k=None), dict(v=None), dict(scales=None), dict(table=None), dict(k=HERE + 8), dict(v=HERE + 1), dict(scales=HERE + 1), dict(table=HERE + 2),
              dict(n_pages=0), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=8192), dict(heads=0), dict(head_dim=96), dict(n_seqs=-1),
              dict(table_width=0), dict(n_pages=2 ** 30), dict(table_width=2 ** 26)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_that_are_refused(bad):
    c, n = cache(**bad), C.c_uint64()
    for rc, name in ((B.lib().cf_kv_append(C.byref(c), C.byref(new()), None), b"kv_append"), (B.lib().cf_kv_attention(C.byref(c), C.byref(query()), None, 0, None), b"kv_attention"),
                     (B.lib().cf_kv_attention_workspace(C.byref(c), C.byref(query()), C.byref(n)), b"kv_attention_workspace")):
        assert rc == B.CF_ERR_ARG
    assert name in B.lib().cf_last_error(None)


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(cu=None), dict(lens=None), dict(k=HERE + 8), dict(v=HERE + 2), dict(cu=HERE + 2), dict(lens=HERE + 1), dict(n_tokens=-1),
                                 dict(dtype=2), dict(dtype=-1), dict(k_row=511), dict(v_head=-128), dict(k_head=4)])
def test_appends_that_are_refused(bad):
    assert B.lib().cf_kv_append(C.byref(cache()), C.byref(new(**bad)), None) == B.CF_ERR_ARG
    assert b"kv_append" in B.lib().cf_last_error(None)


@pytest.mark.parametrize("n_tokens,n_seqs", [(2 ** 28, 1), (2 ** 31 - 1, 1), (9, 2 ** 23), (2 ** 27, 2 ** 22)])
def test_more_tokens_than_a_launch_has_room_for(n_tokens, n_seqs):
    assert B.lib().cf_kv_append(C.byref(cache(n_seqs=n_seqs)), C.byref(new(n_tokens=n_tokens)), None) == B.CF_ERR_ARG
    assert b"too many" in B.lib().cf_last_error(None)


def test_rotations_that_do_not_fit_the_cache():
    right, wrong = B.cf_rope_plan(128, [64]), B.cf_rope_plan(64, [32])
    for rope, pos in ((wrong, HERE * 9), (right, None), (right, HERE * 9 + 2), (B.cf_rope(), HERE * 9)):
        assert B.lib().cf_kv_append(C.byref(cache()), C.byref(new(rope=C.pointer(rope), pos=pos)), None) == B.CF_ERR_ARG


@pytest.mark.parametrize("bad", [dict(q=None), dict(o=None), dict(cu=None), dict(lens=None), dict(q=HERE + 8), dict(o=HERE + 2), dict(cu=HERE + 3), dict(n_tokens=-1), dict(max_q=-1),
                                 dict(heads=6), dict(heads=0), dict(heads=1 << 20), dict(q_row=1020), dict(o_head=-128), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
                                 dict(scale=math.nan)])
def test_queries_that_are_refused(bad):
    ws = C.c_uint64()
    rc = B.lib().cf_kv_attention_workspace(C.byref(cache()), C.byref(query()), C.byref(ws))
    assert rc == B.CF_OK
    assert B.lib().cf_kv_attention(C.byref(cache()), C.byref(query(**bad)), HERE * 16, ws.value, None) == B.CF_ERR_ARG
    assert b"kv_attention" in B.lib().cf_last_error(None)


@pytest.mark.parametrize("o", [dict(o=HERE * 5), dict(o=HERE * 5 + 1024), dict(o_row=512), dict(o_head=64), dict(q_row=2048, o_row=2048, o=HERE * 5 + 1024)])
def test_outputs_over_queries_or_over_one_another(o):
    """In place, half over the queries, rows and heads over one another, and columns of one row that meet by a head; columns side by side are in order."""
    beside = query(q_row=2048, o_row=2048, o=HERE * 5 + 2048)
    assert B.lib().cf_kv_attention(C.byref(cache(table_width=4096)), C.byref(beside), None, 0, None) == B.CF_ERR_ARG
    assert b"workspace" in B.lib().cf_last_error(None)             # (what comes after these checks)
    assert B.lib().cf_kv_attention(C.byref(cache(table_width=4096)), C.byref(query(**o)), None, 0, None) == B.CF_ERR_ARG
    assert b"overlap" in B.lib().cf_last_error(None)


def test_nothing_to_do_is_no_error():
    assert B.lib().cf_kv_append(C.byref(cache()), C.byref(new(n_tokens=0)), None) == B.CF_OK
    assert B.lib().cf_kv_append(C.byref(cache(n_seqs=0)), C.byref(new()), None) == B.CF_OK
    assert B.lib().cf_kv_attention(C.byref(cache()), C.byref(query(n_tokens=0)), None, 0, None) == B.CF_OK
    assert B.lib().cf_kv_attention(C.byref(cache(n_seqs=0)), C.byref(query()), None, 0, None) == B.CF_OK


def test_the_binding_refuses_tensors_that_do_not_fit():
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)          # noqa: E731
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)         # noqa: E731
    k, v, s, t = u8(7, 2, 4, 4, 16, 16), u8(7, 2, 4, 64, 16), u8(7, 2, 4, 2), i32(3, 2)
    c = B.make_kv_cache(k, v, s, t)
    assert (c.c.n_pages, c.c.page_tokens, c.c.heads, c.c.head_dim, c.c.n_seqs, c.c.table_width) == (7, 64, 2, 64, 3, 2)
    B.make_kv_cache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), s, t)
    x, q, cu, lens = torch.zeros(5, 2, 64), torch.zeros(5, 4, 64, dtype=torch.bfloat16), i32(4), i32(3)
    plan, ws = B.cf_rope_plan(64, [16, 16]), u8(1 << 20)
    for bad in (lambda: B.make_kv_cache(k[..., :8], v, s, t), lambda: B.make_kv_cache(k, v[:6], s, t), lambda: B.make_kv_cache(k, v, s.int(), t), lambda: B.make_kv_cache(k, v, s, t.long()),
                lambda: B.make_kv_cache(k, v, s, t[0]), lambda: B.make_kv_cache(k.transpose(0, 1), v, s, t), lambda: B.make_kv_cache(k.float(), v, s, t),
                lambda: B.cf_kv_append(c, x[:, :1], x[:, :1], cu, lens), lambda: B.cf_kv_append(c, x, x.bfloat16(), cu, lens), lambda: B.cf_kv_append(c, x.double(), x.double(), cu, lens),
                lambda: B.cf_kv_append(c, x, x, cu[:3], lens), lambda: B.cf_kv_append(c, x, x, cu.long(), lens), lambda: B.cf_kv_append(c, x, x, cu, i32(4)),
                lambda: B.cf_kv_append(c, x, x, cu, lens, plan, i32(5, 1)), lambda: B.cf_kv_append(c, x, x, cu, lens, plan, None), lambda: B.cf_kv_append(c, x.transpose(1, 2), x, cu, lens),
                lambda: B.cf_kv_append(c, x, x, cu, lens),                                                             # in order, but not on a GPU
                lambda: B.cf_kv_attention(c, q.float(), q.float(), cu, lens), lambda: B.cf_kv_attention(c, q, q[:4], cu, lens), lambda: B.cf_kv_attention(c, q[:, :, :32], q[:, :, :32], cu, lens),
                lambda: B.cf_kv_attention(c, q, q, cu[1:], lens), lambda: B.cf_kv_attention(c, q, q, cu, lens, workspace=ws[::2]), lambda: B.cf_kv_attention(c, q, q, cu, lens, workspace=ws)):
        with pytest.raises(B.ChunkflowError) as e:
            bad()
        assert e.value.code == B.CF_ERR_ARG


def plan(form=-1, c=None, **q):
    out = B.cf_kv_attention_plan()
    rc = B.lib().cf_plan_kv_attention(C.byref(c or cache()), C.byref(query(**q)), form, C.byref(out))
    return rc, out


def test_plans_are_host_arithmetic_and_say_what_workspace_a_form_needs():
    ws = C.c_uint64()
    for form in (-1, 0, 1, 2, 3):
        rc, p = plan(form)
        assert rc == B.CF_OK and (form < 0 or p.form == form) and p.columns == (256 if p.form >= 2 else 32) and p.workgroups > 0
        assert (p.workspace_bytes == 0) == (p.form in (1, 3))
        if form < 0:
            assert B.lib().cf_kv_attention_workspace(C.byref(cache()), C.byref(query()), C.byref(ws)) == B.CF_OK and ws.value == p.workspace_bytes
        # an operand short or misaligned is refused, and so is a form that is none
        if p.workspace_bytes:
            for at, size in ((None, p.workspace_bytes), (HERE * 16 + 128, p.workspace_bytes), (HERE * 16, p.workspace_bytes - 1)):
                assert B.lib().cf_op_kv_attention_form(C.byref(cache()), C.byref(query()), p.form, at, size, None) == B.CF_ERR_ARG
    assert plan(4)[0] == B.CF_ERR_ARG and plan(-2)[0] == B.CF_ERR_ARG
    assert B.lib().cf_op_kv_attention_form(C.byref(cache()), C.byref(query()), -1, HERE * 16, 1 << 40, None) == B.CF_ERR_ARG
    # a call without a workspace that needs one
    big = cache(table_width=4096)
    assert B.lib().cf_kv_attention_workspace(C.byref(big), C.byref(query(n_tokens=3)), C.byref(ws)) == B.CF_OK and ws.value > 0
    assert B.lib().cf_kv_attention(C.byref(big), C.byref(query(n_tokens=3)), None, 0, None) == B.CF_ERR_ARG


def test_the_most_queries_of_a_sequence_count_for_the_plan():
    """Single tokens of many sequences are few columns each; as many queries of one sequence, over as many tokens, are many."""
    wide = cache(n_seqs=64, table_width=512, heads=8)
    assert plan(c=wide, n_tokens=64, heads=8, max_q=1)[1].columns == 32
    assert plan(c=cache(n_seqs=1, table_width=512, heads=8), n_tokens=2000, heads=8)[1].columns == 256


def test_launches_have_room_for_any_number_of_queries():
    for form in range(4):
        assert 0 < plan(form, n_tokens=2 ** 27, heads=8)[1].workgroups <= 2 ** 20


def test_the_helpers_know_the_format():
    """The tests' own e4m3 table and power rule, against torch's type and by hand."""
    every = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(every.view(torch.float8_e4m3fn).double().numpy(), E4M3, equal_nan=True)
    assert [power(x) for x in (0.0, 448.0, 449.0, 224.0, 1.0, 1e-40)] == [-100, 0, 1, -1, -8, -100]
