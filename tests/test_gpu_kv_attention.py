"""Attention over a paged 8-bit cache against the definition in 64 bits: ragged, empty, causal, holes in the table, codes that nobody may see."""
import math

import numpy as np
import pytest
import torch

from paper_2605_11335_amd import binding as B
from tests.kvutil import DEV, Cache, attention, lens_t
from tests.util import bf16_round, dev_bits

pytestmark = pytest.mark.gpu


FORMS = (-1, 0, 1, 2, 3)         # the planner's, few columns cut and whole, many cut and whole


def run(cache, q_bits, cu, lens, causal=False, scale=None, max_q=0, dev=None, stream=None, strided=False, form=-1):
    """Output [rows, heads, hd] in 64 bits; rows of no sequence keep a mark (7)."""
    q = dev_bits(q_bits).view(torch.bfloat16)
    if strided:                                     # heads outside rows, with a gap behind every head
        n, heads, hd = q.shape
        buf = torch.zeros(heads, n + 1, hd, dtype=torch.bfloat16, device=DEV)
        buf[:, :n] = q.transpose(0, 1)
        q, o = buf[:, :n].transpose(0, 1), torch.full((heads, n + 1, 2 * hd), 7.0, dtype=torch.bfloat16, device=DEV)[:, :n, hd:].transpose(0, 1)
    else:
        o = torch.full_like(q, 7.0)
    dev = cache.device(B) if dev is None else dev
    need = B.cf_plan_kv_attention(dev, q, max_q, form).workspace_bytes
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)           # (NaN, should anything be read before it is written)
    if form < 0:
        assert need == B.cf_kv_attention_workspace(dev, q, max_q)
        B.cf_kv_attention(dev, q, o, lens_t(cu), lens_t(lens), causal, scale, max_q, ws, stream)
    else:
        B.cf_op_kv_attention_form(dev, q, o, lens_t(cu), lens_t(lens), form, causal, scale, max_q, ws, stream)
    torch.cuda.synchronize()
    return o.double().cpu().numpy()


def check(cache, q, cu, lens, causal=False, scale=None, forms=FORMS, **kw):
    """Every form against the definition; their outputs."""
    val, bits = bf16_round(q)
    want, tol = attention(cache, val.astype(np.float64), cu, lens, causal, cache.hd ** -0.5 if scale is None else scale)
    mine = ~np.isnan(want[:, 0, 0])
    dev, out = cache.device(B), []
    for form in forms:
        got = run(cache, bits, cu, lens, causal, scale, dev=dev, form=form, **kw)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad[mine].any(), f"form {form}: {bad[mine].sum()} of {bad[mine].size}, worst {np.nanmax((np.abs(got - want) - tol)[mine]):.3e} over, " \
                                    f"at {np.argwhere(bad & mine[:, None, None])[:5].tolist()}"
        assert (got[~mine] == 7).all()
        out.append(got)
    return out


def offsets(n, first=0):
    return np.concatenate([[0], np.cumsum(n)]) + first


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (8, 2), (16, 1)])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("causal", [False, True])
def test_one_query_each(hd, heads, kv_heads, page, causal):
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 130, 1000, 2049]
    rng = np.random.default_rng(hd + heads + page)
    cache = Cache(rng, len(lens), kv_heads, hd, page, max(lens), fill="small")
    check(cache, rng.normal(size=(len(lens), heads, hd)), offsets([1] * len(lens)), lens, causal, max_q=1)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (6, 2)])
@pytest.mark.parametrize("n", [2, 7, 11, 31, 33, 100, 300])
@pytest.mark.parametrize("causal", [False, True])
def test_several_queries(hd, heads, kv_heads, n, causal):
    """Ragged queries and lengths; causal ones with fewer tokens than queries, whose first queries see nothing."""
    rng = np.random.default_rng(hd + heads + n)
    counts, lens = [n, 0, 1, n // 2, n], [700, 50, 65, max(1, n // 3), n]
    cache = Cache(rng, 5, kv_heads, hd, 32, 700, fill="small")
    cu = offsets(counts, 3)
    check(cache, rng.normal(size=(cu[-1] + 2, heads, hd)), cu, lens, causal, max_q=n, strided=n % 2 == 1)


@pytest.mark.parametrize("max_q", [0, 1, 40, 5000])
def test_what_is_said_of_the_most_queries_only_plans(max_q):
    rng = np.random.default_rng(max_q)
    cache = Cache(rng, 3, 2, 128, 64, 900, fill="small")
    check(cache, rng.normal(size=(46, 4, 128)), offsets([5, 1, 40]), [900, 17, 333], True, max_q=max_q)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("hd", [64, 128])
def test_pages_that_are_not_there_and_pages_that_are_shared(n, hd):
    rng = np.random.default_rng(n + hd)
    cache = Cache(rng, 4, 2, hd, 32, 400, fill="small")
    cache.table[0, [0, 3, 12]] = [-1, cache.pages, 2 ** 31 - 1]       # holes, one at the end
    cache.table[1] = -2                                               # no page at all
    cache.table[2] = cache.table[3]
    got = check(cache, rng.normal(size=(4 * n, 4, hd)), offsets([n] * 4), [400, 400, 400, 390], n > 1)
    assert all((g[n:2 * n] == 0).all() for g in got)
    # more tokens than the table has room for, and a negative number of them
    check(cache, rng.normal(size=(4 * n, 4, hd)), offsets([n] * 4), [2 ** 31 - 1, 0, -5, 100000])


@pytest.mark.parametrize("n", [1, 3, 70])
@pytest.mark.parametrize("hd", [64, 128])
def test_codes_that_no_query_sees_are_anything(n, hd):
    """NaN codes, and powers that make everything NaN, behind the lengths and in pages that a table no longer names."""
    rng = np.random.default_rng(n + hd)
    lens = [1, 16, 100, 205]
    cache = Cache(rng, 4, 2, hd, 64, 256, fill="small")
    q, cu = rng.normal(size=(4 * n, 4, hd)), offsets([n] * 4)
    cache.table[3, 1] = -1
    clean = check(cache, q, cu, lens)
    seen = np.zeros((cache.pages, 4, 16), bool)
    for b, held in enumerate(lens):
        for p in range(held):
            at = cache.group(b, p)
            if at:
                seen[at[0], at[1], p % 16] = True
    unseen = ~seen[:, None]                                            # [pages, 1, groups, slots]
    cache.k[np.broadcast_to(unseen[..., None, :, None], cache.k.shape)] = 0x7f
    cache.v[np.broadcast_to(unseen[..., None, :], cache.v.shape)] = 0xff
    cache.scales[np.broadcast_to(~seen.any(-1)[:, None, :, None], cache.scales.shape)] = 255
    for form, got, was in zip(FORMS, check(cache, q, cu, lens), clean):
        assert np.array_equal(got, was), form


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n", [5, 90])
def test_causal_queries_do_not_see_what_comes_after_them(hd, n, form):
    """Keys and values of NaN behind query j leave the queries up to j as they are, and reach all others."""
    rng = np.random.default_rng(hd + n)
    held = n + 37
    cache = Cache(rng, 1, 2, hd, 32, held, fill="small")
    _, bits = bf16_round(rng.normal(size=(n, 4, hd)))
    cu = offsets([n])
    clean = run(cache, bits, cu, [held], True, form=form)
    for which in ("k", "v"):
        for j in (0, n // 2, n - 2):
            pg, g = cache.group(0, held - n + j + 1)
            slot = (held - n + j + 1) % 16
            was = getattr(cache, which).copy()
            if which == "k":
                cache.k[pg, 1, g, 0, slot, 3] = 0x7f
            else:
                cache.v[pg, 1, g, 5, slot] = 0x7f
            got = run(cache, bits, cu, [held], True, form=form)
            assert np.array_equal(got[:, :2], clean[:, :2]) and np.array_equal(got[:j + 1], clean[:j + 1]), (which, j)
            hit = got[j + 1:, 2:] if which == "k" else got[j + 1:, 2:, 5]
            assert np.isnan(hit).all(), (which, j)
            if which == "v":
                assert np.array_equal(np.delete(got, 5, 2), np.delete(clean, 5, 2))
            setattr(cache, which, was)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n", [1, 50])
@pytest.mark.parametrize("step", [0.7, 3.0, 30.0, 200.0])
def test_scores_that_keep_rising_along_the_keys(hd, n, step):
    """Every 64 keys score `step` nats over the ones before: whatever reference the softmax keeps moves again and again."""
    rng = np.random.default_rng(int(step * 10) + hd)
    held = 64 * 12 + 5
    cache = Cache(rng, 1, 1, hd, 64, held, fill="small")
    cache.k[:] &= 0x8f                                                 # small keys (up to 2^-5) but for dim 0, which makes the steps
    q = rng.normal(size=(n, 2, hd))
    q[:, :, 0] = 16.0
    for p in range(held):
        pg, g = cache.group(0, p)
        cache.scales[pg, 0, g, 0] = 127
        want = step * (p // 64) * hd ** 0.5 / 16.0
        cache.k[pg, 0, g, 0, p % 16, 0] = np.nanargmin(np.abs(E_ROUND - min(want, 448.0)))
    check(cache, q, offsets([n]), [held])


E_ROUND = np.where(np.arange(256) < 128, __import__("tests.kvutil", fromlist=["E4M3"]).E4M3, np.nan)


def test_powers_of_two_from_end_to_end_and_a_query_that_is_nan():
    rng = np.random.default_rng(3)
    cache = Cache(rng, 2, 2, 128, 32, 200, fill="small")
    cache.scales[..., 0] = rng.integers(60, 128, cache.scales.shape[:-1])
    cache.scales[..., 1] = rng.integers(40, 215, cache.scales.shape[:-1])
    q = rng.normal(size=(6, 4, 128))
    check(cache, q, offsets([5, 1]), [200, 77])
    q[2, 1] = np.nan
    for form in FORMS:
        got = run(cache, bf16_round(np.where(np.isnan(q), 0, q))[1] | np.where(np.isnan(q), 0x7fc0, 0).astype(np.uint16), offsets([5, 1]), [200, 77], form=form)
        assert np.isnan(got[2, 1]).all() and np.isfinite(np.delete(got.reshape(24, 128), 9, 0)).all()


def test_scale_and_every_power_of_the_format():
    """One key per group, all 254 bytes of the value's power: what comes out is the value itself, or the end of bf16's range."""
    rng = np.random.default_rng(8)
    seqs = 254
    cache = Cache(rng, seqs, 1, 64, 16, 16, fill="small")
    for b in range(seqs):
        cache.scales[cache.table[b, 0], 0, 0, 1] = b + 1
    cache.v[:, 0, 0, :, 0] = np.where(cache.v[:, 0, 0, :, 0] & 0x78, cache.v[:, 0, 0, :, 0], 0x38)        # normal codes
    _, bits = bf16_round(rng.normal(size=(seqs, 1, 64)))
    want = np.stack([cache.held(b, 1)[1][0, 0] for b in range(seqs)])
    inside = (np.abs(want) >= 2.0 ** -126) & (np.abs(want) < 2.0 ** 127)
    for form in FORMS:
        got = run(cache, bits, offsets([1] * seqs), [1] * seqs, scale=3.5, form=form)
        assert np.array_equal(got[:, 0][inside], want[inside]) and (np.abs(got[:, 0] - want)[~inside & (np.abs(want) < 2.0 ** -126)] <= 2.0 ** -126).all()


@pytest.mark.parametrize("n,held,hd,kv_heads", [(1, 20001, 128, 2), (3, 9000, 128, 2), (1, 130001, 128, 2), (1, 130001, 64, 4)])
def test_long_caches(n, held, hd, kv_heads):
    """(Of 130001 tokens: one query each goes past the caches.)"""
    rng = np.random.default_rng(held + hd)
    cache = Cache(rng, 2, kv_heads, hd, 128, held, fill="small")
    check(cache, rng.normal(size=(2 * n, 2 * kv_heads, hd)), offsets([n, n]), [held, held // 3], n > 1, max_q=n)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("n", [1, 64])
def test_a_cache_past_4_gib(n, form):
    """Pages whose codes lie behind 2^32 bytes, among them the last."""
    heads, hd, page, pages = 8, 128, 128, 45000                     # 5.9 GB of K and of V
    k = torch.zeros(pages, heads, page // 16, hd // 16, 16, 16, dtype=torch.uint8, device=DEV)
    v = torch.zeros(pages, heads, page // 16, hd, 16, dtype=torch.uint8, device=DEV)
    scales = torch.full((pages, heads, page // 16, 2), 127, dtype=torch.uint8, device=DEV)
    rng = np.random.default_rng(n)
    small = Cache(rng, 1, heads, hd, page, 600, spare=0, fill="small")
    at = [44999, 32768, 32767, 3, 40001]
    for i, p in enumerate(at):
        src = int(small.table[0, i])
        k[p], v[p], scales[p] = (torch.from_numpy(x[src]).to(DEV) for x in (small.k, small.v, small.scales))
    big = B.make_kv_cache(k, v, scales, torch.tensor([at], dtype=torch.int32, device=DEV))
    _, bits = bf16_round(rng.normal(size=(n, 8, hd)))
    want, got = run(small, bits, offsets([n]), [600], max_q=n, form=form), run(small, bits, offsets([n]), [600], max_q=n, dev=big, form=form)
    assert np.array_equal(want, got)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("n", [1, 60])
def test_replays_of_a_captured_call_on_other_lengths(n, form):
    """... and of two calls that share a workspace, with other calls in it between the replays."""
    rng = np.random.default_rng(n)
    cache = Cache(rng, 3, 2, 128, 32, 3000, fill="small")
    dev = cache.device(B)
    _, bits = bf16_round(rng.normal(size=(3 * n, 8, 128)))
    q = dev_bits(bits).view(torch.bfloat16)
    cu, lens, o, o2 = lens_t(offsets([n] * 3)), lens_t([n] * 3), torch.zeros_like(q), torch.zeros_like(q)
    ws = torch.empty(max(B.cf_plan_kv_attention(dev, q, n, f).workspace_bytes for f in FORMS), dtype=torch.uint8, device=DEV)

    def call(form, o, causal):
        if form < 0:
            B.cf_kv_attention(dev, q, o, cu, lens, causal, None, n, ws)
        else:
            B.cf_op_kv_attention_form(dev, q, o, cu, lens, form, causal, None, n, ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(form, o, True)
        call(2, o2, False)
    for held in ([n, n + 1, 2 * n], [3000, 1, 700], [0, 64, 2999], [3000, 3000, 3000], [3000, 3000, 3000]):
        lens.copy_(lens_t(held))
        o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(o.double().cpu().numpy(), run(cache, bits, offsets([n] * 3), held, True, max_q=n, dev=dev, form=form)), held
        assert np.array_equal(o2.double().cpu().numpy(), run(cache, bits, offsets([n] * 3), held, False, max_q=n, dev=dev, form=2)), held
        call((form + 1) % 4, o, False)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("n,heads", [(1, 6), (60, 6), (700, 12)])
def test_the_same_call_gives_the_same_bits(n, heads, form):
    """Whichever workgroup joins the pieces of a column tile, and when."""
    rng = np.random.default_rng(n)
    cache = Cache(rng, 2, 3, 128, 64, 5000, fill="small")
    dev = cache.device(B)
    _, bits = bf16_round(rng.normal(size=(2 * n, heads, 128)))
    first = run(cache, bits, offsets([n] * 2), [5000, 4321], dev=dev, max_q=n, form=form)
    side = torch.cuda.Stream()
    for stream in (None, side, None, None):
        assert np.array_equal(first, run(cache, bits, offsets([n] * 2), [5000, 4321], dev=dev, max_q=n, stream=stream, form=form))


@pytest.mark.parametrize("form", [0, 1, 2, 3])
def test_outputs_past_4_gib(form):
    """2^25 columns: in the form of a workgroup for each column tile of 32, several to a workgroup.  One token: every query's output is its value."""
    rng = np.random.default_rng(form)
    cache = Cache(rng, 1, 1, 64, 16, 16, fill="small")
    n = 2 ** 20 + 5
    q = torch.ones(n, 32, 64, dtype=torch.bfloat16, device=DEV)
    o, dev = torch.full_like(q, 7.0), cache.device(B)
    ws = torch.empty(B.cf_plan_kv_attention(dev, q, n, form).workspace_bytes, dtype=torch.uint8, device=DEV)
    B.cf_op_kv_attention_form(dev, q, o, lens_t([0, n - 1]), lens_t([1]), form, False, None, n, ws)
    want = torch.from_numpy(cache.held(0, 1)[1][0, 0]).to(DEV, torch.bfloat16)
    assert bool((o[:-1] == want).all()) and bool((o[-1] == 7).all())


@pytest.mark.parametrize("hd,heads", [(64, 1), (64, 8), (128, 1), (128, 4), (128, 5)])
def test_a_column_tile_in_two_pieces_has_one_result(hd, heads):
    """128 sequences of the same tokens, each the work of two of 256 shares, which either the first share's workgroup or the joining kernel puts together:
    no matter which.  Values and scores are such that the halves all but cancel and the last bit of a product is seen."""
    rng = np.random.default_rng(heads)
    seqs, held = 128, 640
    cache = Cache(rng, seqs, 1, hd, 64, held)
    late = np.zeros((cache.pages, 1, 1, 1, 1), bool)
    late[cache.table[:, held // 128:].ravel()] = True
    cache.k[:] = 0
    cache.k[..., 0, :, 0] = np.where(late[..., 0], 0, 0x38)              # 1 or 0 in the first dim: scores q and 0
    cache.v[:] = np.where(late, 0xb8, 0x30)                              # -1, 1 / 2
    cache.scales[:] = 127
    q = bf16_round(np.ones((seqs, heads, hd)))[1]
    dev = cache.device(B)
    shape = dev_bits(q).view(torch.bfloat16)
    assert B.cf_plan_kv_attention(dev, shape, 1, 2).workgroups == 2 * seqs
    for ppm in (5, 10, 20, 40):
        for _ in range(4):
            got = run(cache, q, offsets([1] * seqs), [held] * seqs, scale=math.log(2) * (1 + ppm * 1e-6), dev=dev, max_q=1, form=2)
            assert (got == got[0, 0, 0]).all(), np.unique(got)


def test_the_planner_takes_every_form():
    """A token over a long cache, over a short one, a few thousand queries over a clip, a few hundred over one text for every head."""
    def form(queries, heads, kv_heads, seqs, capacity):
        z = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=DEV)       # noqa: E731
        cache = B.make_kv_cache(z(1, kv_heads, 4, 8, 16, 16), z(1, kv_heads, 4, 128, 16), z(1, kv_heads, 4, 2), torch.zeros(seqs, capacity // 64, dtype=torch.int32, device=DEV))
        return B.cf_plan_kv_attention(cache, torch.empty(queries, heads, 128, dtype=torch.bfloat16, device=DEV)).form
    assert [form(1, 12, 12, 1, 131072), form(16, 8, 8, 16, 512), form(3520, 12, 12, 1, 27264), form(2560, 24, 24, 1, 2048)] == [0, 1, 2, 3]
