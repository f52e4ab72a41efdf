"""Appending to a paged 8-bit cache: powers and codes against the definition, old tokens of a group that gets a larger power, what must stay as it was."""
import numpy as np
import pytest
import torch

from paper_2605_11335_amd import binding as B
from tests.kvutil import DEV, E4M3, E4M3_ABS, E4M3_REL, E_LEAST, ULP, Cache, attention, lens_t, power
from tests.test_gpu_rope import TABLE_TOL, angles, turned
from tests.util import bf16_round

pytestmark = pytest.mark.gpu


def e4m3(x):
    """Nearest code, ties to even, of values up to 448 (torch on the CPU)."""
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def append(cache, k, v, cu, lens, pairs=None, pos=None):
    """The cache (host copy, changed in place) after the call by the definition; codes of turned keys are left to `slack`, a dict
    {(page, group, slot): (values [heads, hd], how far off [heads, hd])} in units of the group's power."""
    slack, was = {}, (cache.k.copy(), cache.v.copy(), cache.scales.copy())
    want = turned(k, angles(pos, pairs, cache.hd)) if pairs else k
    for b in range(len(lens)):
        held = min(max(int(lens[b]), 0), cache.table.shape[1] * cache.page)
        p, end = held, held + cu[b + 1] - cu[b]
        while p < end:
            upto, at = min(end, (p // 16 + 1) * 16), cache.group(b, p)
            rows = slice(cu[b] + p - held, cu[b] + upto - held)
            if at is not None:
                pg, g = at
                a0, a1 = p % 16, (upto - 1) % 16 + 1
                for h in range(cache.heads):
                    for w, x in enumerate((k, v)):
                        y = np.abs(x[rows, h])
                        if w == 0 and pairs:
                            y = y[:, 0::2] + y[:, 1::2]
                        y = y[np.isfinite(y)]
                        e = power(y.max() if y.size else 0)
                        pool = (cache.k[pg, h, g].transpose(1, 0, 2).reshape(16, cache.hd), cache.v[pg, h, g].T)[w].copy()         # [slots, dims]
                        if a0:
                            old = int(was[2][pg, h, g, w]) - 127
                            e = max(e, old)
                            if e > old:
                                pool[:a0] = e4m3(np.ldexp(E4M3[pool[:a0]], old - e))
                        new = np.ldexp((want if w == 0 else v)[rows, h], -e)
                        pool[a0:a1] = e4m3(np.where(np.isfinite(new), np.clip(new, -448, 448), np.nan))
                        cache.scales[pg, h, g, w] = e + 127
                        if w == 0:
                            cache.k[pg, h, g] = pool.reshape(16, cache.hd // 16, 16).transpose(1, 0, 2)
                            for i, slot in enumerate(range(a0, a1)):
                                pair = np.abs(k[rows, h][i]).reshape(-1, 2).sum(-1).repeat(2)
                                s = slack.setdefault((pg, g, slot), (np.zeros((cache.heads, cache.hd)), np.zeros((cache.heads, cache.hd))))
                                s[0][h], s[1][h] = new[i], np.ldexp(pair * (TABLE_TOL + 3 * ULP), -e)
                        else:
                            cache.v[pg, h, g] = pool.T
            p = upto
    return slack if pairs else {}


def check(cache, dev, slack):
    """What the GPU has is what the host copy has, turned keys within half a step of what they should be."""
    torch.cuda.synchronize()
    k, v, scales, table = (t.cpu().numpy() for t in dev.tensors)
    assert np.array_equal(scales, cache.scales) and np.array_equal(table, cache.table)
    assert np.array_equal(E4M3[v], E4M3[cache.v], equal_nan=True)          # (a zero may have either sign)
    mine = np.ones(k.shape, bool)
    for (pg, g, slot), (x, off) in slack.items():
        got = E4M3[k[pg, :, g, :, slot]].reshape(cache.heads, cache.hd)
        ok = np.abs(got - x) <= np.maximum(E4M3_REL * np.abs(x), E4M3_ABS) + off * (1 + E4M3_REL)
        assert (ok | (np.isnan(got) & np.isnan(x))).all(), (pg, g, slot, np.argwhere(~ok)[:4], got[~ok][:4], x[~ok][:4])
        mine[pg, :, g, :, slot] = False
    assert np.array_equal(E4M3[k[mine]], E4M3[cache.k[mine]], equal_nan=True)
    cache.copy_back(dev)


def tokens(rng, n, heads, hd, dtype, size=1.0):
    x = rng.normal(size=(n, heads, hd)) * size
    return (bf16_round(x)[0] if dtype == torch.bfloat16 else x.astype(np.float32)).astype(np.float64)


def go(cache, dev, k, v, cu, lens, dtype, pairs=None, pos=None, strided=False, theta=10000.0):
    def put(x):
        t = torch.from_numpy(x).to(torch.float32).to(dtype)
        if strided:                                    # heads outside rows, values beside keys
            t = torch.cat([t, t], 2).transpose(0, 1).contiguous().transpose(0, 1)[..., :t.shape[2]]
        return t.to(DEV) if not strided else torch.empty_strided(t.shape, (2 * t.shape[2], t.shape[0] * 2 * t.shape[2], 1), dtype=dtype, device=DEV).copy_(t)
    plan = B.cf_rope_plan(cache.hd, pairs) if pairs else None
    B.cf_kv_append(dev, put(k), put(v), lens_t(cu), lens_t(lens), plan, None if pos is None else torch.from_numpy(pos).to(DEV))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("heads", [1, 5])
def test_ragged_batches(dtype, hd, page, rope, heads):
    """Runs that begin and end anywhere in a group, single tokens, none, more than the table has room for; larger and smaller values than before."""
    lens, counts = [0, 1, 15, 16, 20, 33, 250, 100, 7], [40, 1, 1, 1, 5, 0, 20, 16, 3]
    rng = np.random.default_rng(hd + page + heads)
    cache = Cache(rng, len(lens), heads, hd, page, 250)
    assert cache.table.shape[1] * page < 270
    cu = np.concatenate([[2], 2 + np.cumsum(counts)])
    n = cu[-1] + 3
    size = np.exp(rng.normal(size=(n, 1, 1)) * 3)
    k, v = tokens(rng, n, heads, hd, dtype, size), tokens(rng, n, heads, hd, dtype, size[::-1])
    pairs = ([10, 9, 7], [22, 21, 21])[hd == 128] if rope else None
    pos = rng.integers(-1000, 100000, size=(n, 3)).astype(np.int32) if rope else None
    dev = cache.device(B)
    go(cache, dev, k, v, cu, lens, dtype, pairs, pos, strided=heads > 1)
    slack = append(cache, k, v, cu, lens, pairs, pos)
    check(cache, dev, slack)
    go(cache, dev, k, v, cu, lens, dtype, pairs, pos)          # the same again changes nothing
    check(cache, dev, {})


def test_token_by_token_and_all_at_once():
    """Codes of tokens appended one by one, the largest last: every step by the definition; the power is that of all at once, and codes
    differ from those by what two roundings make."""
    rng = np.random.default_rng(1)
    one, all_ = (Cache(np.random.default_rng(9), 2, 3, 128, 32, 64) for _ in range(2))
    n = 39
    k, v = (tokens(rng, n, 3, 128, torch.bfloat16, np.exp(np.linspace(-4, 4, n))[:, None, None]) for _ in range(2))
    pos = np.arange(n, dtype=np.int32)[:, None] * 77
    dev, dev2 = one.device(B), all_.device(B)
    for i in range(n):
        go(one, dev, k[i:i + 1], v[i:i + 1], [0, 1, 1], [i, 5], torch.bfloat16, [64], pos[i:i + 1])
        check(one, dev, append(one, k[i:i + 1], v[i:i + 1], [0, 1, 1], [i, 5], [64], pos[i:i + 1]))
    go(all_, dev2, k, v, [0, n, n], [0, 5], torch.bfloat16, [64], pos)
    check(all_, dev2, append(all_, k, v, [0, n, n], [0, 5], [64], pos))
    assert np.array_equal(one.scales, all_.scales)
    a, b = one.held(0, n), all_.held(0, n)
    for x, y, w in zip(a[:2], b[:2], (0, 1)):
        unit = np.stack([np.ldexp(1.0, one.scales[one.group(0, p)[0], :, one.group(0, p)[1], w].astype(int) - 127) for p in range(n)], 1)[..., None]
        assert (np.abs(x - y) <= 3 * E4M3_REL * np.abs(y) + 17 * E4M3_ABS * unit).all()       # up to 16 roundings of a subnormal


@pytest.mark.parametrize("rope", [False, True])
def test_values_at_the_ends(rope):
    """Zeros, the ends of the fp32 range, values at and next to 448 times a power, subnormals, infinities and NaN."""
    top = 3.3895313892515355e38                                   # bf16's largest
    v = np.zeros((16 * 12, 1, 64))
    for g, x in enumerate([0.0, top, 448.0, 450.0, 449.0 * 2.0 ** 40, 1e-38, 2.0 ** -100 * 448, 2.0 ** -109, 1.0, np.inf, np.nan, -np.inf]):
        v[16 * g + 3, 0, 7] = x
        v[16 * g + 5, 0, 8] = -x / 3
    v[16 * 9 + 1, 0, :] = 5.0                                     # beside the infinity: keeps its own power
    v[16 * 10 + 1, 0, :] = -5.0
    v = bf16_round(np.where(np.isfinite(v), v, 0))[0].astype(np.float64) + np.where(np.isfinite(v), 0, v)
    rng = np.random.default_rng(0)
    cache = Cache(rng, 1, 1, 64, 32, len(v))
    dev = cache.device(B)
    pos = np.zeros((len(v), 1), np.int32)                         # turned by nothing: only the power differs
    t = torch.from_numpy(v).to(torch.bfloat16).to(DEV)
    B.cf_kv_append(dev, t, t, lens_t([0, len(v)]), lens_t([0]), B.cf_rope_plan(64, [32]) if rope else None, torch.from_numpy(pos).to(DEV) if rope else None)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        k = v if not rope else np.where(np.isfinite(v.reshape(-1, 1, 32, 2)).all(-1, keepdims=True), v.reshape(-1, 1, 32, 2), np.nan).reshape(v.shape)
        slack = append(cache, k, v, [0, len(v)], [0])
    if rope:                                                      # |a| + |b| instead of the largest: here both sit in one pair only where said
        for p in range(0, len(v), 16):
            pg, g = cache.group(0, p)
            y = np.abs(k[p:p + 16, 0].reshape(16, 32, 2)).sum(-1)
            y = y[np.isfinite(y)]
            old, e = int(cache.scales[pg, 0, g, 0]) - 127, power(y.max())
            cache.scales[pg, 0, g, 0] = e + 127
            new = np.ldexp(k[p:p + 16, 0], -e)
            cache.k[pg, 0, g] = e4m3(new).reshape(16, 4, 16).transpose(1, 0, 2)
    check(cache, dev, slack)


def test_every_code_moves_to_larger_powers_exactly_as_the_format_says():
    """All finite codes as old tokens, then a token that needs a power larger by 0 ... 20."""
    for up in list(range(10)) + [15, 20, 100]:
        rng = np.random.default_rng(up)
        cache = Cache(rng, 1, 1, 128, 16, 16)
        pg = int(cache.table[0, 0])
        every = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
        flat = np.concatenate([every, np.full(15 * 128 - len(every), 0x7f)]).astype(np.uint8).reshape(15, 128)        # the rest NaN
        cache.k[pg, 0, 0, :, :15] = flat.reshape(15, 8, 16).transpose(1, 0, 2)
        cache.v[pg, 0, 0, :, :15] = flat.T
        cache.scales[pg, 0, 0] = 120
        x = np.zeros((1, 1, 128))
        x[0, 0, 50] = 448.0 * 2.0 ** (up - 7)
        dev = cache.device(B)
        go(cache, dev, x, x, [0, 1], [15], torch.float32)
        append(cache, x, x, [0, 1], [15])
        assert (cache.scales[pg, 0, 0] == 120 + up).all()
        check(cache, dev, {})


def test_pages_that_are_not_there_are_not_written():
    rng = np.random.default_rng(4)
    cache = Cache(rng, 3, 2, 64, 32, 128)
    cache.table[0, 1], cache.table[1, :], cache.table[2, 3] = -1, cache.pages, -2 ** 31
    n = [128, 50, 40]
    cu = np.concatenate([[0], np.cumsum(n)])
    k, v = (tokens(rng, cu[-1], 2, 64, torch.float32) for _ in range(2))
    dev = cache.device(B)
    go(cache, dev, k, v, cu, [0, 3, 100], torch.float32)
    append(cache, k, v, cu, [0, 3, 100])
    check(cache, dev, {})


def test_many_sequences():
    """More sequences than a wave has lanes, most of them without a token."""
    rng = np.random.default_rng(6)
    seqs = 300
    counts, lens = rng.integers(0, 4, seqs) * (rng.random(seqs) < 0.3), rng.integers(0, 40, seqs)
    cache = Cache(rng, seqs, 1, 64, 16, 48)
    cu = np.concatenate([[0], np.cumsum(counts)])
    k, v = (tokens(rng, cu[-1], 1, 64, torch.bfloat16) for _ in range(2))
    dev = cache.device(B)
    go(cache, dev, k, v, cu, lens, torch.bfloat16)
    append(cache, k, v, cu, lens)
    check(cache, dev, {})


def test_a_cache_past_4_gib():
    heads, hd, page, pages = 8, 128, 128, 45000
    k = torch.zeros(pages, heads, page // 16, hd // 16, 16, 16, dtype=torch.uint8, device=DEV)
    v = torch.zeros(pages, heads, page // 16, hd, 16, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(pages, heads, page // 16, 2, dtype=torch.uint8, device=DEV)
    at = [44999, 32768, 3]
    big = B.make_kv_cache(k, v, scales, torch.tensor([at], dtype=torch.int32, device=DEV))
    rng = np.random.default_rng(2)
    cache = Cache(rng, 1, heads, hd, page, 300, spare=0)
    cache.k[:], cache.v[:], cache.scales[:] = 0, 0, 0
    x, y = tokens(rng, 290, heads, hd, torch.bfloat16), tokens(rng, 290, heads, hd, torch.bfloat16)
    small = cache.device(B)
    for dev in (big, small):
        go(cache, dev, x, y, [0, 290], [10], torch.bfloat16)
    torch.cuda.synchronize()
    for t, u in zip(big.tensors[:3], small.tensors[:3]):
        assert torch.equal(t[at], u[cache.table[0].tolist()]) and int(t.view(-1).bool().sum()) == int(u.view(-1).bool().sum())


def test_frames_and_tokens_of_a_stream_and_the_attention_over_them():
    """What a generator of frames does: positions on three axes, q turned, k turned and appended, attention over everything so far, step after step,
    the calls of a step captured into a graph and replayed; the cache against the definition, the attention against the cache in 64 bits."""
    rng = np.random.default_rng(12)
    heads, kv_heads, hd, pairs, seqs = 6, 3, 128, [22, 21, 21], 2
    plan = B.cf_rope_plan(hd, pairs)
    cache = Cache(rng, seqs, kv_heads, hd, 32, 200)
    dev = cache.device(B)
    n = [20, 13]
    cu, lens = np.concatenate([[0], np.cumsum(n)]), np.array([0, 5])
    rows = int(cu[-1])
    q, k, v = (torch.zeros(rows, h, hd, dtype=torch.bfloat16, device=DEV) for h in (heads, kv_heads, kv_heads))
    qr, o, pos = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(rows, 3, dtype=torch.int32, device=DEV)
    cut, before, after = lens_t(cu), lens_t(lens), lens_t(lens + n)
    ws = torch.empty(B.cf_kv_attention_workspace(dev, q, max(n)), dtype=torch.uint8, device=DEV)

    def step():
        B.cf_rope_apply(plan, pos, q, qr)
        B.cf_kv_append(dev, k, v, cut, before, plan, pos)
        B.cf_kv_attention(dev, qr, o, cut, after, max_q=max(n), workspace=ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        size = 2.0 ** (i % 3)
        x = [tokens(rng, rows, t.shape[1], hd, torch.bfloat16, size) for t in (q, k, v)]
        for t, y in zip((q, k, v), x):
            t.copy_(torch.from_numpy(y))
        p = np.stack([np.full(rows, 1000 + i), np.arange(rows) // 5, np.arange(rows) % 5], 1).astype(np.int32)
        pos.copy_(torch.from_numpy(p))
        before.copy_(lens_t(lens))
        after.copy_(lens_t(lens + n))
        graph.replay() if i != 2 else step()
        check(cache, dev, append(cache, x[1], x[2], cu, lens, pairs, p))
        want, tol = attention(cache, qr.double().cpu().numpy(), cu, lens + n, False, hd ** -0.5)
        assert (np.abs(o.double().cpu().numpy() - want) <= tol).all(), i
        lens = lens + n
    assert E_LEAST == -100
