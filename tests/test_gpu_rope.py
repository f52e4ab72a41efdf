"""Rotary tables, and q and k turned by several axes' positions, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import workload as wl
from oracle import block as ob
from paper_2605_11335_amd import binding as B
from paper_2605_11335_amd.runner import BlockRunner
from tests.util import max_abs, rel_l2

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ULP = 2.0 ** -24
# cos and sin: angle to 2^-33 turns, its conversion, factor and product (2^-25 rad and two roundings of at most pi / 4), the series and
# its last sum (2 roundings of values up to 1): 2.3e-8 + 9.4e-8 + 1.2e-7 < 4 * 2^-24
TABLE_TOL = 4 * ULP
AXES = {64: ([32], [10, 11, 9], [16, 16], [1, 2, 3, 4]), 128: ([64], [22, 21, 21], [28, 28], [16, 16, 16, 16])}


def positions(rng, n, axes):
    pos = rng.integers(-50, 2000, size=(n, axes))
    far = np.array([0, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6, 123456789])
    pos[rng.integers(0, n, size=6), rng.integers(0, axes, size=6)] = far
    return pos.astype(np.int32)


def angles(pos, pairs, hd, theta=10000.0):
    a, p = np.zeros((pos.shape[0], hd // 2), np.longdouble), 0
    for axis, m in enumerate(pairs):
        for j in range(m):
            a[:, p] = pos[:, axis].astype(np.longdouble) * np.power(np.longdouble(theta), -np.longdouble(j) / m)
            p += 1
    return a


def turned(x, a):
    """[n, heads, hd] in 64 bits."""
    c, s = np.cos(a).astype(np.float64)[:, None], np.sin(a).astype(np.float64)[:, None]
    out = np.empty_like(x)
    out[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    out[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    return out


def bound(x, want, dtype):
    """Both coefficients off by TABLE_TOL, two roundings in fp32, half a step of the result's type."""
    pair = np.repeat(np.abs(x[..., 0::2]) + np.abs(x[..., 1::2]), 2, axis=-1)
    return pair * (TABLE_TOL + 2 * ULP) + torch.finfo(dtype).eps / 2 * np.abs(want)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("n", [1, 7, 333])
def test_tables(hd, which, n):
    pairs = AXES[hd][which]
    rng = np.random.default_rng(hd + 10 * which + n)
    pos = positions(rng, n, len(pairs))
    cos, sin = (torch.full((n + 1, hd // 2), 7.0, device=DEV) for _ in range(2))
    B.cf_rope_tables(B.cf_rope_plan(hd, pairs), torch.from_numpy(pos).to(DEV), cos[:n], sin[:n])
    torch.cuda.synchronize()
    a = angles(pos, pairs, hd)
    assert np.abs(cos[:n].cpu().numpy() - np.cos(a)).max() <= TABLE_TOL and np.abs(sin[:n].cpu().numpy() - np.sin(a)).max() <= TABLE_TOL
    assert (cos[n] == 7).all() and (sin[n] == 7).all()          # the row behind stays
    assert sum(pairs) == hd // 2 or (cos[:n, sum(pairs):] == 1).all() and (sin[:n, sum(pairs):] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,heads,kv_heads", [(1, 1, 0), (1, 3, 1), (5, 12, 4), (37, 24, 24), (300, 17, 2), (2, 130, 1)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation(dtype, hd, n, heads, kv_heads, inverse):
    pairs = AXES[hd][(n + heads) % 4]
    rng = np.random.default_rng(n * 100 + heads + hd)
    pos = positions(rng, n, len(pairs))
    plan, p = B.cf_rope_plan(hd, pairs), torch.from_numpy(pos).to(DEV)
    # q and k as columns of one row, with a column between them that is nobody's
    buf = torch.from_numpy(rng.normal(size=(n, heads + 1 + kv_heads, hd)).astype(np.float32)).to(DEV).to(dtype)
    q, k = buf[:, :heads], buf[:, heads + 1:]
    a = angles(pos, pairs, hd) * (-1 if inverse else 1)
    want = [turned(t.double().cpu().numpy(), a) for t in (q, k)]
    tol = [bound(t.double().cpu().numpy(), w, dtype) for t, w in zip((q, k), want)]
    # q's output head after head, k's row after row
    q_out, k_out = torch.full((heads, n + 1, hd), 3.0, device=DEV, dtype=dtype), torch.full((n + 1, kv_heads, hd), 3.0, device=DEV, dtype=dtype)
    qo, ko = q_out[:, :n].transpose(0, 1), k_out[:n]
    args = (k, ko) if kv_heads else (None, None)
    B.cf_rope_apply(plan, p, q, qo, *args, inverse=inverse)
    torch.cuda.synchronize()
    assert (np.abs(qo.double().cpu().numpy() - want[0]) <= tol[0]).all() and (q_out[:, n] == 3).all()
    if kv_heads:
        assert (np.abs(ko.double().cpu().numpy() - want[1]) <= tol[1]).all() and (k_out[n] == 3).all()
    # in place: the same bits, and nothing beside them touched
    was = buf.clone()
    B.cf_rope_apply(plan, p, q, q, *((k, k) if kv_heads else (None, None)), inverse=inverse)
    torch.cuda.synchronize()
    assert torch.equal(q, qo) and (not kv_heads or torch.equal(k, ko)) and torch.equal(buf[:, heads], was[:, heads])


def test_the_inverse_is_the_gradient():
    """L = sum(w * y(x)): its gradient by the inverse, by the formula in 64 bits and by differences (y is linear in x, so any step does)."""
    n, heads, hd, pairs = 9, 3, 128, [22, 21, 21]
    rng = np.random.default_rng(5)
    pos = positions(rng, n, 3)
    plan, p = B.cf_rope_plan(hd, pairs), torch.from_numpy(pos).to(DEV)
    x, w = (torch.from_numpy(rng.normal(size=(n, heads, hd)).astype(np.float32)).to(DEV) for _ in range(2))
    g, y = torch.empty_like(x), torch.empty_like(x)
    B.cf_rope_apply(plan, p, w, g, inverse=True)
    a = angles(pos, pairs, hd)
    w64 = w.double().cpu().numpy()
    want = turned(w64, -a)
    assert (np.abs(g.double().cpu().numpy() - want) <= bound(w64, want, torch.float32)).all()

    def loss(x):
        B.cf_rope_apply(plan, p, x, y)
        return float((w.double() * y.double()).sum())

    for at in [(0, 0, 0), (4, 1, 77), (8, 2, 127), (3, 0, 64)]:
        hi, lo = x.clone(), x.clone()
        hi[at] += 4.0
        lo[at] -= 4.0
        step = float(hi[at]) - float(lo[at])
        # each of the two outputs that differ is off by bound() of values up to |x| + 4 + |partner| < 12, on both sides, times |w|
        tol = 2 * 2 * 12 * (TABLE_TOL + 3 * ULP) * float(w.abs().max()) / step
        assert abs((loss(hi) - loss(lo)) / step - float(g[at])) <= tol + 12 * (TABLE_TOL + 3 * ULP)


def test_broadcast_input_and_strides_past_32_bits():
    hd, plan = 64, B.cf_rope_plan(64, [32])
    p = torch.tensor([[3], [-9], [100000]], dtype=torch.int32, device=DEV)
    row = torch.randn(1, 1, hd, device=DEV, dtype=torch.bfloat16)
    dense, got = torch.empty(3, 5, hd, device=DEV, dtype=torch.bfloat16), torch.empty(3, 5, hd, device=DEV, dtype=torch.bfloat16)
    B.cf_rope_apply(plan, p, row.expand(3, 5, hd).contiguous(), dense)
    B.cf_rope_apply(plan, p, row.expand(3, 5, hd), got)
    assert torch.equal(dense, got)
    far = torch.empty(2 * (1 << 31) + 5 * hd, device=DEV, dtype=torch.bfloat16).as_strided((3, 5, hd), (1 << 31, hd, 1))
    far.copy_(row.expand(3, 5, hd))
    B.cf_rope_apply(plan, p, far, far)
    assert torch.equal(dense, far)


def test_another_stream_and_a_captured_graph():
    n, heads, hd = 40, 6, 128
    plan = B.cf_rope_plan(hd, [32, 32])
    p = torch.randint(-100, 100, (n, 2), dtype=torch.int32, device=DEV)
    x, want, y = torch.randn(n, heads, hd, device=DEV), torch.empty(n, heads, hd, device=DEV), torch.empty(n, heads, hd, device=DEV)
    cos, sin, c2, s2 = (torch.empty(n, hd // 2, device=DEV) for _ in range(4))
    B.cf_rope_apply(plan, p, x, want)
    B.cf_rope_tables(plan, p, cos, sin)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.cf_rope_apply(plan, p, x, y, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cf_rope_apply(plan, p, x, y)
        B.cf_rope_tables(plan, p, c2, s2)
    for i in range(3):
        x.normal_()
        p += i
        y.zero_()
        B.cf_rope_apply(plan, p, x, want)
        B.cf_rope_tables(plan, p, cos, sin)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(c2, cos) and torch.equal(s2, sin)


def test_a_block_over_positions_on_three_axes():
    """Tables made from (time, height, width) as a block's rope_cos and rope_sin: the block against the oracle with tables in 64 bits."""
    cfg = wl.BlockConfig("rope_axes", wl.KIND_DIT, n_blocks=1, d=512, n_heads=4, head_dim=128, f=1024, n_total=588, sp_degree=2, sp_rank=0, l_ctx=77,
                         qk_rmsnorm=True, n_chunks=6, rope=True)
    params, inputs = wl.gen_block_params(cfg, 0), wl.gen_block_inputs(cfg, 0)
    r = np.arange(cfg.n_local)
    pos = np.stack([5000 + r // 84, r // 12 % 7, r % 12], 1).astype(np.int32)
    a = angles(pos, [22, 21, 21], 128)
    inputs["rope_cos"], inputs["rope_sin"] = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
    run = BlockRunner(cfg)
    try:
        run.register_params(0, params)
        t = run.make_io({k: v for k, v in inputs.items() if not k.startswith("rope_")})
        t.update(run.rope_tables(B.cf_rope_plan(128, [22, 21, 21]), torch.from_numpy(pos).to(DEV)))
        run.run_block(0, t)
        want = ob.block_forward(cfg, params, inputs)["y"]
        got = t["y"].cpu().numpy()
        print(f"rel_l2={rel_l2(got, want):.3e} max_abs={max_abs(got, want):.3e}", flush=True)
        assert rel_l2(got, want) <= 1e-2 and max_abs(got, want) <= 5e-2
        with pytest.raises(B.ChunkflowError):
            run.rope_tables(B.cf_rope_plan(128, [64]), torch.zeros(5, 1, dtype=torch.int32, device=DEV))
    finally:
        run.close()


@pytest.mark.parametrize("dtype,hd,heads", [(torch.bfloat16, 64, 17), (torch.bfloat16, 128, 8), (torch.float32, 64, 5), (torch.float32, 128, 3)])
def test_operands_that_caches_do_not_hold(dtype, hd, heads):
    """Outputs of more than 64 MiB, which go past the caches: the bits of the same rows a few at a time."""
    n = (68 << 20) // (heads * hd * dtype.itemsize) + 5
    plan = B.cf_rope_plan(hd, [hd // 4, hd // 8])
    p = torch.randint(-1000, 1000000, (n, 2), dtype=torch.int32, device=DEV)
    x = torch.randn(n, heads, hd, device=DEV).to(dtype)
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    B.cf_rope_apply(plan, p, x, whole)
    for i in range(0, n, n // 3 + 1):
        B.cf_rope_apply(plan, p[i:i + n // 3 + 1], x[i:i + n // 3 + 1], parts[i:i + n // 3 + 1])
    assert torch.equal(whole, parts)
    B.cf_rope_apply(plan, p, x, x)
    assert torch.equal(whole, x)
