"""Rotary positions with several axes, a paged key/value cache in 8 bits, and the attention that reads it, as cases that can be timed and checked.

Four operators:

* "tables": cos and sin of every (row, pair) from integer positions on up to four axes, as a block's rope_cos / rope_sin.
* "rotate": q and k of a block turned by the same angles (or turned back, which is the gradient).
* "append": new keys (rotated on the way) and values written behind what a paged cache holds, as e4m3 codes with one power of two for
  each 16 tokens of a head.
* "attend": softmax attention of ragged queries over that cache, grouped heads, causal or not.

The cache: positions of a sequence fall into pages (a row of the page table), pages into groups of 16 tokens.
K codes [page][head][group][hd / 16][16 tokens][16 dims], V codes [page][head][group][hd][16 tokens], scales [page][head][group][2]:
a byte b for K and one for V, the codes of the group stand for code * 2^(b - 127).
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
THETA = 10000.0
E_LEAST = -100            # of a group's power of two


# ---------------------------------------------------------------------------------------------------------------------- cases
def _tables(name, rows, hd, axes, far):
    return dict(name=name, op="tables", rows=rows, hd=hd, axes=axes, far=far)


def _rotate(name, rows, heads, kv_heads, hd, axes, far, dtype="bf16", inverse=False):
    return dict(name=name, op="rotate", rows=rows, heads=heads, kv_heads=kv_heads, hd=hd, axes=axes, far=far, dtype=dtype, inverse=inverse)


def _append(name, seqs, new, old, spread, heads, hd, page, axes, dtype="bf16"):
    return dict(name=name, op="append", seqs=seqs, new=new, old=old, spread=spread, heads=heads, hd=hd, page=page, axes=axes, dtype=dtype)


def _attend(name, seqs, q, kv, spread, heads, kv_heads, hd, page, causal=False):
    return dict(name=name, op="attend", seqs=seqs, q=q, kv=kv, spread=spread, heads=heads, kv_heads=kv_heads, hd=hd, page=page, causal=causal)


def listed():
    return [
        # One rank's rows of an image (an eighth of 4608 tokens), two axes: a call whose launch decides.
        _tables("tables_image", 576, 128, "32,32", 64),
        # The video model's rows (half of a 31 x 22 x 40 grid), three axes, late in a long stream.
        _tables("tables_clip", 13640, 128, "22,21,21", 100000),
        # q and k of those rows in one block, all heads.
        _rotate("rotate_clip", 13640, 24, 24, 128, "22,21,21", 100000),
        # Gradients of the image model's rotated q and k, in fp32, fewer key heads, pairs left over that no axis turns.
        _rotate("unrotate_image", 2304, 24, 8, 128, "28,28", 64, "f32", True),
        # One token more for each of a batch of sequences, at odd places of their pages.
        _append("append_tokens", 16, 1, 4011, 0.9, 8, 128, 64, "64"),
        # Three quarters of a clip at once behind a partly filled group, 12 heads: the largest writes.
        _append("append_clip", 1, 20460, 6823, 0.0, 12, 128, 64, "22,21,21"),
        # One query over a short cache of the toy model: nothing but latency.
        _attend("attend_token", 1, 1, 512, 0.0, 8, 8, 64, 16),
        # One token each for a ragged batch, four query heads to a key head.
        _attend("attend_tokens_batch", 32, 1, 8201, 0.8, 32, 8, 128, 64),
        # One token over a very long cache.
        _attend("attend_token_long", 1, 1, 131001, 0.0, 12, 12, 128, 128),
        # Four new latent frames of the video model (880 tokens each) over the clip so far, 12 heads: the most arithmetic.
        _attend("attend_frames", 1, 3520, 27280, 0.0, 12, 12, 128, 64),
        # A ragged batch of prompts, causal, with a prefix that was there already.
        _attend("attend_prompts", 5, 1200, 2711, 0.7, 32, 8, 128, 32, True),
        # A video model's queries over the kept keys and values of its text, all heads.
        _attend("attend_text", 1, 13640, 512, 0.0, 24, 24, 128, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _axes(rng, hd):
    n = rng.choice((1, 2, 3))
    left, pairs = hd // 2 - rng.choice((0, 0, 2, 8)), []
    for i in range(n):
        take = left if i == n - 1 else max(1, left // (n - i))
        pairs.append(take)
        left -= take
    return ",".join(str(p) for p in pairs)


def draw(rng):
    op = rng.choice(("tables", "rotate", "append", "attend", "attend", "attend"))
    hd = rng.choice((64, 128, 128))
    page = rng.choice((16, 32, 64, 128))
    if op == "tables":
        return {k: v for k, v in _tables("", _log(rng, 1, 30000), hd, _axes(rng, hd), _log(rng, 50, 1000000)).items() if k != "name"}
    if op == "rotate":
        heads = rng.choice((3, 8, 12, 24))
        kv = rng.choice([h for h in (1, 2, 3, 4, 8, 12, 24) if heads % h == 0])
        c = _rotate("", _log(rng, 1, 13000), heads, kv, hd, _axes(rng, hd), _log(rng, 50, 1000000), rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.3)
    elif op == "append":
        seqs = _log(rng, 1, 64)
        new = 1 if rng.random() < 0.4 else _log(rng, 2, max(3, 16000 // seqs))
        c = _append("", seqs, new, rng.choice((0, _log(rng, 1, min(8000, 60000 // seqs)))), rng.choice((0.0, 0.5, 0.9)), rng.choice((2, 3, 8, 12)), hd, page,
                    rng.choice(("", _axes(rng, hd))), rng.choice(("bf16", "bf16", "f32")))
    else:
        heads = rng.choice((3, 8, 12, 24, 32))
        kv_heads = rng.choice([h for h in (1, 2, 3, 4, 8, 12, 24) if heads % h == 0 and heads // h <= 16])
        seqs = _log(rng, 1, 48)
        kv = _log(rng, 1, min(120000, 1500000 // (seqs * kv_heads)))           # an attend_token_long at the most
        most = max(1, min(330000 // (seqs * heads), int(1.1e9 / (seqs * kv * heads))))           # an attend_frames or attend_text at the most
        q, causal = rng.choice((1, 1, _log(rng, 1, min(16, most)), _log(rng, 1, most))), rng.random() < 0.5
        q = min(q, kv) if causal else q
        c = _attend("", seqs, q, kv, rng.choice((0.0, 0.5, 0.9)), heads, kv_heads, hd, page, causal)
    return {k: v for k, v in c.items() if k != "name"}


def _ragged(n, seqs, spread):
    """Lengths of a batch: the first n, the others down to n * (1 - spread) in even steps, none under 1 (0 where n is 0)."""
    return [max(min(n, 1), n - int(n * spread * b / max(1, seqs - 1))) for b in range(seqs)]


def _lengths(c):
    """(new tokens or queries, tokens that the cache holds) of each sequence."""
    if c["op"] == "append":
        return _ragged(c["new"], c["seqs"], c["spread"]), _ragged(c["old"], c["seqs"], c["spread"])
    n, held = _ragged(c["q"], c["seqs"], c["spread"]), _ragged(c["kv"], c["seqs"], c["spread"])
    return n, [max(a, b) for a, b in zip(n, held)] if c["causal"] else held


def _pairs(c):
    return [int(p) for p in c["axes"].split(",")] if c["axes"] else []


# ---------------------------------------------------------------------------------------------------------------------- inputs
def _positions(g, rows, axes, far):
    """Rows of a grid whose first axis begins somewhere up to `far`, the others run through a picture of 22 x 40."""
    r = torch.arange(rows, device=DEV)
    first = int(torch.randint(0, far + 1, (1,), generator=g, device=DEV))
    each = [first + r] if axes == 1 else [first + r // 40, r % 40] if axes == 2 else [first + r // 880, r // 40 % 22, r % 40]
    return torch.stack(each, 1).to(torch.int32).contiguous()


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _pool(g, n_pages, heads, groups, hd, which):
    """Codes and powers of a cache that holds something in every slot: channels of different sizes, as keys have them."""
    shape = (n_pages, heads, groups, hd // 16, 16, 16) if which == "k" else (n_pages, heads, groups, hd, 16)
    x = torch.empty(shape, device=DEV).normal_(generator=g)
    channel = torch.empty(hd, device=DEV).normal_(generator=g).mul_(0.4).exp_()
    x *= channel.view(1, 1, 1, hd // 16, 1, 16) if which == "k" else 0.5 * channel.view(1, 1, 1, hd, 1)
    e = torch.ceil(torch.log2(x.abs().flatten(3).amax(3) / 448.0))
    x *= torch.exp2(-e).view(e.shape + (1,) * (x.dim() - 3))
    return x.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _cache(g, c, heads, lens):
    groups, most = c["page"] // 16, max(1, max(-(-n // c["page"]) for n in lens))
    need = [-(-n // c["page"]) for n in lens]
    n_pages = sum(need) + 2
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), most), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    k, ke = _pool(g, n_pages, heads, groups, c["hd"], "k")
    v, ve = _pool(g, n_pages, heads, groups, c["hd"], "v")
    return dict(k_pool=k, v_pool=v, scales=torch.stack((ke, ve), 3).contiguous(), table=table)


def _offsets(n):
    return torch.tensor([0] + [sum(n[:i + 1]) for i in range(len(n))], dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 17)
    c = dict(case)
    if c["op"] in ("tables", "rotate"):
        s = dict(case=c, pos=_positions(g, c["rows"], len(_pairs(c)), c["far"]))
        if c["op"] == "tables":
            s["cos"], s["sin"] = (torch.empty(c["rows"], c["hd"] // 2, device=DEV) for _ in range(2))
        else:
            # q and k as a projection leaves them: columns of one row
            qk = torch.empty(c["rows"], c["heads"] + c["kv_heads"], c["hd"], device=DEV).normal_(generator=g).to(_dtype(c))
            s["q"], s["k"] = qk[:, :c["heads"]], qk[:, c["heads"]:]
            s["q_out"], s["k_out"] = torch.empty_like(s["q"], memory_format=torch.contiguous_format), torch.empty_like(s["k"], memory_format=torch.contiguous_format)
        return s
    n, held = _lengths(c)
    s = dict(case=c, cu=_offsets(n), lens=torch.tensor(held, dtype=torch.int32, device=DEV), most_new=max(n), most_held=max(held))
    if c["op"] == "append":
        s |= _cache(g, c, c["heads"], [a + b for a, b in zip(n, held)])
        s["pos"] = _positions(g, sum(n), len(_pairs(c)), 5000) if c["axes"] else None
        for w in ("k", "v"):
            s[w] = torch.empty(sum(n), c["heads"], c["hd"], device=DEV).normal_(generator=g).to(_dtype(c))
    else:
        s |= _cache(g, c, c["kv_heads"], held)
        s["q"] = torch.empty(sum(n), c["heads"], c["hd"], device=DEV).normal_(generator=g).to(torch.bfloat16)
        s["o"] = torch.empty_like(s["q"])
    return s


# ---------------------------------------------------------------------------------------------------------------------- plain forms
def _cos_sin(c, pos):
    """[rows, hd / 2] each; angles in 64 bits, pairs that belong to no axis at zero."""
    pairs, half = _pairs(c), c["hd"] // 2
    rate = [THETA ** (-j / n) for n in pairs for j in range(n)]
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    rate = torch.tensor(rate + [0.0] * (half - len(rate)), dtype=torch.float64, device=pos.device)
    axis = torch.tensor(axis + [0] * (half - len(axis)), device=pos.device)
    angle = pos[:, axis].double() * rate
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turned(x, cos, sin):
    """Pairs (2p, 2p + 1) of [rows, heads, hd] turned, in 32 bits."""
    a, b = x.float().unflatten(-1, (-1, 2)).unbind(-1)
    cos, sin = cos[:, None], sin[:, None]
    return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)


def _power(m):
    """The smallest e with m <= 224 * 2^e, m half of what has to fit under 448 * 2^e."""
    f, e = torch.frexp(m)
    return torch.where(m > 0, e - 8 + (f > 0.875), E_LEAST).clamp_min(E_LEAST)


def _codes(x, e):
    return torch.ldexp(x, -e).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _append_plain(s):
    c, cu, lens, table = s["case"], s["cu"].long(), s["lens"].long(), s["table"].long()
    page, groups, heads, hd = c["page"], c["page"] // 16, c["heads"], c["hd"]
    k, v = s["k"].float(), s["v"].float()
    halves = 0.5 * k.abs().unflatten(-1, (-1, 2))
    mk = halves.sum(-1).amax(-1) if c["axes"] else halves.amax((-1, -2))
    if c["axes"]:
        k = _turned(k, *_cos_sin(c, s["pos"]))
    need = torch.stack((_power(mk), _power((0.5 * v.abs()).amax(-1))), -1).float()                     # [tokens, heads, 2]
    n_new = cu.diff()
    seq = torch.repeat_interleave(torch.arange(len(n_new), device=cu.device), n_new, output_size=k.shape[0])
    at = lens[seq] + torch.arange(k.shape[0], device=cu.device) - cu[seq]
    pg, grp, slot = table[seq, at // page], at % page // 16, at % 16
    # the largest power that a group's new tokens need, and the one its old tokens have
    e = torch.full((s["scales"].shape[0], groups, heads, 2), -1000.0, device=cu.device)
    e.view(-1, heads * 2).index_reduce_(0, pg * groups + grp, need.reshape(-1, heads * 2), "amax")
    part = lens % 16 > 0
    pg0, grp0 = table[torch.arange(len(lens), device=cu.device), lens // page], lens % page // 16       # (every sequence gets a token)
    old = s["scales"][pg0, :, grp0].float() - 127
    e.view(-1, heads * 2).index_reduce_(0, pg0 * groups + grp0, torch.where(part[:, None, None], old, -1000.0).reshape(-1, heads * 2), "amax")
    # old codes at the new power
    now = e[pg0, grp0]
    kept = part[:, None, None] & (torch.arange(16, device=cu.device) < (lens % 16)[:, None])[:, None]    # [sequences, 1, slots]
    shift = torch.where(part[:, None, None], now - old, 0.0).int()
    kp, vp = s["k_pool"][pg0, :, grp0], s["v_pool"][pg0, :, grp0]
    kq = _codes(kp.view(torch.float8_e4m3fn).float(), shift[:, :, 0, None, None, None])
    vq = _codes(vp.view(torch.float8_e4m3fn).float(), shift[:, :, 1, None, None])
    kp, vp = torch.where(kept[:, :, None, :, None], kq, kp), torch.where(kept[:, :, None], vq, vp)
    s["k_pool"][pg0, :, grp0] = kp
    s["v_pool"][pg0, :, grp0] = vp
    # the new ones
    mine = e[pg, grp].int()
    s["k_pool"][pg, :, grp, :, slot] = _codes(k, mine[..., 0, None]).view(-1, heads, hd // 16, 16)
    s["v_pool"][pg, :, grp, :, slot] = _codes(v, mine[..., 1, None])
    s["scales"][pg, :, grp] = (mine + 127).to(torch.uint8)


def _held(pool, scales, table, which):
    """[sequences, heads, positions, hd] in 32 bits: what a cache stands for."""
    x = pool[table].view(torch.float8_e4m3fn).float()
    x = x * torch.exp2(scales[table][..., which].float() - 127).view(x.shape[:4] + (1,) * (x.dim() - 4))
    x = x.permute(0, 2, 1, 3, 5, 4, 6) if which == 0 else x.permute(0, 2, 1, 3, 5, 4)
    return x.reshape(x.shape[0], x.shape[1], -1, pool.shape[3] * (16 if which == 0 else 1))


def _attend_plain(s):
    c, cu, lens = s["case"], s["cu"].long(), s["lens"].long()
    times = c["heads"] // c["kv_heads"]
    table = s["table"].long().clamp_min(0)
    k, v = (_held(s[p], s["scales"], table, w)[:, :, :s["most_held"]] for w, p in enumerate(("k_pool", "v_pool")))
    n = cu.diff()
    i = torch.arange(s["most_new"], device=cu.device)
    row = (cu[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)                       # padded: a row for each query of the longest
    q = s["q"].float()[row]                                                        # [sequences, queries, heads, hd]
    q = q.unflatten(2, (-1, times)).permute(0, 2, 3, 1, 4).flatten(2, 3)           # [sequences, kv heads, times * queries, hd]
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * (c["hd"] ** -0.5)
    j = torch.arange(k.shape[2], device=cu.device)
    last = (lens - n)[:, None] + i if c["causal"] else (lens - 1)[:, None].expand(-1, len(i))
    seen = (j <= last[..., None]) & (j < lens[:, None, None])                      # [sequences, queries, keys]
    score = score.unflatten(2, (times, -1)).masked_fill_(~seen[:, None, None], -math.inf)
    score = (score - score.amax(-1, keepdim=True)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.flatten(2, 3), v).unflatten(2, (times, -1)) / total
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)                                 # [sequences, queries, heads, hd]
    seq = torch.repeat_interleave(torch.arange(len(n), device=cu.device), n, output_size=s["o"].shape[0])
    s["o"].copy_(out[seq, torch.arange(s["o"].shape[0], device=cu.device) - cu[seq]])


# ---------------------------------------------------------------------------------------------------------------------- a pass
def _kept(s):
    """What a program makes once and keeps: the plan of its positions, the cache's handle, a workspace."""
    from paper_2605_11335_amd import binding as B
    if "kept" not in s:
        c, kept = s["case"], {"B": B}
        if c.get("axes"):
            kept["rope"] = B.cf_rope_plan(c["hd"], _pairs(c), THETA)
        if "k_pool" in s:
            kept["cache"] = B.make_kv_cache(s["k_pool"], s["v_pool"], s["scales"], s["table"])
        if c["op"] == "attend":
            need = B.cf_kv_attention_workspace(kept["cache"], s["q"], s["most_new"])
            kept["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        s["kept"] = kept
    return s["kept"]


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        m = _kept(s)
        B = m["B"]
        if op == "tables":
            B.cf_rope_tables(m["rope"], s["pos"], s["cos"], s["sin"])
        elif op == "rotate":
            B.cf_rope_apply(m["rope"], s["pos"], s["q"], s["q_out"], s["k"], s["k_out"], inverse=s["case"]["inverse"])
        elif op == "append":
            B.cf_kv_append(m["cache"], s["k"], s["v"], s["cu"], s["lens"], m.get("rope"), s["pos"])
        else:
            B.cf_kv_attention(m["cache"], s["q"], s["o"], s["cu"], s["lens"], causal=s["case"]["causal"], max_q=s["most_new"], workspace=m["workspace"])
    elif op == "tables":
        s["cos"], s["sin"] = _cos_sin(s["case"], s["pos"])
    elif op == "rotate":
        cos, sin = _cos_sin(s["case"], s["pos"])
        sin = -sin if s["case"]["inverse"] else sin
        s["q_out"].copy_(_turned(s["q"], cos, sin))
        s["k_out"].copy_(_turned(s["k"], cos, sin))
    elif op == "append":
        _append_plain(s)
    else:
        _attend_plain(s)
    if op == "tables":
        return s["cos"], s["sin"]
    if op == "rotate":
        return s["q_out"], s["k_out"]
    if op == "append":
        return s["k_pool"].view(torch.float8_e4m3fn), s["v_pool"].view(torch.float8_e4m3fn), s["scales"].view(torch.float8_e8m0fnu)
    return s["o"]


def work(case):
    c = case
    if c["op"] == "tables":
        return {"bytes": c["rows"] * (4 * len(_pairs(c)) + 4 * c["hd"]), "flops": c["rows"] * c["hd"] // 2 * 20}
    if c["op"] == "rotate":
        values = c["rows"] * (c["heads"] + c["kv_heads"]) * c["hd"]
        return {"bytes": 2 * values * (2 if c["dtype"] == "bf16" else 4) + 4 * c["rows"] * len(_pairs(c)), "flops": 3 * values}
    n, held = _lengths(c)
    if c["op"] == "append":
        values = 2 * sum(n) * c["heads"] * c["hd"]
        return {"bytes": values * ((2 if c["dtype"] == "bf16" else 4) + 1) + 4 * sum(n) * len(_pairs(c)), "flops": 6 * values}
    seen = sum(a * b - (a * (a - 1) // 2 if c["causal"] else 0) for a, b in zip(n, held))
    return {"bytes": 2 * sum(held) * c["kv_heads"] * (c["hd"] + 1 / 16) + 4 * sum(n) * c["heads"] * c["hd"], "flops": 4 * seen * c["heads"] * c["hd"]}


# ---------------------------------------------------------------------------------------------------------------------- 64 bits
def _angles64(c, pos):
    out = torch.zeros(pos.shape[0], c["hd"] // 2, dtype=torch.float64, device=pos.device)
    p = 0
    for a, n in enumerate(_pairs(c)):
        for j in range(n):
            out[:, p] = pos[:, a].double() / THETA ** (j / n)
            p += 1
    return out


def _turn64(x, angle):
    z = torch.view_as_complex(x.double().unflatten(-1, (-1, 2)).contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.view_as_real(z).flatten(-2)


def _power64(m):
    e = torch.ceil(torch.log2(m / 448.0)).clamp_min(E_LEAST)
    e = torch.where(448.0 * torch.exp2(e) < m, e + 1, e)
    return torch.where((448.0 * torch.exp2(e - 1) >= m) & (e > E_LEAST), e - 1, e)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "tables":
        a = _angles64(c, s["pos"])
        return torch.cos(a), torch.sin(a)
    if c["op"] == "rotate":
        a = _angles64(c, s["pos"])
        a = -a if c["inverse"] else a
        return _turn64(s["q"], a), _turn64(s["k"], a)
    cu, lens, table, page, hd = s["cu"].tolist(), s["lens"].tolist(), s["table"].tolist(), c["page"], c["hd"]
    k = s["k_pool"].view(torch.float8_e4m3fn).double()
    v = s["v_pool"].view(torch.float8_e4m3fn).double()
    p = s["scales"].double() - 127
    if c["op"] == "append":
        x, y = s["k"].double(), s["v"].double()
        mk = x.abs().unflatten(-1, (-1, 2)).sum(-1).amax(-1) if c["axes"] else x.abs().amax(-1)
        my = y.abs().amax(-1)
        if c["axes"]:
            x = _turn64(x, _angles64(c, s["pos"]))
        for b in range(len(lens)):
            at, end = lens[b], lens[b] + cu[b + 1] - cu[b]
            if end - at > 4096:           # whole pages of a long run at once
                long = end // page * page - -(-at // page) * page
            else:
                long = 0
            if long > 0:
                lo = -(-at // page) * page
                r = slice(cu[b] + lo - at, cu[b] + lo - at + long)
                pages = torch.tensor(table[b][lo // page:(lo + long) // page], device=DEV)
                blocks = lambda t: t[r].unflatten(0, (len(pages), page // 16, 16))             # noqa: E731
                ek, ey = _power64(blocks(mk).amax(2)).transpose(1, 2), _power64(blocks(my).amax(2)).transpose(1, 2)     # [pages, heads, groups]
                p[pages] = torch.stack((ek, ey), -1)
                k[pages] = (blocks(x).permute(0, 3, 1, 2, 4) / torch.exp2(ek)[..., None, None]).unflatten(-1, (hd // 16, 16)).transpose(3, 4)
                v[pages] = (blocks(y).permute(0, 3, 1, 2, 4) / torch.exp2(ey)[..., None, None]).transpose(3, 4)
            while at < end:
                if long > 0 and at == lo:
                    at += long
                    continue
                upto = min(end, (at // 16 + 1) * 16)
                r = slice(cu[b] + at - lens[b], cu[b] + upto - lens[b])
                pg, g, a0, a1 = table[b][at // page], at % page // 16, at % 16, (upto - 1) % 16 + 1
                for which, (pool, new, m) in enumerate(((k, x, mk), (v, y, my))):
                    e = _power64(m[r].amax(0))
                    e = torch.maximum(e, p[pg, :, g, which]) if a0 else e
                    was = torch.exp2(p[pg, :, g, which] - e)
                    q = new[r] / torch.exp2(e)[:, None]
                    if which == 0:
                        pool[pg, :, g, :, :a0] *= was[:, None, None, None]
                        pool[pg, :, g, :, a0:a1] = q.unflatten(-1, (hd // 16, 16)).permute(1, 2, 0, 3)
                    else:
                        pool[pg, :, g, :, :a0] *= was[:, None, None]
                        pool[pg, :, g, :, a0:a1] = q.permute(1, 2, 0)
                    p[pg, :, g, which] = e
                at = upto
        return k, v, torch.exp2(p)
    k, v = k * torch.exp2(p[..., 0])[..., None, None, None], v * torch.exp2(p[..., 1])[..., None, None]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, held in enumerate(lens):
        pages = torch.tensor(table[b][:-(-held // page)], device=DEV)
        n = cu[b + 1] - cu[b]
        for h in range(c["kv_heads"]):
            kk = k[pages, h].transpose(2, 3).reshape(-1, hd)[:held]                # [pages, groups, tokens, chunks, 16]
            vv = v[pages, h].transpose(2, 3).reshape(-1, hd)[:held]
            for t in range(c["heads"] // c["kv_heads"]):
                at = h * (c["heads"] // c["kv_heads"]) + t
                z = s["q"][cu[b]:cu[b + 1], at].double() @ kk.t().contiguous() / math.sqrt(hd)
                if c["causal"]:
                    z += torch.full_like(z, -math.inf).triu(held - n + 1)
                out[cu[b]:cu[b + 1], at] = torch.softmax(z, -1) @ vv
    return out
