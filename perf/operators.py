"""The operators on cached rows -- storing them in 4 bits and loading them, attention over them, copying them -- as cases
that can be timed and compared: in plain torch (own = False), and through the library (own = True).

A 4-bit row holds, for every kv head, head_dim codes of 4 bits (sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; element 2i in
the low half of byte i) and one exponent byte E for each 32 channels; a value is code * 2^(E - 127).  E - 127 is the
largest magnitude's exponent less 2, or less 1 where the magnitude is over 1.75 times its power of two, between -125 and
125; codes round to nearest, ties to the even code, at most 6.

Keys, values and queries are N(0, 1), the distribution that the library's seeded layers produce.  A case's lengths come
from its own "lengths" number inside the [min, max] ranges, its tensors from prepare()'s seed.
"""
from __future__ import annotations

import functools
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32
GAP = 5                  # unused rows behind every region of a pool
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

# The layer of the cases is the 8B-class one of paper_2504_12397_amd/workloads.py (32 query heads in 8 groups, head size 128, bf16), or the
# fp32 block of its tests (4 heads of 64) and odd relatives of it.
BASE = dict(dtype="bf16", q=32, kv=8, h=128, layers=1, lengths=1)


def _store(name, ranges, rows_min, rows_max, **kw):
    return dict(BASE, op="store", name=name, ranges=ranges, rows_min=rows_min, rows_max=rows_max, **kw)


def _copy(name, ranges, rows_min, rows_max, **kw):
    return dict(BASE, op="copy", name=name, ranges=ranges, rows_min=rows_min, rows_max=rows_max, bits=16, forks=0, **kw)


def _attend(name, sequences, cached, new=(1, 1), contexts=0, context=0, **kw):
    return dict(BASE, op="attend", name=name, sequences=sequences, contexts=contexts, context=context, cached_min=cached[0],
                cached_max=cached[1], new_min=new[0], new_max=new[1], **kw)


def listed():
    return [
        # the new rows of a decode step of 64 sequences go into a 4-bit cache and are read back: latency
        _store("store_step_rows", 64, 1, 1),
        # a finished context of 16384 tokens is parked in 4 bits in eight layers, and taken up again
        _store("store_context", 1, 16384, 16384, layers=8),
        # fp32 rows of an odd head size (the last block of a head has 16 channels), ragged ranges
        _store("store_odd_f32", 7, 1, 900, dtype="f32", kv=5, h=80, lengths=3),
        # the last few rows of a conversation are forked for another adapter and closed up to the rows before them, in 32 layers: latency
        _copy("copy_fork_rows", 1, 17, 17, layers=32),
        # four adapters fork a context of 8192 rows in eight layers
        dict(_copy("copy_fork_context", 1, 8192, 8192, layers=8), forks=4),
        # a 4-bit pool is moved to another pool and closed up there in place, sequences of ragged lengths; its values are read
        dict(_copy("copy_compact_4bit", 24, 100, 6000, layers=4, lengths=5), bits=4),
        # five short conversations decode one token each: latency
        _attend("attend_step_short", 5, (0, 200), lengths=2),
        # a full serving batch decodes one token each over 16448 cached rows
        _attend("attend_step_batch", 64, (16448, 16448)),
        # one sequence decodes over a very long context
        _attend("attend_step_long", 1, (131070, 131070)),
        # eight adapters answer over one shared context of 32768 rows, some tokens each
        _attend("attend_adapters", 8, (0, 40), new=(9, 23), contexts=1, context=32768, lengths=4),
        # a suffix of 128 tokens is prefilled over a cached context
        _attend("attend_prefill", 1, (32768, 32768), new=(128, 128)),
        # the fp32 block of the tests, ragged sequences and suffixes
        _attend("attend_f32", 6, (1, 3000), new=(1, 30), dtype="f32", q=4, kv=4, h=64, lengths=6),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["store", "copy", "attend", "attend"])
    shape = rng.choice([dict(), dict(), dict(q=8, kv=2), dict(q=16, kv=16), dict(q=24, kv=8, h=64), dict(dtype="f32", q=4, kv=4, h=64),
                        dict(dtype="f32", q=10, kv=5, h=80), dict(q=20, kv=4, h=48)])
    c = dict(BASE, op=op, **shape)
    c["lengths"] = rng.randrange(1, 1 << 20)
    cost = c["kv"] * c["h"] / 1024 * (2 if c["dtype"] == "f32" else 1)
    if op == "attend":
        plain = c["dtype"] == "f32" or c["h"] % 64 != 0
        c["sequences"] = _spread(rng, 1, 64)
        c["contexts"] = rng.choice([0, 0, 1, 2]) if c["sequences"] > 1 else 0
        room = (60000 if plain else 500000) / max(1.0, cost) / c["sequences"]
        c["context"] = _spread(rng, 20, max(21, min(32768, int(room)))) if c["contexts"] else 0
        new = 1 if rng.random() < 0.5 else _spread(rng, 2, 160 if c["sequences"] < 9 else 24)
        c["new_min"], c["new_max"] = max(1, new // 3), new
        left = max(1, min(16384 if c["contexts"] else 131072, int(room) - c["context"]))
        c["cached_max"] = _spread(rng, 1, left)
        c["cached_min"] = rng.choice([0, c["cached_max"] // 2, c["cached_max"]])
    else:
        c["layers"] = _spread(rng, 1, 16)
        c["ranges"] = _spread(rng, 1, 64)
        most = max(2, int(100000 / max(1.0, cost) / c["layers"] / c["ranges"]))
        c["rows_max"] = _spread(rng, 1, min(16384, most))
        c["rows_min"] = max(1, rng.choice([1, c["rows_max"] // 2, c["rows_max"]]))
        if op == "copy":
            c["bits"] = rng.choice([16, 4])
            c["forks"] = rng.choice([0, 0, 2, 3]) if c["ranges"] <= 16 else 0
    return c


def _between(case, name, n):
    rng = random.Random("%d %s" % (case["lengths"], name))
    lo, hi = {"rows": ("rows_min", "rows_max"), "cached": ("cached_min", "cached_max"), "new": ("new_min", "new_max")}[name]
    return [rng.randint(case[lo], case[hi]) for _ in range(n)]


def _move_plan(case):
    """Ranges (source row, destination row, rows) of a store or copy, and the rows of the two pools.

    Ranges lie behind one another with gaps in the source, and close together, in another order, in the destination.  Forks: every range goes to
    that many places.  A copy without forks is followed by a second one that closes the destination up in place, where the ranges
    begin GAP rows from each other and overlap where they were."""
    n = case["ranges"]
    rows = _between(case, "rows", n)
    order = list(range(n))
    random.Random("%d order" % case["lengths"]).shuffle(order)
    src = [GAP * (i + 1) + sum(rows[:i]) for i in range(n)]
    forks = max(1, case.get("forks", 0))
    first, second, at, packed = [], [], GAP, 0
    for i in order:
        for _ in range(forks):
            first.append((src[i], at, rows[i]))
            second.append((at, packed, rows[i]))
            at += rows[i] + GAP
            packed += rows[i]
    total = sum(rows) + GAP * (n + 1)
    again = case["op"] == "copy" and not case.get("forks", 0)
    return np.array(first, dtype=np.int64), np.array(second if again else [], dtype=np.int64).reshape(-1, 3), total, at


def _attend_plan(case):
    """The pool rows of every sequence: a shared prefix (or none), then its own rows, the new ones last."""
    B, C = case["sequences"], case["contexts"]
    cached, new = _between(case, "cached", B), _between(case, "new", B)
    at = C * (case["context"] + GAP)
    off = []
    for c, n in zip(cached, new):
        off.append(at)
        at += c + n + GAP
    ctx = [b * C // B for b in range(B)] if C else [0] * B
    return dict(new=np.array(new), own=np.array(cached) + np.array(new), off=np.array(off, dtype=np.int64), rows=at,
                plen=np.full(B, case["context"] if C else 0, dtype=np.int32),
                poff=np.array([x * (case["context"] + GAP) for x in ctx], dtype=np.int64),
                live=[(x * (case["context"] + GAP), case["context"]) for x in range(C)] + [(o, c + n) for o, c, n in zip(off, cached, new)])


def _normal(gen, shape, dtype):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat, step = out.view(-1), 1 << 26
    for lo in range(0, flat.numel(), step):
        n = min(step, flat.numel() - lo)
        flat[lo:lo + n] = torch.randn(n, generator=gen, device=DEV).to(dtype)
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt, kv, h = DTYPES[case["dtype"]], case["kv"], case["h"]
    state = dict(case=case)
    if case["op"] == "attend":
        p = _attend_plan(case)
        state["plan"] = p
        state["q"] = _normal(gen, (int(p["new"].sum()), case["q"] * h), dt)
        state["cu"] = np.concatenate([[0], np.cumsum(p["new"])]).astype(np.int32)
        for x in "kv":
            codes = torch.zeros((p["rows"], kv, h // 2), dtype=torch.uint8, device=DEV)
            scale = torch.full((p["rows"], kv, (h + BLOCK - 1) // BLOCK), 127, dtype=torch.uint8, device=DEV)
            for at, n in p["live"]:
                for lo in range(at, at + n, 16384):
                    hi = min(at + n, lo + 16384)
                    codes[lo:hi], scale[lo:hi] = _quantise(torch.randn((hi - lo, kv, h), generator=gen, device=DEV))
            state[x], state[x + "_scale"] = codes, scale
        return state
    first, second, n_src, n_dst = _move_plan(case)
    state.update(first=first, second=second, n_src=n_src, n_dst=n_dst)
    shape = (case["layers"], n_src, kv, h)
    for x in "kv":
        src = _normal(gen, shape, dt)
        if case["op"] == "copy" and case["bits"] == 4:
            state["src_" + x], state["src_" + x + "_scale"] = _quantise(src.float())
        else:
            state["src_" + x] = src
        # what comes back lands here; rows that no range names keep this
        state["dst_" + x] = torch.full((case["layers"], n_dst, kv, h), 0.75, dtype=dt, device=DEV)
        state["mid_" + x] = torch.zeros((case["layers"], n_dst, kv, h // 2), dtype=torch.uint8, device=DEV)
        state["mid_" + x + "_scale"] = torch.full((case["layers"], n_dst, kv, (h + BLOCK - 1) // BLOCK), 127, dtype=torch.uint8, device=DEV)
    return state


# ---- plain forms --------------------------------------------------------------------------------------------------
def _quantise(x):
    """fp32 [..., h] -> codes [..., h / 2], exponents [..., ceil(h / 32)]."""
    h = x.shape[-1]
    blocks = torch.nn.functional.pad(x, (0, -h % BLOCK)).unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(blocks.abs().amax(-1))                      # amax = m 2^e, m in [0.5, 1)
    ex = (e - 3 + (m > 0.875)).clamp(-125, 125)
    ex = torch.where(m == 0, torch.full_like(ex, -125), ex)
    y = torch.ldexp(blocks, -ex.unsqueeze(-1))
    a = y.abs()
    step = 0.5 + 0.5 * (a >= 2) + (a >= 4)
    a = torch.clamp(torch.round(a / step) * step, max=6)           # (round: ties to even)
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, 4 + a / 2)).to(torch.uint8)
    code = (code + 8 * torch.signbit(y)).flatten(-2)[..., :h]
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), (ex + 127).to(torch.uint8)


@functools.lru_cache(maxsize=None)
def _pairs():
    """The two values of every byte."""
    v = [s * x for s in (1, -1) for x in LEVELS]
    return torch.tensor([[v[b & 15], v[b >> 4]] for b in range(256)], dtype=torch.float32, device=DEV)


def _values(codes, scale):
    """codes [..., h / 2], exponents [..., ceil(h / 32)] -> fp32 [..., h]."""
    v = _pairs()[codes.long()].flatten(-2)
    s = torch.ldexp(torch.ones_like(scale, dtype=torch.float32), scale.int() - 127)
    return v * s.repeat_interleave(BLOCK, dim=-1)[..., :v.shape[-1]]


def _rows(ranges, column):
    return torch.from_numpy(np.concatenate([np.arange(r[column], r[column] + r[2]) for r in ranges])).to(DEV)


def _plain_store(s):
    i, j = _rows(s["first"], 0), _rows(s["first"], 1)
    for_k, for_v = (_values(*_quantise(s["src_" + x][:, i].float())) for x in "kv")
    s["dst_k"][:, j] = for_k.to(s["dst_k"].dtype)
    s["dst_v"][:, j] = for_v.to(s["dst_v"].dtype)
    return s["dst_k"], s["dst_v"]


def _plain_copy(s):
    four = s["case"]["bits"] == 4
    names = ("k", "v", "k_scale", "v_scale") if four else ("k", "v")
    to = "mid_" if four else "dst_"
    i, j = _rows(s["first"], 0), _rows(s["first"], 1)
    [s[to + x].index_copy_(1, j, s["src_" + x].index_select(1, i)) for x in names]
    if len(s["second"]):
        i, j = _rows(s["second"], 0), _rows(s["second"], 1)
        [s[to + x].index_copy_(1, j, s[to + x].index_select(1, i)) for x in names]
    if four:
        return tuple(_values(s["mid_" + x], s["mid_" + x + "_scale"]).to(s["dst_" + x].dtype) for x in "kv")
    return s["dst_k"], s["dst_v"]


def _plain_attend(s):
    c, p = s["case"], s["plan"]
    B, kv, h, G = c["sequences"], c["kv"], c["h"], c["q"] // c["kv"]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)[:, None]  # noqa: E731
    plen, poff, off, n_own, new, first = (dev(a) for a in (p["plen"], p["poff"], p["off"], p["own"], p["new"], s["cu"][:-1]))
    length = plen + n_own
    pos = torch.arange(int((p["plen"] + p["own"]).max()), device=DEV)[None]
    row = torch.where(pos < plen, poff + pos, off + torch.minimum(pos - plen, n_own - 1))      # [B, L] pool rows
    i = torch.arange(int(p["new"].max()), device=DEV)[None]
    valid = i < new                                                                            # [B, S]
    q = s["q"].float()[first + torch.minimum(i, new - 1)].view(B, -1, kv, G, h).permute(0, 2, 3, 1, 4).flatten(2, 3)
    k = _values(s["k"][row], s["k_scale"][row]).permute(0, 2, 3, 1)
    sc = (torch.matmul(q, k) / math.sqrt(h)).view(B, kv, G, i.shape[1], -1)
    del k
    sees = pos[:, None] <= (length - new + i)[:, :, None]                                      # [B, S, L]
    sc = sc.masked_fill(~sees[:, None, None], -math.inf)
    e = torch.exp(sc - sc.amax(-1, keepdim=True))
    v = _values(s["v"][row], s["v_scale"][row]).transpose(1, 2)
    o = torch.matmul(e.flatten(2, 3), v).view(B, kv, G, i.shape[1], h) / e.sum(-1, keepdim=True)
    return o.permute(0, 3, 1, 2, 4).flatten(2)[valid].to(s["q"].dtype)


# ---- through the library ------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _context():
    from paper_2504_12397_amd import binding as ab
    return ab.Context(0)


def _handles(s):
    """The cache objects of a program, which wrap its tensors."""
    from paper_2504_12397_amd import binding as ab
    c = s["case"]
    if c["op"] == "attend":
        p = s["plan"]
        return ab.QCache.from_tensors(s["k"], s["v"], s["k_scale"], s["v_scale"], seq_offset=p["off"], seq_capacity=p["own"],
                                      seq_len=p["own"] + p["plen"], prefix_offset=p["poff"], prefix_len=p["plen"])
    rows = lambda to: [ab.KVCache.from_tensors(k, v) for k, v in zip(s[to + "_k"], s[to + "_v"])]  # noqa: E731
    four = lambda to: [ab.QCache.from_tensors(*t) for t in zip(*(s[to + x] for x in ("_k", "_v", "_k_scale", "_v_scale")))]  # noqa: E731
    src = four("src") if c["op"] == "copy" and c["bits"] == 4 else rows("src")
    return src, four("mid"), rows("dst")


def _own(s):
    from paper_2504_12397_amd import binding as ab
    c, ctx = s["case"], _context()
    if "handles" not in s:
        s["handles"] = _handles(s)
    if c["op"] == "attend":
        return ab.alora_qcache_attend(ctx, s["handles"], s["q"], s["cu"], c["q"])
    src, mid, dst = s["handles"]
    if c["op"] == "store":
        ab.alora_qcache_store(ctx, mid, src, s["first"])
        stored = s["first"][:, [1, 1, 2]]
        ab.alora_qcache_load(ctx, dst, mid, stored)
    elif c["bits"] == 4:
        ab.alora_qcache_copy(ctx, mid, src, s["first"])
        if len(s["second"]):
            ab.alora_qcache_copy(ctx, mid, mid, s["second"])
        ab.alora_qcache_load(ctx, dst, mid, [(0, 0, s["n_dst"])])
    else:
        ab.alora_cache_copy(ctx, dst, src, s["first"])
        if len(s["second"]):
            ab.alora_cache_copy(ctx, dst, dst, s["second"])
    return s["dst_k"], s["dst_v"]


def run(state):
    if own:
        return _own(state)
    return {"store": _plain_store, "copy": _plain_copy, "attend": _plain_attend}[state["case"]["op"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    kv, h = case["kv"], case["h"]
    full = 2 * kv * h * (4 if case["dtype"] == "f32" else 2)                # bytes of a token's key and value
    four = 2 * kv * (h // 2 + (h + BLOCK - 1) // BLOCK)                     # ... in 4 bits
    if case["op"] == "attend":
        p = _attend_plan(case)
        esz = 4 if case["dtype"] == "f32" else 2
        keys = int(p["own"].sum()) + case["contexts"] * case["context"]
        seen = int(((p["plen"] + p["own"]) * p["new"] - p["new"] * (p["new"] - 1) // 2).sum())
        return {"bytes": keys * four + 2 * int(p["new"].sum()) * case["q"] * h * esz, "flops": 4.0 * case["q"] * h * seen}
    first, second, n_src, n_dst = _move_plan(case)
    rows, again = int(first[:, 2].sum()), int(second[:, 2].sum())
    src = rows // max(1, case.get("forks", 0))                             # (distinct rows read)
    if case["op"] == "store":
        b = rows * 2 * (full + four)
    elif case["bits"] == 4:
        b = (src + rows + 2 * again) * four + n_dst * (four + full)
    else:
        b = (src + rows + 2 * again) * full
    return {"bytes": b * case["layers"], "flops": 0.0 if case["op"] == "copy" else 4.0 * rows * kv * h * case["layers"]}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------
def _levels64(codes, exponents, h):
    """Values of 4-bit rows, code by code from the definition."""
    out = torch.empty(codes.shape[:-1] + (h,), dtype=torch.float64, device=codes.device)
    table = torch.tensor(LEVELS, dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        c = (codes >> (4 * half)) & 15
        out[..., half::2] = table[(c & 7).long()] * (1.0 - 2.0 * (c >> 3).double())
    for n in range(exponents.shape[-1]):
        out[..., n * BLOCK:(n + 1) * BLOCK] *= torch.exp2(exponents[..., n:n + 1].double() - 127)
    return out


def _round64(x):
    """Values that 4-bit rows of x stand for: thresholds between the levels, a tie to the even code."""
    x = x.double()
    out = torch.empty_like(x)
    for lo in range(0, x.shape[-1], BLOCK):
        b = x[..., lo:lo + BLOCK]
        top = b.abs().amax(-1, keepdim=True)
        e = torch.floor(torch.log2(top.clamp(min=1e-300)))
        e = e + (torch.exp2(e + 1) <= top).double() - (torch.exp2(e) > top).double()
        e = torch.where(top > 1.75 * torch.exp2(e), e - 1, e - 2).clamp(-125, 125)
        y = b.abs() / torch.exp2(e)
        level = torch.zeros_like(y)
        for n, t in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
            past = (y >= t) if n % 2 else (y > t)
            level = torch.where(past, torch.full_like(level, LEVELS[n + 1]), level)
        out[..., lo:lo + BLOCK] = torch.copysign(level * torch.exp2(e), b)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    h = case["h"]
    if case["op"] == "store":
        out = []
        for x in "kv":
            d = torch.full(s["dst_" + x].shape, 0.75, dtype=torch.float64, device=DEV)
            for a, b, n in s["first"].tolist():
                for layer in range(case["layers"]):
                    d[layer, b:b + n] = _round64(s["src_" + x][layer, a:a + n])
            out.append(d)
        return tuple(out)
    if case["op"] == "copy":
        out = []
        for x in "kv":
            if case["bits"] == 4:
                src = _levels64(s["src_" + x], s["src_" + x + "_scale"], h)
                d = torch.zeros(s["dst_" + x].shape, dtype=torch.float64, device=DEV)
            else:
                src = s["src_" + x].double()
                d = torch.full(s["dst_" + x].shape, 0.75, dtype=torch.float64, device=DEV)
            for a, b, n in s["first"].tolist():
                d[:, b:b + n] = src[:, a:a + n]
            was = d.clone()
            for a, b, n in s["second"].tolist():
                d[:, b:b + n] = was[:, a:a + n]
            out.append(d)
        return tuple(out)
    p, G = s["plan"], case["q"] // case["kv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for b in range(case["sequences"]):
        o, n, pl, po = int(p["off"][b]), int(p["own"][b]), int(p["plen"][b]), int(p["poff"][b])
        at = torch.cat([torch.arange(po, po + pl), torch.arange(o, o + n)]).to(DEV)
        lo, hi = int(s["cu"][b]), int(s["cu"][b + 1])
        cut = torch.arange(pl + n, device=DEV)[None] > torch.arange(pl + n - (hi - lo), pl + n, device=DEV)[:, None]
        for g in range(case["kv"]):
            K = _levels64(s["k"][at, g], s["k_scale"][at, g], h)
            V = _levels64(s["v"][at, g], s["v_scale"][at, g], h)
            for j in range(g * G, (g + 1) * G):
                w = s["q"][lo:hi, j * h:(j + 1) * h].double() @ K.T / math.sqrt(h)
                out[lo:hi, j * h:(j + 1) * h] = torch.softmax(w.masked_fill(cut, -math.inf), dim=-1) @ V
    return out
