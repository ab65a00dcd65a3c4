"""The 8-bit K/V cache and the attention that reads it, one call at a time.

A case is one call of an operator, as a serving program makes it for one layer:

  append  a pass's new keys and values are rounded to 8 bits and written into the rows' pages
  attend  the pass's queries attend causally over everything their rows hold
  select  each query attends to the pages that a score on the pages' key bounds selects for it

Head counts and widths are those of the workloads (16 heads of 64, 32 heads of 128) and of
grouped heads; rows are ragged, their pages lie in arbitrary order in the pool.

Layout of one layer's cache: pages of 64 positions; keys [page][head][64][dim] and values
[page][head][16][dim][4] (position t of a page at [t / 4][:][t % 4]) as e4m3, one power-of-two
scale for each page and head of K and of V, and two int8 bounds per page, head and channel:
the largest ceil(key / 4) and the smallest floor(key / 4) in units of the scale.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn


def _case(name, kind, rows, heads, group, dim, lo, hi, new_lo, new_hi, dtype, fused=False, n_select=0):
    return dict(name=name, kind=kind, rows=rows, heads=heads, group=group, dim=dim, lo=lo, hi=hi, new_lo=new_lo,
                new_hi=new_hi, dtype=dtype, fused=fused, n_select=n_select)


def listed():
    return [
        # one robot of the 12-layer policy: the K/V of one fed-back action token
        _case("append-1tok", "append", 1, 16, 1, 64, 290, 290, 1, 1, "f32", fused=True),
        # the same for a batch of 64 robots at the 7B width, ragged
        _case("append-b64", "append", 64, 32, 1, 128, 200, 768, 1, 1, "f16", fused=True),
        # the prefixes of those 64 rows when their contexts are built
        _case("append-build", "append", 64, 32, 1, 128, 200, 400, 200, 400, "bf16", fused=True),
        # one robot, a short context: the latency of one decode step's attention
        _case("attend-b1", "attend", 1, 16, 1, 64, 97, 97, 1, 1, "f16"),
        # 64 robots at the 7B width: the decode step's attention
        _case("attend-b64", "attend", 64, 32, 1, 128, 200, 768, 1, 1, "bf16"),
        # 16 robots that decode action chunks after a 600-token prefix, in full precision
        _case("attend-b16-f32", "attend", 16, 32, 1, 128, 600, 656, 1, 1, "f32", fused=True),
        # four long histories with grouped heads: one decode step over some 100,000 positions each
        _case("attend-long", "attend", 4, 8, 4, 128, 70001, 131072, 1, 1, "bf16"),
        # new observation tokens of 64 robots over their contexts
        _case("attend-extend", "attend", 64, 32, 1, 128, 216, 700, 9, 16, "f16", fused=True),
        # eight long prefixes built from nothing, grouped heads
        _case("attend-build", "attend", 8, 8, 4, 128, 1500, 2048, 1500, 2048, "bf16"),
        # one robot with a long history: a decode step over 8 of its 63 pages
        _case("select-b1", "select", 1, 16, 1, 64, 4001, 4001, 1, 1, "f16", n_select=8),
        # eight long histories, grouped heads: a decode step over 64 of up to 1,024 pages
        _case("select-long", "select", 8, 8, 4, 128, 30000, 65536, 1, 1, "bf16", n_select=64),
        # new observation tokens over long histories, each with pages of its own
        _case("select-extend", "select", 4, 8, 4, 128, 8000, 16384, 33, 64, "f16", fused=True, n_select=32),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _draw(rng):
    kind = rng.choice(["append", "attend", "attend", "select"])
    heads, group = rng.choice([(16, 1), (32, 1), (8, 4), (8, 1), (4, 7), (2, 8), (5, 3), (1, 16)])
    dim = rng.choice([64, 128])
    dtype = rng.choice(["f32", "f16", "bf16", "f16", "bf16"])
    fused = rng.random() < 0.5
    rows = _log(rng, 1, 64)
    if kind == "append":
        hi = _log(rng, 1, 2048)
        lo = rng.randint(max(1, hi // 2), hi)
        new_hi = rng.choice([1, hi, _log(rng, 1, lo)])
        return _case("", kind, rows, heads, group, dim, lo, hi, min(new_hi, rng.randint(1, lo)), min(new_hi, lo), dtype,
                     fused)
    if kind == "attend":
        form = rng.choice(["decode", "decode", "extend", "build"])
        hi = _log(rng, 1, 131072 if form == "decode" else 4096 if form == "extend" else 2048)
        lo = rng.randint(max(1, hi // 2), hi)
        new_hi = 1 if form == "decode" else min(lo, _log(rng, 2, 64)) if form == "extend" else lo
        new_lo = new_hi if form == "build" else rng.randint(max(1, new_hi // 2), new_hi)
        return _case("", kind, rows, heads, group, dim, lo, hi, new_lo, new_hi, dtype, fused)
    hi = _log(rng, 200, 65536)
    lo = rng.randint(hi // 2, hi)
    new_hi = rng.choice([1, 1, _log(rng, 2, 64)])
    return _case("", kind, rows, heads, group, dim, lo, hi, rng.randint(max(1, new_hi // 2), new_hi), new_hi, dtype,
                 fused, n_select=rng.choice([4, 8, 13, 16, 32, 64]))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    wide = max(c["rows"] * c["heads"] * c["hi"] * c["dim"] for c in listed())  # the padded cache of the plain form
    while True:
        c = _draw(rng)
        w = work(c)
        padded = c["rows"] * c["heads"] * c["hi"] * c["dim"]
        scores = c["rows"] * c["heads"] * c["group"] * c["new_hi"] * c["hi"]
        picked = c["rows"] * c["heads"] * c["new_hi"] * c["n_select"] * PAGE * c["dim"]
        if all(w[k] <= most[k] for k in most) and max(padded, 2 * scores, picked) <= wide:
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi in no order."""
    return [lo + (hi - lo) * ((i * 7919) % n) // max(n - 1, 1) for i in range(n)]


def _shape(case):
    """Positions that each row holds after the call, and how many of them are new."""
    lens = _spread(case["lo"], case["hi"], case["rows"])
    new = [min(n, m) for n, m in zip(_spread(case["new_lo"], case["new_hi"], case["rows"]), lens)]
    return lens, new


def _inputs(case, g, n_tok, heads, kv_heads):
    """Queries, keys and values of a pass: slices of one projection's output, or tensors of their own."""
    dim, dt = case["dim"], DTYPES[case["dtype"]]
    width = [heads * dim, kv_heads * dim, kv_heads * dim]
    if case["fused"]:
        x = torch.randn(n_tok, sum(width), device="cuda", generator=g).to(dt)
        parts = torch.split(x, width, dim=1)
    else:
        parts = [torch.randn(n_tok, w, device="cuda", generator=g).to(dt) for w in width]
    return [p.unflatten(1, (-1, dim)) for p in parts]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    lens, new = _shape(case)
    rows, kv, dim = case["rows"], case["heads"], case["dim"]
    need = [-(-n // PAGE) for n in lens]
    width, pages = max(need), sum(need) + 3
    # pages that hold keys with a drift of their own, every slot written, and values
    k = torch.randn(pages, kv, PAGE, dim, device="cuda", generator=g).mul_(40)
    k.add_(torch.randn(pages, kv, 1, dim, device="cuda", generator=g).mul_(25)).clamp_(-448, 448)
    k = k.to(E4M3)
    v = torch.randn(pages, kv, PAGE // 4, dim, 4, device="cuda", generator=g).mul_(60).clamp_(-448, 448).to(E4M3)
    hi, lo = k.to(torch.float16).amax(2), k.to(torch.float16).amin(2)
    bounds = torch.stack([torch.ceil(hi / 4), torch.floor(lo / 4)], 2).to(torch.int8)
    scale = [torch.exp2(torch.randint(-7, -4, (pages, kv), device="cuda", generator=g).float()) for _ in range(2)]
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    off = torch.tensor([0] + np.cumsum(new).tolist(), dtype=torch.int32, device="cuda")
    q, k_new, v_new = _inputs(case, g, sum(new), kv * case["group"], kv)
    return dict(kind=case["kind"], k=k, v=v, k_scale=scale[0], v_scale=scale[1], bounds=bounds, table=table, off=off,
                lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), max_new=max(new), max_len=max(lens), q=q,
                k_new=k_new, v_new=v_new, n_select=case["n_select"], softmax_scale=1 / math.sqrt(dim))


def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "append":
        _append(s)
        return dict(k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"], bounds=s["bounds"])
    return _attend(s) if s["kind"] == "attend" else _select(s)


def _run_own(s):
    if "cache" not in s:  # the handle that a program keeps
        from paper_2508_10259_amd.qcache import QuantCache
        s["cache"] = QuantCache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["bounds"], s["table"])
    c = s["cache"]
    if s["kind"] == "append":
        c.append(s["k_new"], s["v_new"], s["off"], s["lens"], max_new=s["max_new"])
        return dict(k=c.k, v=c.v, k_scale=c.k_scale, v_scale=c.v_scale, bounds=c.k_bounds)
    if s["kind"] == "attend":
        return c.attend(s["q"], s["off"], s["lens"], max_new=s["max_new"], max_len=s["max_len"],
                        scale=s["softmax_scale"])
    out, selected = c.attend_selected(s["q"], s["off"], s["lens"], s["n_select"], max_new=s["max_new"],
                                      max_len=s["max_len"], scale=s["softmax_scale"])
    return dict(out=out, selected=selected)


# --- the plain forms --------------------------------------------------------------------------


def _tokens(s):
    """Each new token's row, its place among the row's new tokens and its position."""
    n = s["q"].shape[0]
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    row = torch.searchsorted(s["off"][1:].contiguous(), t, right=True)
    i = t - s["off"][row]
    pos = s["lens"][row] - (s["off"][row + 1] - s["off"][row]) + i
    return row, i.long(), pos.long()


def _exponent(a):
    """The least e with a <= 448 2^e, at least -32."""
    m, x = torch.frexp(a)
    e = x - 9 + (m > 0.875)
    return torch.where(a > 0, e, -32).clamp(-32, 8)


def _append(s):
    row, i, pos = _tokens(s)
    page, slot = s["table"][row, pos // PAGE].long(), pos % PAGE
    # the first slot that each page gets, and each row's first page, which may hold older slots
    first = torch.full(s["k_scale"].shape[:1], PAGE, device="cuda").index_reduce_(0, page, slot, "amin")
    head_page = page[s["off"][:-1].long()]
    older = torch.arange(PAGE, device="cuda") < first[head_page][:, None]
    code, ratio = _scaled(s, "k", page, first, head_page, older[:, None, :, None])
    s["k"].view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
    value = code.float() / 4
    hi, lo = s["bounds"][:, :, 0].float(), s["bounds"][:, :, 1].float()
    up = torch.full_like(hi, -128).index_reduce_(0, page, torch.ceil(value), "amax")
    down = torch.full_like(lo, 127).index_reduce_(0, page, torch.floor(value), "amin")
    hi, lo = torch.ceil(hi * ratio[:, :, None]), torch.floor(lo * ratio[:, :, None])
    kept = (first > 0)[:, None, None]
    hi, lo = torch.where(kept, torch.maximum(hi, up), up), torch.where(kept, torch.minimum(lo, down), down)
    s["bounds"].copy_(torch.stack([hi, lo], 2).to(torch.int8))
    code, _ = _scaled(s, "v", page, first, head_page, older.view(-1, 1, PAGE // 4, 1, 4))
    s["v"].view(torch.uint8)[page, :, slot // 4, :, slot % 4] = code.view(torch.uint8)


def _scaled(s, name, page, first, head_page, older):
    """Brings the pages' scales up to date, and their older slots to them; the new tokens' codes, and old / new scales."""
    x, pool, scale = s[name + "_new"].float().clamp(-65504, 65504), s[name], s[name + "_scale"]
    need = _exponent(torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(2), "amax"))
    was = torch.frexp(scale)[1] - 1
    e = torch.where(first[:, None] > 0, torch.maximum(need, was), need)
    now = torch.exp2(torch.where(first[:, None] < PAGE, e, was).float())
    ratio = scale / now
    held = pool[head_page]
    grown = (held.float() * ratio[head_page].view(*held.shape[:2], *[1] * (held.dim() - 2))).to(E4M3)
    pool.view(torch.uint8)[head_page] = torch.where(older, grown.view(torch.uint8), held.view(torch.uint8))
    scale.copy_(now)
    return (x / now[page][:, :, None]).to(E4M3), ratio


def _padded_queries(s):
    """[row][KV head][new token][group][dim], and which of the new tokens there are."""
    n = s["off"][1:] - s["off"][:-1]
    i = torch.arange(s["max_new"], device="cuda")
    t = (s["off"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1).long()
    kv = s["k_scale"].shape[1]
    q = s["q"][t].float().unflatten(2, (kv, -1)).transpose(1, 2)
    visible = s["lens"][:, None] - n[:, None] + 1 + i  # positions that a token sees
    return q, visible


def _softmax_product(q, k, v, mask, scale):
    """softmax(scale q k^T) v over the positions of the mask; q [..., m, d], k and v [..., n, d]."""
    x = (torch.matmul(q, k.transpose(-1, -2)) * scale).masked_fill_(~mask, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    return torch.matmul(x, v) / x.sum(-1, keepdim=True)


def _attend(s):
    q, visible = _padded_queries(s)
    rows, kv, n, group, dim = q.shape
    pages = s["table"].clamp(min=0).long()
    k = (s["k"][pages].float() * s["k_scale"][pages][..., None, None]).transpose(1, 2).reshape(rows, kv, -1, dim)
    v = (s["v"][pages].float() * s["v_scale"][pages][..., None, None, None]).transpose(-1, -2)
    v = v.transpose(1, 2).reshape(rows, kv, -1, dim)
    mask = torch.arange(k.shape[2], device="cuda") < visible[..., None]
    o = _softmax_product(q.reshape(rows, kv, n * group, dim), k, v,
                         mask[:, None, :, None].expand(-1, -1, -1, group, -1).reshape(rows, 1, n * group, -1),
                         s["softmax_scale"])
    row, i, _ = _tokens(s)
    o = o.view(rows, kv, n, group, dim).transpose(1, 2)[row, i]
    return o.reshape(-1, kv * group, dim).to(s["q"].dtype)


def _select(s):
    q, visible = _padded_queries(s)
    rows, kv, n, group, dim = q.shape
    pages = s["table"].clamp(min=0).long()
    width = pages.shape[1]
    # the score: bounds of q . k in whole numbers
    _, x = torch.frexp(q.abs().amax((-1, -2), keepdim=True))
    whole = torch.round(torch.ldexp(q, 7 - x)).clamp(-127, 127)
    parts = torch.cat([whole.clamp(min=0), whole.clamp(max=0)], -1).reshape(rows, kv, n * group, 2 * dim)
    bounds = s["bounds"][pages].float().transpose(1, 2).reshape(rows, kv, width, 2 * dim)
    score = torch.matmul(parts, bounds.transpose(-1, -2)).view(rows, kv, n, group, width).amax(3)
    score = score * s["k_scale"][pages].transpose(1, 2)[:, :, None]
    count = ((visible + PAGE - 1) // PAGE)[:, None, :, None]
    at = torch.arange(width, device="cuda")
    score = score.masked_fill(at == count - 1, math.inf).masked_fill(at >= count, -math.inf)
    score, chosen = torch.sort(score, dim=-1, descending=True, stable=True)
    score, chosen = score[..., :s["n_select"]], chosen[..., :s["n_select"]]
    chosen = torch.where(score > -math.inf, chosen, width).sort(-1).values  # [row][head][token][page]
    there = chosen < width
    # attention over the chosen pages
    physical = pages[torch.arange(rows, device="cuda")[:, None, None, None], chosen.clamp(max=width - 1)]
    head = torch.arange(kv, device="cuda")[:, None, None]
    k = s["k"].view(torch.uint8)[physical, head].view(E4M3).float() * s["k_scale"][physical, head][..., None, None]
    v = s["v"].view(torch.uint8)[physical, head].view(E4M3).float().transpose(-1, -2).flatten(-3, -2)
    v = v * s["v_scale"][physical, head][..., None, None]
    pos = chosen[..., None] * PAGE + torch.arange(PAGE, device="cuda")
    mask = there[..., None] & (pos < visible[:, None, :, None, None])
    o = _softmax_product(q, k.flatten(-3, -2), v.flatten(-3, -2), mask.flatten(-2)[..., None, :], s["softmax_scale"])
    row, i, _ = _tokens(s)
    selected = torch.where(there, chosen, -1).to(torch.int32).transpose(1, 2)[row, i]
    if selected.shape[-1] < s["n_select"]:
        selected = torch.nn.functional.pad(selected, (0, s["n_select"] - selected.shape[-1]), value=-1)
    return dict(out=o.transpose(1, 2)[row, i].reshape(-1, kv * group, dim).to(s["q"].dtype), selected=selected)


# --- work, and the definition in 64 bits ------------------------------------------------------


def work(case):
    lens, new = _shape(case)
    kv, group, dim = case["heads"], case["group"], case["dim"]
    es = {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    tok = sum(new)
    if case["kind"] == "append":
        touched = sum((n - 1) // PAGE - (n - m) // PAGE + 1 for n, m in zip(lens, new))
        return dict(bytes=2 * tok * kv * dim * (es + 1) + touched * kv * (4 * dim + 16), flops=8 * tok * kv * dim)
    io = 2 * tok * kv * group * dim * es
    if case["kind"] == "attend":
        held = sum(lens) * kv * 2 * dim + sum(-(-n // PAGE) for n in lens) * kv * 8
        pairs = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))
        return dict(bytes=held + io, flops=4 * pairs * kv * group * dim)
    seen = [-(-n // PAGE) for n in lens]
    picked = [min(case["n_select"], p) for p in seen]
    read = sum(min(p, m * c) for p, m, c in zip(seen, new, picked))
    return dict(bytes=kv * (sum(seen) * (2 * dim + 4) + read * (PAGE * 2 * dim + 8)) + io + 4 * tok * kv * case["n_select"],
                flops=4 * dim * kv * group * sum(m * (p + c * PAGE) for p, m, c in zip(seen, new, picked)))


def _values(codes):
    """What e4m3 codes stand for, in 64 bits: 4 exponent bits of bias 7, 3 bits of mantissa, no infinities."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, np.ldexp(m / 8.0, -6), np.ldexp(1 + m / 8.0, e - 7))
    v = np.where((c & 127) == 127, np.nan, v) * np.where(c & 128, -1.0, 1.0)
    return torch.from_numpy(v).cuda()[codes.view(torch.uint8).int()]


def _nearest(x):
    """The e4m3 value nearest to x in 64 bits (|x| <= 448), ties to even."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _shape(case)
    off = np.cumsum([0] + new).tolist()
    kv, group, dim = case["heads"], case["group"], case["dim"]
    table = s["table"].tolist()
    if case["kind"] == "append":
        k, v = _values(s["k"]), _values(s["v"]).transpose(-1, -2).reshape(s["k"].shape).contiguous()
        scales, bounds = [s["k_scale"].double(), s["v_scale"].double()], s["bounds"].double()
        for r, (n, m) in enumerate(zip(lens, new)):
            for p in range((n - m) // PAGE, (n - 1) // PAGE + 1):
                page, a, b = table[r][p], max(n - m - p * PAGE, 0), min(n - p * PAGE, PAGE)
                t = off[r] + p * PAGE + a - (n - m)
                for pool, scale, x in ((k, scales[0], s["k_new"]), (v, scales[1], s["v_new"])):
                    x = x[t:t + b - a].double().clamp(-65504, 65504).transpose(0, 1)
                    e = torch.exp2(torch.ceil(torch.log2(x.abs().amax((1, 2)) / 448)).clamp(-32, 8))
                    if a:
                        e = torch.maximum(e, scale[page])
                    ratio = scale[page] / e
                    pool[page, :, :a] = _nearest(pool[page, :, :a] * ratio[:, None, None])
                    pool[page, :, a:b] = _nearest(x / e[:, None, None])
                    scale[page] = e
                    if pool is k:
                        hi, lo = torch.ceil(k[page, :, a:b] / 4).amax(1), torch.floor(k[page, :, a:b] / 4).amin(1)
                        if a:
                            hi = torch.maximum(hi, torch.ceil(bounds[page, :, 0] * ratio[:, None]))
                            lo = torch.minimum(lo, torch.floor(bounds[page, :, 1] * ratio[:, None]))
                        bounds[page] = torch.stack([hi, lo], 1)
        v = v.view(-1, kv, PAGE // 4, 4, dim).transpose(-1, -2)
        return dict(k=k, v=v, k_scale=scales[0], v_scale=scales[1], bounds=bounds.to(torch.int8))
    pairs = sum(m * n for n, m in zip(lens, new))
    if case["kind"] == "select" and off[-1] * kv > 4000 or pairs * kv * group * dim > 4e11:
        return None
    out = torch.zeros(off[-1], kv * group, dim, dtype=torch.float64, device="cuda")
    selected = torch.full((off[-1], kv, case["n_select"]), -1, dtype=torch.int32, device="cuda")
    for r, (n, m) in enumerate(zip(lens, new)):
        pages = torch.tensor(table[r][:-(-n // PAGE)], device="cuda")
        q = s["q"][off[r]:off[r + 1]].double().view(m, kv, group, dim)
        seen = torch.arange(n - m, n, device="cuda") + 1
        for h in range(kv):
            ks, vs = s["k_scale"][pages, h].double(), s["v_scale"][pages, h].double()
            k = (_values(s["k"][pages, h]) * ks[:, None, None]).reshape(-1, dim)
            v = (_values(s["v"][pages, h]).transpose(-1, -2).reshape(-1, PAGE, dim) * vs[:, None, None]).reshape(-1, dim)
            keep = torch.arange(k.shape[0], device="cuda") < seen[:, None]
            if case["kind"] == "select":
                hi, lo = s["bounds"][pages, h, 0].double(), s["bounds"][pages, h, 1].double()
                top = q[:, h].abs().amax((1, 2), keepdim=True)
                w = torch.round(q[:, h] * torch.exp2(6 - torch.floor(torch.log2(top)))).clamp(-127, 127)
                score = torch.where(w > 0, w, 0) @ hi.t() + torch.where(w < 0, w, 0) @ lo.t()
                score = score.amax(1) * ks
                for i in range(m):
                    last = (int(n - m + i) + PAGE) // PAGE - 1
                    best = sorted(range(last), key=lambda p, x=score[i].tolist(): (-x[p], p))[:case["n_select"] - 1]
                    best = sorted(best + [last])
                    selected[off[r] + i, h, :len(best)] = torch.tensor(best, dtype=torch.int32, device="cuda")
                    mine = torch.zeros(len(pages), dtype=torch.bool, device="cuda")
                    mine[best] = True
                    keep[i] &= mine.repeat_interleave(PAGE)
            x = (q[:, h].reshape(m * group, dim) @ k.t()) * s["softmax_scale"]
            x = x.masked_fill(~keep.repeat_interleave(group, 0), -math.inf)
            o = torch.softmax(x, -1) @ v
            out[off[r]:off[r + 1]].view(m, kv, group, dim)[:, h] = o.view(m, group, dim)
    return out if case["kind"] == "attend" else dict(out=out, selected=selected)
