"""The operators of the paged cache - append, attend, copy, compact - as cases that can be timed and compared.

A composed cache that goes on living is kept in pages: ``k`` and ``v`` are ``[layer][page][kv head][row][d]`` ("heads") or
``[layer][page][row][kv head][d]`` ("tokens"), a request is a list of pages and a length.  ``op`` says what a pass does:

* ``append``   the projections of new tokens: queries and keys are normed for each head (where a model does that), rotated to
  their positions, and the keys and values written to their rows of the pages
* ``attend``   attention of one new token of every request over the rows ``[first, length)`` of its pages
* ``copy``     the first rows of pages are copied to other pages, in all layers: what a fork or a move takes
* ``compact``  rows that a compressor keeps - its own for each layer and head - go to the front of new pages

Pages lie in the store in no order, as after hours of serving.  Sizes are those of the repository's own workloads
(``inputs.py``) and the ranges around them.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DEFAULTS = dict(op="attend", layers=1, hq=32, hkv=8, d=128, dtype="bf16", order="heads", page=16, batch=1, lo=512, hi=512, layout=1,
                 norm=False, pairing=0, rotary=0, theta=500000.0, scale=1.0, original=0, low=1.0, high=4.0, magnitude=1.0,
                 first=False, empty=0, lse=False, outliers=0, pairs=1, whole=True, keep=0.41, per_head=True)


def _case(**kw):
    c = dict(_DEFAULTS, **kw)
    c["rotary"] = c["rotary"] or c["d"]
    return c


def listed():
    return [
        # the smallest append there is: one token of one request, 4/2 heads of 64, fp32; launches and host time
        _case(name="append_tiny_f32", op="append", hq=4, hkv=2, d=64, dtype="f32", pairing=1, theta=10000.0, lo=433, hi=433),
        # one decode step of sixteen requests of a model that norms q and k, positions beyond its original context; latency
        _case(name="append_step_b16", op="append", batch=16, hq=28, hkv=4, theta=1000000.0, norm=True, scale=8.0, original=8192, page=64,
              lo=2000, hi=133120),
        # a whole prompt of sixteen documents goes into the pages, part of each head rotated: reading and writing is all there is
        _case(name="append_prompt_33280", op="append", layers=1, page=64, order="tokens", norm=True, rotary=64, scale=4.0, original=32768,
              high=32.0, magnitude=0.1 * math.log(4.0) + 1.0, lo=0, hi=33280),
        # a step of the smallest model: 433 rows, fp32
        _case(name="attend_tiny_f32", hq=4, hkv=2, d=64, dtype="f32", lo=433, hi=433, lse=True),
        # one answer after one ordinary question over five passages; latency
        _case(name="attend_question_2785", lo=2785, hi=2785),
        # requests of uneven lengths, some behind a window, one slot of the batch unused, group of 7 heads, outlier channels
        _case(name="attend_uneven_b8", hq=28, hkv=4, batch=8, order="tokens", lo=300, hi=21120, first=True, empty=1, outliers=2),
        # one request over a very long context: the cache is split over all of the GPU
        _case(name="attend_long_133120", page=64, lo=133120, hi=133120, lse=True),
        # sixteen long requests: the largest pass, bound by reading the cache
        _case(name="attend_b16_33280", page=64, batch=16, lo=33280, hi=33280),
        # sixteen answers fork off one question: the rows of its last, half-full page are copied for each, in every layer
        _case(name="copy_fork_16", op="copy", layers=32, pairs=16, whole=False),
        # a request's 33,280 rows move within the store
        _case(name="copy_move_520", op="copy", layers=8, page=64, pairs=520),
        # one request's prompt is thinned out to two fifths, every head its own rows
        _case(name="compact_question", op="compact", layers=8, lo=2785, hi=2785),
        # four long requests at once
        _case(name="compact_b4_10560", op="compact", layers=8, batch=4, page=64, order="tokens", lo=8000, hi=10560),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        h = rng.choice([(32, 8), (32, 8), (28, 4), (8, 2), (14, 2), (6, 6), (16, 1), (20, 1)])
        d = rng.choice([64, 128, 128])
        c = dict(op=rng.choice(["append", "append", "attend", "attend", "attend", "copy", "compact"]), hq=h[0], hkv=h[1], d=d,
                 dtype=rng.choice(["f32", "bf16", "bf16", "bf16"]), order=rng.choice(["heads", "tokens"]), layout=rng.randrange(1 << 30),
                 page=rng.choice([16, 16, 32, 64, 128, rng.randint(1, 200)]))
        if c["op"] == "append":
            a, b = sorted((_log(rng, 1, 133120), _log(rng, 1, 133120)))
            c.update(batch=_log(rng, 1, 256), lo=a, hi=b, norm=rng.random() < 0.5, pairing=rng.choice([0, 0, 1]),
                     rotary=rng.choice([d, d, d // 2, 16, 48]), theta=rng.choice([10000.0, 500000.0, 1000000.0]),
                     scale=rng.choice([1.0, 1.0, 2.0, 8.0]), original=rng.choice([0, 8192]), high=rng.choice([4.0, 32.0]))
            if rng.random() < 0.4:                         # a chunk of prompt instead of a step
                c.update(batch=1, lo=0, hi=_log(rng, 2, 33280))
        elif c["op"] == "attend":
            a, b = sorted((_log(rng, 1, 133120), _log(rng, 1, 133120)))
            c.update(batch=_log(rng, 1, 256), lo=a, hi=b, first=rng.random() < 0.3, empty=rng.choice([0, 0, 1, 2]),
                     outliers=rng.choice([0, 0, 2]))
            c["lse"] = c["empty"] == 0 and not c["first"] and rng.random() < 0.5
        elif c["op"] == "copy":
            c.update(layers=_log(rng, 1, 32), pairs=_log(rng, 1, 1000), whole=rng.random() < 0.5)
        else:
            a, b = sorted((_log(rng, 16, 33280), _log(rng, 16, 33280)))
            c.update(layers=_log(rng, 1, 32), batch=_log(rng, 1, 16), lo=a, hi=b, keep=round(rng.uniform(0.05, 0.9), 2),
                     per_head=rng.random() < 0.7)
        c = _case(**c)
        if work(c)["bytes"] <= most:
            return c


def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _lens(case):
    """Length of every request: they depend on the case alone."""
    rng = random.Random(case["layout"])
    n = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    n[0] = case["hi"]
    if case["op"] == "attend":
        for b in range(min(case["empty"], case["batch"] - 1)):
            n[-1 - b] = 0
    return n


def _firsts(case):
    rng = random.Random(case["layout"] + 1)
    return [rng.randint(0, n // 2) if case["first"] and rng.random() < 0.5 else 0 for n in _lens(case)]


def _rows(case):
    """Rows that every page of a copy hands on."""
    rng = random.Random(case["layout"] + 2)
    return [case["page"] if case["whole"] else rng.randint(1, case["page"]) for _ in range(case["pairs"])]


def _kept(case):
    return [max(1, int(n * case["keep"])) for n in _lens(case)]


def _new_tokens(case):
    """Tokens of an append: a step brings one token per request, a prompt all of them."""
    return case["hi"] if case["lo"] == 0 else case["batch"]


def work(case):
    e, d, hq, hkv = _elem(case), case["d"], case["hq"], case["hkv"]
    if case["op"] == "append":
        t = _new_tokens(case)
        return {"bytes": t * ((hq + 2 * hkv) * d * e * 2 + 8), "flops": t * (hq + hkv) * (3 * case["rotary"] + (4 * d if case["norm"] else 0))}
    if case["op"] == "attend":
        rows = sum(n - f for n, f in zip(_lens(case), _firsts(case)))
        return {"bytes": 2 * rows * hkv * d * e + 2 * case["batch"] * hq * d * e, "flops": 4 * rows * hq * d}
    if case["op"] == "copy":
        return {"bytes": 4 * sum(_rows(case)) * case["layers"] * hkv * d * e, "flops": 0}
    n = sum(_kept(case))
    return {"bytes": n * case["layers"] * hkv * (4 * d * e + 4) if case["per_head"] else n * (case["layers"] * hkv * 4 * d * e + 4), "flops": 0}


def _store(case, gen, n_pages):
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    inner = (case["hkv"], case["page"]) if case["order"] == "heads" else (case["page"], case["hkv"])
    shape = (case["layers"], n_pages, *inner, case["d"])
    k = torch.empty(shape, dtype=dt, device="cuda")
    v = torch.empty(shape, dtype=dt, device="cuda")
    for t in (k, v):
        for layer in t:
            layer.copy_(torch.randn(layer.shape, generator=gen, device="cuda", dtype=torch.float32))
        if case["outliers"]:
            at = torch.randint(0, case["d"], (case["outliers"],), generator=gen, device="cuda")
            t[..., at] *= 8
    return k, v


def _tables(case, seed, lens, n_pages, perm_from=0):
    """Page table [batch][longest] on the GPU, -1 behind a request's last page, pages drawn from the store in no order."""
    need = [-(-n // case["page"]) for n in lens]
    perm = torch.randperm(n_pages - perm_from, generator=torch.Generator().manual_seed(seed)) + perm_from
    table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n].int()
        at += n
    return table


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    lens = _lens(case)
    s = {"case": case}
    if case["op"] == "append":
        prompt = case["lo"] == 0
        t = _new_tokens(case)
        pos = list(range(t)) if prompt else [n - 1 for n in lens]
        # a step writes into the last page of each request; the pages in front of it stay as they are and are not made
        n_pages = (-(-t // page) if prompt else t) + 3
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
        slots = torch.tensor([int(order[i // page if prompt else i]) * page + p % page for i, p in enumerate(pos)], dtype=torch.int32)
        s["k"], s["v"] = _store(case, gen, n_pages)
        qkv = torch.randn((t, (hq + 2 * hkv) * d), generator=gen, device="cuda").to(dt)
        s["q_new"], s["k_new"], s["v_new"] = (x.unflatten(-1, (-1, d)) for x in qkv.split((hq * d, hkv * d, hkv * d), dim=-1))
        s["positions"], s["slots"] = torch.tensor(pos, dtype=torch.int32, device="cuda"), slots.cuda()
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"], s["k_weight"] = (1 + 0.2 * torch.randn((2, d), generator=gen, device="cuda")).to(dt)
        s["q_out"] = torch.empty((t, hq, d), dtype=dt, device="cuda")
    elif case["op"] == "attend":
        n_pages = sum(-(-n // page) for n in lens) + 3
        s["k"], s["v"] = _store(case, gen, n_pages)
        s["table"], s["lens"] = _tables(case, seed, lens, n_pages).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["first"] = torch.tensor(_firsts(case), dtype=torch.int32, device="cuda") if case["first"] else None
        s["q"] = torch.randn((case["batch"], hq, d), generator=gen, device="cuda").to(dt)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((case["batch"], hq), device="cuda") if case["lse"] else None
        s["longest"] = max(lens)
    elif case["op"] == "copy":
        s["k"], s["v"] = _store(case, gen, 2 * case["pairs"] + 3)
        order = torch.randperm(2 * case["pairs"] + 3, generator=torch.Generator().manual_seed(seed)).tolist()
        # a fork hands one page's rows to all; a move takes every page once
        s["dst"] = order[:case["pairs"]]
        s["src"] = order[case["pairs"]:2 * case["pairs"]] if case["whole"] else [order[case["pairs"]]] * case["pairs"]
        s["rows"] = None if case["whole"] else _rows(case)
    else:
        kept = _kept(case)
        need = sum(-(-n // page) for n in lens)
        n_pages = need + sum(-(-n // page) for n in kept) + 3
        s["k"], s["v"] = _store(case, gen, n_pages)
        s["table"], s["lens"] = _tables(case, seed, lens, need).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
        # the last page is no request's
        s["new_table"] = _tables(case, seed, kept, n_pages - 1, perm_from=need).cuda()
        lk, hk = (case["layers"], hkv) if case["per_head"] else (1, 1)
        lists = torch.zeros((case["batch"], lk, hk, max(kept)), dtype=torch.int32, device="cuda")
        for b, (n, m) in enumerate(zip(lens, kept)):
            # the rows with the m largest scores, in their order, as a compressor leaves them
            lists[b, :, :, :m] = torch.rand((lk, hk, n), generator=gen, device="cuda").topk(m, dim=-1).indices.sort(dim=-1).values.int()
        s["kept"], s["n_kept"] = lists, torch.tensor(kept, dtype=torch.int32, device="cuda")
    if own:
        from paper_2604_13226_b200 import binding as kvp
        s["cache"] = kvp.PagedCache(s["k"], s["v"], n_q_heads=hq, order=case["order"], max_batch=case["batch"])
        if case["op"] == "append":
            s["rope"] = kvp.Rope(d, rotary_dim=case["rotary"], theta=case["theta"], pairing=case["pairing"], scale=case["scale"],
                                 original_positions=case["original"], low_rotations=case["low"], high_rotations=case["high"],
                                 magnitude=case["magnitude"])
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        cache = s["cache"]
        if op == "append":
            cache.append(0, s["k_new"], s["v_new"], s["positions"], s["slots"], rope=s["rope"], q=s["q_new"], q_out=s["q_out"],
                         q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6)
            return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
        if op == "attend":
            cache.attend(0, s["q"], s["table"], s["lens"], s["out"], lse=s["lse"], first=s["first"])
            return {"out": s["out"], "lse": s["lse"]}
        if op == "copy":
            cache.copy(s["src"], s["dst"], rows=s["rows"])
        else:
            cache.compact(s["table"], s["lens"], s["new_table"], s["kept"], s["n_kept"])
        return {"k": s["k"], "v": s["v"]}
    return {"append": _append, "attend": _attend, "copy": _copy, "compact": _compact}[op](s)


# ---- the plain forms --------------------------------------------------------------------------------------------

def _by_head(case, pages):
    """[..., page][kv head][row][d] whatever the order."""
    return pages if case["order"] == "heads" else pages.transpose(-2, -3)


def _frequencies(case):
    r = case["rotary"]
    f = case["theta"] ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    turns = f * case["original"] / (2 * math.pi)
    smooth = ((turns - case["low"]) / (case["high"] - case["low"])).clamp(0, 1) if case["original"] else torch.zeros_like(f)
    return f * (smooth + (1 - smooth) / case["scale"])


def _norm_rotate(case, x, weight, positions):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
    angle = positions.double()[:, None] * _frequencies(case)
    cos, sin = (case["magnitude"] * t.float()[:, None] for t in (angle.cos(), angle.sin()))
    r = case["rotary"]
    turned, rest = x[..., :r], x[..., r:]
    if case["pairing"] == 0:
        a, b = turned.chunk(2, dim=-1)
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    return torch.cat((turned, rest), dim=-1)


def _append(s):
    case, dt = s["case"], s["k"].dtype
    k, v = _by_head(case, s["k"][0]), _by_head(case, s["v"][0])
    slots = s["slots"].long()
    page, row = slots // case["page"], slots % case["page"]
    k[page, :, row] = _norm_rotate(case, s["k_new"], s["k_weight"], s["positions"]).to(dt)
    v[page, :, row] = s["v_new"]
    return {"q": _norm_rotate(case, s["q_new"], s["q_weight"], s["positions"]).to(dt), "k": s["k"], "v": s["v"]}


def _attend(s):
    case = s["case"]
    g = case["hq"] // case["hkv"]
    rows = torch.arange(s["longest"], device="cuda")
    page = s["table"].long()[:, rows // case["page"]].clamp(min=0)
    there = rows < s["lens"][:, None]
    if s["first"] is not None:
        there = there & (rows >= s["first"][:, None])
    row = (rows % case["page"]).expand_as(page)
    k = _by_head(case, s["k"][0])[page, :, row].float()                            # [batch][row][kv head][d]
    q = s["q"].float().unflatten(1, (case["hkv"], g))
    score = torch.einsum("bhgd,bnhd->bhgn", q, k) / math.sqrt(case["d"])
    del k
    there = there[:, None, None]
    score = score.masked_fill(~there, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (score - top).exp().masked_fill(~there, 0.0)
    total = p.sum(-1, keepdim=True)
    v = _by_head(case, s["v"][0])[page, :, row].float()
    out = torch.einsum("bhgn,bnhd->bhgd", p, v) / total.clamp(min=1e-30)
    return {"out": out.flatten(1, 2).to(s["q"].dtype), "lse": (top + total.log()).flatten(1) if s["lse"] is not None else None}


def _copy(s):
    case = s["case"]
    src, dst = torch.tensor(s["src"], device="cuda"), torch.tensor(s["dst"], device="cuda")
    k, v = _by_head(case, s["k"]), _by_head(case, s["v"])
    if s["rows"] is None:
        k[:, dst] = k[:, src]
        v[:, dst] = v[:, src]
    else:
        goes = (torch.arange(case["page"], device="cuda") < torch.tensor(s["rows"], device="cuda")[:, None])[:, None, :, None]
        k[:, dst] = torch.where(goes, k[:, src], k[:, dst])
        v[:, dst] = torch.where(goes, v[:, src], v[:, dst])
    return {"k": s["k"], "v": s["v"]}


def _compact(s):
    case, page = s["case"], s["case"]["page"]
    kept = s["kept"].long().expand(-1, case["layers"], case["hkv"], -1)               # [batch][layer][kv head][i]
    b = torch.arange(case["batch"], device="cuda")[:, None, None, None]
    layer = torch.arange(case["layers"], device="cuda")[None, :, None, None]
    head = torch.arange(case["hkv"], device="cuda")[None, None, :, None]
    i = torch.arange(kept.shape[-1], device="cuda")
    goes = (i < s["n_kept"][:, None])[:, None, None]
    at = (layer, s["table"].long()[b, kept // page].clamp(min=0), head, kept % page)
    # entries behind a request's last kept row write nothing: they go to a row of the spare page at the end of the store
    to = s["new_table"].long()[b, (i // page)[None, None, None].clamp(max=s["new_table"].shape[1] - 1)].expand_as(kept)
    spare = s["k"].shape[1] - 1
    to = (layer, torch.where(goes & (to >= 0), to, spare), head, (i % page).expand_as(kept))
    k, v = _by_head(case, s["k"]), _by_head(case, s["v"])
    k[to] = torch.where(goes[..., None], k[at], k[to])
    v[to] = torch.where(goes[..., None], v[at], v[to])
    return {"k": s["k"], "v": s["v"]}


# ---- the definitions, in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("copy", "compact"):
        return None                                       # rows move, nothing is computed
    g, page, heads = case["hq"] // case["hkv"], case["page"], case["order"] == "heads"
    if case["op"] == "attend":
        out = torch.zeros((case["batch"], case["hq"], case["d"]), dtype=torch.float64, device="cuda")
        lse = torch.full((case["batch"], case["hq"]), -math.inf, dtype=torch.float64, device="cuda")
        for b, (f, n) in enumerate(zip(_firsts(case), _lens(case))):
            if n <= f:
                continue
            pages = s["table"][b, :-(-n // page)].long()
            for h in range(case["hkv"]):
                k, v = ((t[0, pages, h] if heads else t[0, pages, :, h]).reshape(-1, case["d"])[f:n].double() for t in (s["k"], s["v"]))
                score = s["q"][b, h * g:(h + 1) * g].double() @ k.T * case["d"] ** -0.5
                lse[b, h * g:(h + 1) * g] = score.logsumexp(-1)
                out[b, h * g:(h + 1) * g] = score.softmax(-1) @ v
        return {"out": out, "lse": lse if case["lse"] else None}
    r = case["rotary"]
    new = {}
    for name, w in (("q_new", s["q_weight"]), ("k_new", s["k_weight"])):
        x = s[name].double()
        if w is not None:
            x = x / (x.pow(2).sum(-1, keepdim=True) / case["d"] + 1e-6).sqrt() * w.double()
        y = x.clone()
        for i in range(r // 2):
            f = math.exp(-2.0 * i / r * math.log(case["theta"]))
            if case["original"] == 0:
                f = f / case["scale"]
            else:
                part = (case["original"] * f / (2 * math.pi) - case["low"]) / (case["high"] - case["low"])
                part = min(1.0, max(0.0, part))
                f = (1 - part) * f / case["scale"] + part * f
            a, b = (i, i + r // 2) if case["pairing"] == 0 else (2 * i, 2 * i + 1)
            turn = torch.polar(torch.full(s["positions"].shape, case["magnitude"], dtype=torch.float64, device="cuda"), s["positions"].double() * f)
            z = torch.complex(x[..., a], x[..., b]) * turn[:, None]
            y[..., a], y[..., b] = z.real, z.imag
        new[name] = y
    k, v = s["k"].double(), s["v"].double()
    p, row = s["slots"].long() // page, s["slots"].long() % page
    if heads:
        k[0, p, :, row], v[0, p, :, row] = new["k_new"], s["v_new"].double()
    else:
        k[0, p, row], v[0, p, row] = new["k_new"], s["v_new"].double()
    return {"q": new["q_new"], "k": k, "v": v}
