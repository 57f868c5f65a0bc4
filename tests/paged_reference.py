"""Plain 64-bit forms of the paged cache's operators, and how far fp32 arithmetic over bf16 or fp32 data may be from them."""
import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def pages(shape, order, dtype, seed=0, device="cuda", scale=1.0):
    """k, v of (layers, pages, kv heads, page size, d), in the given order."""
    g = torch.Generator(device=device).manual_seed(seed)
    L, P, H, S, D = shape
    s = (L, P, H, S, D) if order == "heads" else (L, P, S, H, D)
    return tuple((scale * torch.randn(s, generator=g, device=device)).to(dtype) for _ in range(2))


def row_of(t, order, layer, page, head, row):
    return t[layer, page, head, row] if order == "heads" else t[layer, page, row, head]


def gather(t, order, layer, table_row, page_size, rows):
    """[rows][kv head][d] in float64 of the given row numbers."""
    pg = table_row[torch.div(rows, page_size, rounding_mode="floor")].long()
    r = rows % page_size
    x = t[layer].double() if t[layer].numel() < 1 << 24 else None
    if x is None:                                                # a store too large to widen: row by row of what is read
        return (t[layer][pg, :, r] if order == "heads" else t[layer][pg, r]).double()
    return x[pg, :, r] if order == "heads" else x[pg, r]


def attend(k, v, order, layer, q, table, lens, first, page_size, scale):
    """out, lse and the tolerances of both, in float64.

    Scores: products of bf16 (or fp32) numbers summed in fp32, d terms: off by (d + 4) 2^-24 sum |q_i k_i| scale at most
    (2^-23 where a tensor core cuts instead of rounding).  A probability is off by the error of two scores and by 2^-21 from
    exp2; a bf16 cache's are carried in two bf16 numbers, 2^-16.  Sums over n keys: n 2^-23 of the sum of magnitudes.  The
    output is rounded once."""
    n_pages = k.shape[1]
    hkv = k.shape[2 if order == "heads" else 3]
    B, hq, d = q.shape
    g = hq // hkv
    out = torch.zeros((B, hq, d), dtype=torch.float64, device=q.device)
    lse = torch.full((B, hq), -math.inf, dtype=torch.float64, device=q.device)
    tol_out, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    tab = table.cpu()
    for b in range(B):
        n = min(max(int(lens[b]), 0), table.shape[1] * page_size)
        rows = torch.arange(min(max(int(first[b]), 0), n) if first is not None else 0, n)
        if len(rows):
            pg = tab[b][torch.div(rows, page_size, rounding_mode="floor")]
            rows = rows[(pg >= 0) & (pg < n_pages)]
        if not len(rows):
            continue
        rows = rows.to(q.device)
        K, V = (gather(t, order, layer, table[b], page_size, rows) for t in (k, v))
        Q = q[b].double().view(hkv, g, d)
        s = torch.einsum("hgd,nhd->hgn", Q, K) * scale
        mag = torch.einsum("hgd,nhd->hgn", Q.abs(), K.abs()).amax(-1, keepdim=True) * scale
        p = s.softmax(-1)
        out[b] = torch.einsum("hgn,nhd->hgd", p, V).reshape(hq, d)
        lse[b] = s.logsumexp(-1).reshape(hq)
        ds = (d + 4) * 2.0 ** -23 * mag + 2.0 ** -22 * s.abs().amax(-1, keepdim=True)
        rel = 2 * ds + 2.0 ** -21 + (2.0 ** -16 if q.dtype == torch.bfloat16 else 0.0) + (len(rows) + 64) * 2.0 ** -23
        whole = torch.einsum("hgn,nhd->hgd", p, V.abs())
        tol_out[b] = (2 * rel * whole).reshape(hq, d) + HALF_STEP[q.dtype] * out[b].abs() * 1.001
        tol_lse[b] = (ds + 2.0 ** -21 + (len(rows) + 64) * 2.0 ** -23).reshape(hq) + 2.0 ** -23 * lse[b].abs() + 2.0 ** -22
    return out, lse, tol_out, tol_lse


def frequencies(r, theta, scale=1.0, original=0.0, low=1.0, high=4.0):
    out = []
    for i in range(r // 2):
        f = theta ** (-2.0 * i / r)
        if original:
            turns = original * f / (2 * math.pi)
            w = min(1.0, max(0.0, (turns - low) / (high - low)))
            out.append(f * w + f / scale * (1 - w))
        else:
            out.append(f / scale)
    return out


def norm_rotate(x, weight, eps, positions, freqs, pairing, magnitude):
    """Result in float64 and its tolerance before the output's rounding: a norm of d squares, a product of three numbers, a
    rotation of two products whose sine and cosine are off by 2^-22 (rounded part of a turn, 2 pi times 2^-25, and the
    function): 2^-20 of the pair's magnitudes covers them with d 2^-24 for the sum of squares."""
    d = x.shape[-1]
    y = x.double()
    if weight is not None:
        y = y / (y.pow(2).mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    r = 2 * len(freqs)
    size = y.abs()
    out, span = y.clone(), size.clone()
    if r:
        f = torch.tensor(freqs, dtype=torch.float64, device=x.device)
        ang = positions.double()[:, None, None] * f
        c, s = ang.cos() * magnitude, ang.sin() * magnitude
        a, b = (slice(0, r // 2), slice(r // 2, r)) if pairing == 0 else (slice(0, r, 2), slice(1, r, 2))
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., a] * s + y[..., b] * c
        span[..., a] = span[..., b] = (size[..., a] + size[..., b]) * magnitude
    return out, span * (2.0 ** -20 + (d * 2.0 ** -24 if weight is not None else 0.0))


def check(got, want, tol, what=""):
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(err[bad].max()), float(tol[bad].min()))
