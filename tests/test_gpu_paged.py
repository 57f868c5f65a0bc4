"""The paged cache on the GPU: single-token attention, append with norms and rotation, copies, compaction, against plain forms
in 64 bits; and a composed cache that goes on in pages."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2604_13226_b200 import binding as kvp

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def table_of(lens, page, n_pages, seed=0, cols=None, spare=-1):
    """Pages drawn in no order; `spare` behind a request's last page."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    order = torch.randperm(n_pages, generator=g)
    t = torch.full((len(lens), cols or max(1, max(need))), spare, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n].int()
        at += n
    assert at <= n_pages
    return t.cuda()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def run_attend(k, v, order, hq, q, table, lens, first=None, layer=0, scale=0.0, with_lse=True):
    c = kvp.PagedCache(k, v, hq, order=order, max_batch=max(1, q.shape[0]), softmax_scale=scale)
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, device="cuda") if with_lse else None
    c.attend(layer, q, table, ints(lens), out, lse=lse, first=None if first is None else ints(first))
    return c, out, lse


def check_attend(k, v, order, hq, q, table, lens, first=None, layer=0, scale=0.0):
    c, out, lse = run_attend(k, v, order, hq, q, table, lens, first, layer, scale)
    want = ref.attend(k, v, order, layer, q, table, lens, first, c.page_size, scale or q.shape[-1] ** -0.5)
    ref.check(out, want[0], want[2], "out")
    empty = want[1] == -math.inf
    assert torch.equal(lse == -math.inf, empty) and not out[empty].any()
    ref.check(lse[~empty], want[1][~empty], want[3][~empty], "lse")
    return out, lse


LENS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 100, 433]


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("hq,hkv", [(4, 2), (8, 1), (7, 1), (6, 6), (16, 2), (9, 1), (16, 1), (20, 1), (33, 1), (28, 4)])
@pytest.mark.parametrize("order,page", [("heads", 16), ("tokens", 16), ("heads", 1), ("tokens", 13), ("heads", 100)])
def test_attend(dtype, d, hq, hkv, order, page):
    n_pages = sum(-(-n // page) for n in LENS) + 2
    k, v = ref.pages((2, n_pages, hkv, page, d), order, DT[dtype], seed=hq + page)
    q = torch.randn(len(LENS), hq, d, device="cuda").to(DT[dtype])
    check_attend(k, v, order, hq, q, table_of(LENS, page, n_pages), LENS, layer=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[1], [5000], [2049, 0, 0, 1], [0, 0, 0], [1] * 33, [7, 300] * 35, [0] * 40 + [900] + [0] * 30, list(range(0, 300))])
def test_attend_batches(dtype, lens):
    """One request to three hundred, empty ones in front, behind and between."""
    page, hkv, hq, d = 16, 2, 8, 64
    n_pages = sum(-(-n // page) for n in lens) + 2
    k, v = ref.pages((1, n_pages, hkv, page, d), "heads", DT[dtype], seed=len(lens))
    q = torch.randn(len(lens), hq, d, device="cuda").to(DT[dtype])
    check_attend(k, v, "heads", hq, q, table_of(lens, page, n_pages), lens)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("hq,hkv", [(17, 1), (48, 2), (32, 1), (49, 1), (71, 1)])
@pytest.mark.parametrize("lens", [[1], [5000], [9, 0, 0, 333, 7000, 16], [7, 300] * 150])
def test_attend_many_heads_share_a_head(dtype, d, hq, hkv, lens):
    """Groups wider than a warp's rows: one unit or several, of a few rows or full, inside a CTA and cut into parts."""
    page = 16
    n_pages = sum(-(-n // page) for n in lens) + 2
    k, v = ref.pages((1, n_pages, hkv, page, d), "heads", DT[dtype], seed=hq)
    q = torch.randn(len(lens), hq, d, device="cuda").to(DT[dtype])
    check_attend(k, v, "heads", hq, q, table_of(lens, page, n_pages), lens)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (7, 1), (16, 1), (20, 1), (28, 4)])
@pytest.mark.parametrize("lens", [[60000], [30001, 3, 0, 9000, 17000]])
def test_attend_units_of_many_parts(dtype, d, hq, hkv, lens):
    """Units that dozens of CTAs share, joined in groups of parts first; twice on one cache, the second time the same."""
    page = 64
    n_pages = sum(-(-n // page) for n in lens) + 2
    k, v = ref.pages((1, n_pages, hkv, page, d), "tokens", DT[dtype], seed=hq)
    q = torch.randn(len(lens), hq, d, device="cuda").to(DT[dtype])
    table = table_of(lens, page, n_pages)
    out, lse = check_attend(k, v, "tokens", hq, q, table, lens)
    c = kvp.PagedCache(k, v, hq, order="tokens", max_batch=len(lens))
    for _ in range(2):
        again, lse_again = torch.empty_like(out), torch.empty_like(lse)
        c.attend(0, q, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), out=again, lse=lse_again)
        assert torch.equal(again, out) and torch.equal(lse_again, lse)
    c.close()


@pytest.mark.parametrize("dtype,hq", [("f32", 8), ("bf16", 8), ("bf16", 24)])
@pytest.mark.parametrize("page", [16, 24])
def test_attend_windows(dtype, hq, page):
    """A first visible row anywhere: at a page's border, inside it, at the length, behind it, far behind, negative."""
    lens = [100, 100, 100, 100, 100, 100, 500, 500, 33, 0, 1]
    first = [0, 16, 17, 99, 100, 2 ** 31 - 1, 48, 433, -5, 3, 0]
    n_pages = sum(-(-n // page) for n in lens) + 2
    k, v = ref.pages((1, n_pages, 2, page, 128), "tokens", DT[dtype], seed=3)
    q = torch.randn(len(lens), hq, 128, device="cuda").to(DT[dtype])
    check_attend(k, v, "tokens", hq, q, table_of(lens, page, n_pages), lens, first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -float("inf"), "lowest"])
def test_what_is_not_visible_is_not_read(dtype, fill):
    """Rows behind the length, in front of `first` and on pages of nobody hold NaN, infinities or the lowest value."""
    page, lens, first = 16, [1, 17, 40, 300, 0, 64], [0, 3, 16, 170, 0, 0]
    n_pages = sum(-(-n // page) for n in lens) + 3
    k, v = ref.pages((1, n_pages, 2, page, 64), "heads", DT[dtype], seed=4)
    q = torch.randn(len(lens), 8, 64, device="cuda").to(DT[dtype])
    table = table_of(lens, page, n_pages)
    seen = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
    for b, (f, n) in enumerate(zip(first, lens)):
        r = torch.arange(f, n, device="cuda")
        seen[table[b, r // page].long(), r % page] = True
    want = run_attend(k, v, "heads", 8, q, table, lens, first)[1:]
    x = torch.finfo(DT[dtype]).min if fill == "lowest" else fill
    hide = ~seen[None, :, None, :, None]
    got = run_attend(k.masked_fill(hide, x), v.masked_fill(hide, x), "heads", 8, q, table, lens, first)[1:]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_outside_the_store_are_not_followed(dtype):
    """A page number outside the store: its rows are not there; a request of such pages alone has no row.  Lengths beyond the
    table end with it, negative ones are none."""
    page, lens = 16, [100, 64, 10 ** 6, -3, 40]
    k, v = ref.pages((1, 30, 2, page, 64), "heads", DT[dtype], seed=5)
    table = table_of([100, 64, 112, 0, 40], page, 30, cols=7)
    table[0, 2] = 30
    table[0, 5] = 2 ** 31 - 1
    table[1, :4] = torch.tensor([-1, -2 ** 31, 30, 999])
    table[2, 6] = -7
    q = torch.randn(5, 4, 64, device="cuda").to(DT[dtype])
    out, lse = check_attend(k, v, "heads", 4, q, table, lens)
    assert not out[1].any() and not out[3].any()


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 32, 8), ("bf16", 64, 28, 4), ("f32", 128, 8, 2), ("bf16", 128, 16, 1)])
def test_long_and_short_together(dtype, d, hq, hkv):
    lens = [20000, 3, 7777, 0, 12345, 1]
    page = 64
    n_pages = sum(-(-n // page) for n in lens) + 2
    k, v = ref.pages((1, n_pages, hkv, page, d), "heads", DT[dtype], seed=6)
    q = 2 * torch.randn(len(lens), hq, d, device="cuda")
    check_attend(k, v, "heads", hq, q.to(DT[dtype]), table_of(lens, page, n_pages), lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_peaked_rows_and_scales(dtype):
    """Scores up to a few hundred, rising and falling along the cache, and a scale of the caller's."""
    n, page = 3001, 16
    k, v = ref.pages((1, 190, 2, page, 64), "heads", DT[dtype], seed=7)
    table = table_of([n, n], page, 190 * 2)[:, :188] % 190
    table[1] = table[0].flip(0)
    ramp = torch.linspace(0.1, 8.0, 190, device="cuda").to(DT[dtype])
    order = torch.empty(190, dtype=torch.long, device="cuda")
    order[table[0].long()] = torch.arange(188, device="cuda")
    k = k * ramp[order.clamp(0, 189)][None, :, None, None, None]
    q = 6 * torch.randn(2, 4, 64, device="cuda").to(DT[dtype])
    for scale in (0.0, 0.5):
        check_attend(k, v, "heads", 4, q, table, [n, n], scale=scale)


def test_strided_operands():
    """q out of a fused projection, out and the store as parts of larger tensors, a table with rows to spare."""
    page, hq, hkv, d = 16, 8, 2, 128
    lens = [50, 200, 0, 33]
    big = torch.randn(3, 40, 2, hkv, page, d + 64, device="cuda").bfloat16()
    k, v = big[:, :, 0, :, :, :d], big[:, :, 1, :, :, :d]
    qkv = torch.randn(4, (hq + 2 * hkv) * d, device="cuda").bfloat16()
    q = qkv[:, :hq * d].unflatten(-1, (hq, d))
    wide = torch.full((4, hq, 2 * d), 5.0, device="cuda").bfloat16()
    out = wide[..., d:]
    table = torch.full((4, 40), -1, dtype=torch.int32, device="cuda")
    table[:, :13] = table_of(lens, page, 40, cols=13)
    for layer in (0, 2):
        c = kvp.PagedCache(k, v, hq, max_batch=4)
        c.attend(layer, q, table[:, :13], ints(lens), out)
        want = ref.attend(k, v, "heads", layer, q, table[:, :13], lens, None, page, d ** -0.5)
        ref.check(out, want[0], want[2])
        assert bool((wide[..., :d] == 5.0).all())


def test_results_repeat_to_the_bit_and_streams_may_be_others():
    """The parts of a split request are joined in their order, whoever comes last; on any stream."""
    lens = [30000, 500, 9000]
    k, v = ref.pages((1, 700, 8, 64, 128), "heads", torch.bfloat16, seed=8)
    q = torch.randn(3, 32, 128, device="cuda").bfloat16()
    table = table_of(lens, 64, 700)
    c, out, lse = run_attend(k, v, "heads", 32, q, table, lens)
    n, s = ints(lens), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for i in range(50):
        o, e = torch.empty_like(out), torch.empty_like(lse)
        with torch.cuda.stream(s):
            c.attend(0, q, table, n, o, lse=e)
        s.synchronize()
        assert torch.equal(o, out) and torch.equal(e, lse)
    o = torch.empty_like(out)
    s.wait_stream(torch.cuda.current_stream())
    c.attend(0, q, table, n, o, stream=s)
    s.synchronize()
    assert torch.equal(o, out)


def test_a_captured_step_follows_growing_lengths():
    """append and attend of a step in a graph; replayed while positions, slots, lengths and the table change in place."""
    page, hq, hkv, d, B = 16, 8, 2, 64, 3
    k, v = ref.pages((1, 60, hkv, page, d), "heads", torch.bfloat16, seed=9)
    k0, v0 = k.clone(), v.clone()
    lens = [15, 40, 0]
    full = table_of([15 + 80, 40 + 80, 80], page, 60, cols=8)
    rope = kvp.Rope(d, theta=500000.0)
    c = kvp.PagedCache(k, v, hq, max_batch=B)
    qkv = torch.zeros(B, (hq + 2 * hkv) * d, device="cuda").bfloat16()
    q, kn, vn = (x.unflatten(-1, (-1, d)) for x in qkv.split((hq * d, hkv * d, hkv * d), -1))
    q_rot, out = torch.zeros(B, hq, d, device="cuda").bfloat16(), torch.zeros(B, hq, d, device="cuda").bfloat16()
    pos, slots, n = ints([0] * B), ints([-1] * B), ints(lens)
    table = torch.full_like(full, -1)

    def step():
        c.append(0, kn, vn, pos, slots, rope=rope, q=q, q_out=q_rot)
        c.attend(0, q_rot, table, n, out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    k.copy_(k0); v.copy_(v0)
    k2, v2 = k0.clone(), v0.clone()
    c2 = kvp.PagedCache(k2, v2, hq, max_batch=B)
    q2, out2 = torch.zeros_like(q_rot), torch.zeros_like(out)
    for i in range(60):
        qkv.copy_(torch.randn(qkv.shape, device="cuda"))
        at = [x + i for x in lens]
        pos.copy_(ints(at))
        slots.copy_(torch.stack([full[b, x // page] * page + x % page for b, x in enumerate(at)]))
        n.copy_(ints([x + 1 for x in at]))
        for b, x in enumerate(at):
            table[b, x // page] = full[b, x // page]
            table[b, :x // page] = full[b, :x // page]
        graph.replay()
        c2.append(0, kn, vn, pos, slots, rope=rope, q=q, q_out=q2)
        c2.attend(0, q2, table, n, out2)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(q_rot, q2) and torch.equal(k, k2) and torch.equal(v, v2)
    want = ref.attend(k, v, "heads", 0, q_rot, table, n.tolist(), None, page, d ** -0.5)
    ref.check(out, want[0], want[2])


def test_rows_beyond_four_gigabytes():
    """Offsets of pages that pass 32 bits, in bytes and in elements: append to them, attend to them, copy and compact them."""
    page, hkv, d, hq = 64, 8, 128, 32
    n_pages = 40000                                                # 5.2 GB of keys and as much of values
    k = torch.empty(1, n_pages, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    high = torch.arange(n_pages - 6, n_pages, device="cuda")
    low = torch.arange(0, 6, device="cuda")
    for t in (k, v):
        t[:, high] = torch.randn(1, 6, hkv, page, d, device="cuda").bfloat16()
        t[:, low] = 0
    c = kvp.PagedCache(k, v, hq, max_batch=2)
    kn, vn = (torch.randn(2, hkv, d, device="cuda").bfloat16() for _ in range(2))
    slots = ints([(n_pages - 1) * page + 5, 3])
    c.append(0, kn, vn, None, slots)
    assert torch.equal(k[0, n_pages - 1, :, 5], kn[0]) and torch.equal(v[0, n_pages - 1, :, 5], vn[0]) and torch.equal(k[0, 0, :, 3], kn[1])
    table = high.flip(0).int()[None].contiguous()
    q = torch.randn(1, hq, d, device="cuda").bfloat16()
    out = torch.empty_like(q)
    c.attend(0, q, table, ints([350]), out)
    want = ref.attend(k[:, high], v[:, high], "heads", 0, q, (table - (n_pages - 6)).contiguous(), [350], None, page, d ** -0.5)
    ref.check(out, want[0], want[2])
    c.copy([n_pages - 2], [1])
    assert torch.equal(k[0, 1], k[0, n_pages - 2]) and torch.equal(v[0, 1], v[0, n_pages - 2])
    kept = ints([1, 64, 200, 349])[None, None, None]
    c.compact(table, ints([350]), ints([[2]]), kept, ints([4]))
    for i, r in enumerate([1, 64, 200, 349]):
        assert torch.equal(k[0, 2, :, i], k[0, int(table[0, r // page]), :, r % page])


# ---- append ---------------------------------------------------------------------------------------------------------

ROPES = [dict(), dict(pairing=1), dict(rotary_dim=16), dict(rotary_dim=48, pairing=1), dict(rotary_dim=0),
         dict(theta=500000.0, scale=8.0, original_positions=8192), dict(scale=4.0, magnitude=1.1386), None]


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rope", ROPES, ids=str)
@pytest.mark.parametrize("n", [1, 3, 1301])
def test_append(dtype, d, norm, rope, n):
    hq, hkv, page, order = 6, 2, 16, "heads" if n != 3 else "tokens"
    dt = DT[dtype]
    n_pages = -(-n // page) + 4
    k, v = ref.pages((2, n_pages, hkv, page, d), order, dt, seed=n)
    was = k.clone(), v.clone()
    g = torch.Generator().manual_seed(n)
    slots = torch.randperm(n_pages * page, generator=g)[:n].int()
    pos = torch.randint(0, 2 ** 20, (n,), generator=g).int()
    if n > 2:
        slots[1], slots[2] = -1, n_pages * page                    # padding: written nowhere
        pos[0], pos[1], pos[2] = 0, -7, 2 ** 31 - 1
    slots, pos = slots.cuda(), pos.cuda()
    qkv = (3 * torch.randn(n, (hq + 2 * hkv) * d, device="cuda")).to(dt)
    q, kn, vn = (x.unflatten(-1, (-1, d)) for x in qkv.split((hq * d, hkv * d, hkv * d), -1))
    w = [(1 + 0.3 * torch.randn(d, device="cuda")).to(dt) if norm else None for _ in range(2)]
    r = kvp.Rope(d, **rope) if rope is not None else None
    c = kvp.PagedCache(k, v, hq, order=order)
    q_out, k_out = (torch.full((n, h, d), 9.0, device="cuda", dtype=dt) for h in (hq, hkv))
    c.append(1, kn, vn, pos, slots, rope=r, q=q, q_out=q_out, k_out=k_out, q_weight=w[0], k_weight=w[1], eps=1e-5)
    freqs = [] if rope is None else ref.frequencies(rope.get("rotary_dim", d), rope.get("theta", 10000.0), rope.get("scale", 1.0),
                                                    rope.get("original_positions", 0))
    m = 1.0 if rope is None else rope.get("magnitude", 1.0)
    for got, x, wt in ((q_out, q, w[0]), (k_out, kn, w[1])):
        want, tol = ref.norm_rotate(x, wt, 1e-5, pos, freqs, 0 if rope is None else rope.get("pairing", 0), m)
        ref.check(got, want, tol + 1.001 * ref.HALF_STEP[dt] * want.abs())
    if norm is False and not freqs:
        assert torch.equal(q_out, q) and torch.equal(k_out, kn)
    for t, old, new in ((k, was[0], k_out), (v, was[1], vn)):
        want = old.clone()
        for i in range(n):
            s = int(slots[i])
            if 0 <= s < n_pages * page:
                if order == "heads":
                    want[1, s // page, :, s % page] = new[i]
                else:
                    want[1, s // page, s % page] = new[i]
        assert torch.equal(t, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 40, 1500])
def test_norm_rope_without_pages(dtype, n):
    """q and k alone, together, in place; an output between other data is all that is written."""
    d, hq, hkv, dt = 128, 5, 3, DT[dtype]
    rope = kvp.Rope(d, rotary_dim=64, theta=1e6)
    pos = torch.arange(1000, 1000 + n, device="cuda", dtype=torch.int32)
    x = torch.randn(n, hq + hkv, d, device="cuda").to(dt)
    q, k = x[:, :hq], x[:, hq:]
    w = (1 + torch.rand(d, device="cuda")).to(dt)
    wide = torch.full((n, hq, 2 * d), 5.0, device="cuda", dtype=dt)
    ko = torch.empty(n, hkv, d, device="cuda", dtype=dt)
    kvp.norm_rope(q, k, pos, rope, wide[..., :d], ko, q_weight=w)
    f = ref.frequencies(64, 1e6)
    for got, src, wt in ((wide[..., :d], q, w), (ko, k, None)):
        want, tol = ref.norm_rotate(src, wt, 1e-6, pos, f, 0, 1.0)
        ref.check(got, want, tol + 1.001 * ref.HALF_STEP[dt] * want.abs())
    assert bool((wide[..., d:] == 5.0).all())
    alone = torch.empty_like(ko)
    kvp.norm_rope(None, k, pos, rope, None, alone)
    assert torch.equal(alone, ko)
    y = x.clone()
    kvp.norm_rope(y[:, :hq], y[:, hq:], pos, rope, y[:, :hq], y[:, hq:], q_weight=w)
    assert torch.equal(y[:, :hq], wide[..., :d]) and torch.equal(y[:, hq:], ko)
    kvp.norm_rope(q[:0], None, pos[:0], rope, wide[:0, :, :d])


def test_rotation_keeps_relative_positions():
    """q at p + t against k at p gives the same scores wherever p lies: the identity that re-basing of packets rests on."""
    d = 128
    rope = kvp.Rope(d, theta=500000.0)
    q, k = torch.randn(1, 1, d, device="cuda"), torch.randn(1, 1, d, device="cuda")
    scores = []
    for p in (0, 1000, 131072, 10 ** 6):
        a, b = torch.empty_like(q), torch.empty_like(k)
        kvp.norm_rope(q, None, ints([p + 77]), rope, a)
        kvp.norm_rope(None, k, ints([p]), rope, None, b)
        scores.append(float((a.double() * b.double()).sum()))
    # each factor is off by 2^-20 of its pair's magnitudes at most, both together by 2^-19, and a score has d / 2 pairs
    bound = float(2 ** -18 * (q.abs().double().sum() * k.abs().double().max()))
    assert max(scores) - min(scores) <= bound


# ---- copy, fork, compact ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d,order", [("f32", 64, "heads"), ("bf16", 128, "heads"), ("bf16", 64, "tokens"), ("f32", 128, "tokens")])
@pytest.mark.parametrize("page,n", [(16, 1), (16, 40), (1, 7), (37, 300), (37, 301), (200, 9), (5, 1301), (5, 2700)])
def test_copy(dtype, d, order, page, n):
    layers, hkv = 3, 2
    k, v = ref.pages((layers, 2 * n + 1, hkv, page, d), order, DT[dtype], seed=n)
    c = kvp.PagedCache(k, v, 4, order=order)
    g = torch.Generator().manual_seed(n)
    p = torch.randperm(2 * n + 1, generator=g).tolist()
    dst, src = p[:n], [p[n + i // 2] for i in range(n)]            # every page twice
    rows = torch.randint(0, page + 1, (n,), generator=g).tolist()
    want = k.clone(), v.clone()
    head, row = (3, 2) if order == "tokens" else (2, 3)
    for w in want:
        old = w.clone()
        for s, t, r in zip(src, dst, rows):
            w[:, t].narrow(row - 1, 0, r).copy_(old[:, s].narrow(row - 1, 0, r))
    c.copy(src, dst, rows)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    c.copy(src, dst)
    assert torch.equal(k[:, dst], k[:, src]) and torch.equal(v[:, dst], v[:, src])
    c.copy([], [])


def test_fork_copies_the_last_page_of_each():
    page, n = 16, 37
    k, v = ref.pages((2, 20, 2, page, 64), "heads", torch.bfloat16, seed=1)
    c = kvp.PagedCache(k, v, 4)
    p = c.take(3)
    forks = c.fork(p, n, 4)
    assert all(f[:2] == p[:2] for f in forks) and len({f[2] for f in forks} | {p[2]}) == 5 and c.free_pages == 13
    for f in forks:
        assert torch.equal(k[:, f[2], :, :5], k[:, p[2], :, :5]) and torch.equal(v[:, f[2], :, :5], v[:, p[2], :, :5])
    with pytest.raises(kvp.KvpError) as e:
        c.fork(p, n, 14)
    assert e.value.code == 2 and c.free_pages == 13
    c.release(p)
    for f in forks:
        c.release(f)
    assert c.free_pages == 20


@pytest.mark.parametrize("dtype,d,order", [("f32", 64, "heads"), ("bf16", 128, "heads"), ("bf16", 64, "tokens")])
@pytest.mark.parametrize("page", [1, 16, 30])
@pytest.mark.parametrize("per_layer,per_head", [(True, True), (False, True), (True, False), (False, False)])
def test_compact(dtype, d, order, page, per_layer, per_head):
    layers, hkv = 2, 3
    lens, n_kept = [1, 70, 200, 33, 0], [1, 64, 65, 0, 0]
    need = sum(-(-n // page) for n in lens)
    n_pages = need + sum(-(-n // page) for n in n_kept) + 2
    k, v = ref.pages((layers, n_pages, hkv, page, d), order, DT[dtype], seed=page)
    table = table_of(lens, page, need)
    new = torch.where((t := table_of(n_kept, page, n_pages - need)) >= 0, t + need, t)
    kept = torch.full((5, layers if per_layer else 1, hkv if per_head else 1, 70), -1, dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(page)
    for b, (n, m) in enumerate(zip(lens, n_kept)):
        for l in range(kept.shape[1]):
            for h in range(kept.shape[2]):
                kept[b, l, h, :m] = torch.randperm(n, generator=g)[:m].sort().values.int().cuda()
    if page == 16:
        kept[1, 0, 0, 3], kept[2, 0, 0, 64], kept[1, 0, 0, 5] = 70, 2 ** 31 - 1, -9       # not rows of theirs: left as it is
    want = k.clone(), v.clone()
    for w, t in zip(want, (k, v)):
        for b, m in enumerate(n_kept):
            for l in range(layers):
                for h in range(hkv):
                    for i in range(m):
                        r = int(kept[b, l if per_layer else 0, h if per_head else 0, i])
                        if 0 <= r < lens[b]:
                            x = ref.row_of(t, order, l, int(table[b, r // page]), h, r % page)
                            ref.row_of(w, order, l, int(new[b, i // page]), h, i % page).copy_(x)
    c = kvp.PagedCache(k, v, 3, order=order)
    c.compact(table, ints(lens), new, kept, ints(n_kept))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_compact_leaves_alone_what_lies_outside():
    """Pages outside the store, lists longer than the new pages or than the count says."""
    k, v = ref.pages((1, 8, 2, 4, 64), "heads", torch.float32, seed=2)
    was = k.clone()
    c = kvp.PagedCache(k, v, 2)
    kept = torch.arange(8, device="cuda", dtype=torch.int32).expand(1, 1, 1, 8)
    c.compact(ints([[0, 8]]), ints([8]), ints([[2]]), kept, ints([100]))
    assert torch.equal(k[0, 2], was[0, 0])
    k[0, 2] = was[0, 2]
    assert torch.equal(k, was)
    c.compact(ints([[0, 1]]), ints([8]), ints([[-1, 99]]), kept, ints([8]))
    c.compact(ints([[0, 1]]), ints([8]), ints([[2, 3]]), kept, ints([-4]))
    assert torch.equal(k, was)


# ---- together ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 8, 2), ("bf16", 64, 4, 2), ("f32", 64, 4, 2)])
def test_a_composed_cache_goes_on_in_pages(dtype, d, hq, hkv):
    """Packets are composed and asked; the cache is exported into pages and three answers fork from it, each generated token by
    token: what the first one sees is what the composed cache gives when the same tokens continue it there."""
    from paper_2604_13226_b200 import inputs as gen
    from paper_2604_13226_b200.session import Session
    page, steps, ql = 16, 20, 24
    shape = gen.ModelShape(2, hq, hkv, d, dtype, 500000.0, 0)
    wl = gen.make_workload(shape, [100, 37, 260], [[(0, 0), (2, 0), (1, 0)]], q_len=ql, seed=3)
    sess = Session(wl, max_query_tokens=ql + steps)
    ctx, dt = sess.ctx, DT[dtype]
    aid, (prefix,) = ctx.assemble(wl.items)
    k = torch.zeros(2, 120, hkv, page, d, dtype=dt, device="cuda")
    v = torch.zeros_like(k)
    cache = kvp.PagedCache(k, v, hq, max_batch=3)
    n = prefix + ql
    mine = cache.take(-(-n // page))
    rows = torch.arange(n)
    slots = ints([mine[r // page] * page + r % page for r in rows.tolist()])
    for layer in range(2):
        q, kn, vn = sess.query_tensors(layer)
        ctx.query_prefill(aid, layer, q, kn, vn, ql, torch.empty_like(q))
        ck, cv = ctx.export_cache(aid, layer, 0, prefix, ql)
        cache.append(layer, ck, cv, None, slots)
    lists = [mine] + cache.fork(mine, n, 2)
    rope = kvp.Rope(d, theta=500000.0)
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(steps):
        if (n + i) % page == 0:
            for x in lists:
                x += cache.take(1)
        at = n + i
        table = ints([x + [-1] * (120 - len(x)) for x in lists])
        lens, pos = ints([at + 1] * 3), ints([at] * 3)
        slot = ints([x[at // page] * page + at % page for x in lists])
        for layer in range(2):
            q = torch.randn(3, hq, d, generator=g, device="cuda").to(dt)
            kn, vn = (torch.randn(3, hkv, d, generator=g, device="cuda").to(dt) for _ in range(2))
            rot, out = torch.empty_like(q), torch.empty_like(q)
            cache.append(layer, kn, vn, pos, slot, rope=rope, q=q, q_out=rot)
            cache.attend(layer, rot, table, lens, out)
            want = ref.attend(k, v, "heads", layer, rot, table, lens.tolist(), None, page, d ** -0.5)
            ref.check(out, want[0], want[2])
            there = torch.empty(1, 1, hq, d, device="cuda", dtype=dt)
            ctx.query_prefill(aid, layer, q[:1, None].contiguous(), kn[:1, None].contiguous(), vn[:1, None].contiguous(), 1, there,
                              flags=kvp.CONTINUE | kvp.ROPE_QUERY)
            # both within the documented bounds of the same attention; the composed one rotates q where pages hold rotated keys
            tol = 2e-2 if dtype == "bf16" else 2e-5
            assert float((there[0, 0].double() - out[0].double()).abs().max()) <= tol
    # the forks went ways of their own, the question's whole pages are still everybody's
    assert all(x[:n // page] == mine[:n // page] for x in lists) and len({x[-1] for x in lists}) == 3
    # one of them is thinned out per head and goes on, at the positions it was at
    total, keep = n + steps, (n + steps) // 2
    kept = torch.rand(1, 2, hkv, total, generator=g, device="cuda").topk(keep, -1).indices.sort(-1).values.int().contiguous()
    new = cache.take(-(-(keep + 1) // page))
    table = ints([lists[1]])
    cache.compact(table, ints([total]), ints([new]), kept, ints([keep]))
    q = torch.randn(1, hq, d, generator=g, device="cuda").to(dt)
    kn, vn = (torch.randn(1, hkv, d, generator=g, device="cuda").to(dt) for _ in range(2))
    rot, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(1, hq, device="cuda")
    cache.append(1, kn, vn, ints([total]), ints([new[keep // page] * page + keep % page]), rope=rope, q=q, q_out=rot)
    cache.attend(1, rot, ints([new]), ints([keep + 1]), out, lse=lse)
    old = ref.gather(k, "heads", 1, table[0], page, torch.arange(total, device="cuda")), ref.gather(v, "heads", 1, table[0], page, torch.arange(total, device="cuda"))
    last = [ref.row_of(t, "heads", 1, new[keep // page], slice(None), keep % page).double() for t in (k, v)]
    for h in range(hkv):
        K, V = (torch.cat([t[kept[0, 1, h].long(), h], x[h][None]]) for t, x in zip(old, last))
        s = rot[0].double().view(hkv, -1, d)[h] @ K.T * d ** -0.5
        got = out[0].double().view(hkv, -1, d)[h]
        want = s.softmax(-1) @ V
        tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * want.abs() + 2.0 ** -12 * (s.softmax(-1) @ V.abs())
        ref.check(got, want, tol)
    for x in lists + [new]:
        cache.release(x)
    assert cache.free_pages == 120
    sess.close()
