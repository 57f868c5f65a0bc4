"""Calls on the paged cache as programs make them: queued without a wait among the library's other calls, on two streams at once,
recorded into graphs, over stores of unusual strides, with nothing to do."""
import pytest
import torch

import paged_reference as ref
from paper_2604_13226_b200 import binding as kvp
from paper_2604_13226_b200 import inputs as gen
from paper_2604_13226_b200.session import Session
from test_gpu_paged import check_attend, ints, table_of

pytestmark = pytest.mark.gpu


def test_queued_among_the_other_calls():
    """assemble, prefill, norm_rope into the next prefill, append, attend, copy, compact: every call's kernel may begin while the
    one in front ends.  A hundred rounds queued without a wait give the bits of a round that waits after every call."""
    hq, hkv, d, page, ql = 8, 2, 128, 16, 16
    shape = gen.ModelShape(2, hq, hkv, d, "bf16", 500000.0, 0)
    wl = gen.make_workload(shape, [200, 333, 64, 500], [[(0, 0), (2, 0)], [(3, 0), (1, 0)]], q_len=ql, seed=4)
    sess = Session(wl, max_assemblies=2)
    rope = kvp.Rope(d, theta=500000.0)
    w = (1 + torch.rand(d, device="cuda")).bfloat16()
    qkv = [sess.query_tensors(layer) for layer in range(2)]
    pos = torch.arange(2 * ql, device="cuda", dtype=torch.int32)
    lens, slots = ints([64 + ql, 40 + ql]), ints([b * 8 * page + n + i for b, n in ((0, 64), (1, 40)) for i in range(ql)])
    table = torch.arange(16, device="cuda", dtype=torch.int32).view(2, 8)
    new, kept = table + 16, torch.arange(0, 40, 2, device="cuda", dtype=torch.int32).expand(2, 1, 1, 20)
    k0, v0 = ref.pages((2, 40, hkv, page, d), "heads", torch.bfloat16, seed=1)

    def round_(wait):
        step = torch.cuda.synchronize if wait else (lambda: None)
        k, v = k0.clone(), v0.clone()
        step()
        cache = kvp.PagedCache(k, v, hq, max_batch=2)
        out = [torch.empty(2, ql, hq, d, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        q1, k1 = torch.empty(2 * ql, hq, d, device="cuda", dtype=torch.bfloat16), torch.empty(2 * ql, hkv, d, device="cuda", dtype=torch.bfloat16)
        att, rot = torch.empty(2, hq, d, device="cuda", dtype=torch.bfloat16), torch.empty(2 * ql, hq, d, device="cuda", dtype=torch.bfloat16)
        aid, _ = sess.ctx.assemble(wl.items)
        step()
        sess.ctx.query_prefill(aid, 0, *qkv[0], ql, out[0])
        step()
        kvp.norm_rope(qkv[1][0].view(2 * ql, hq, d), qkv[1][1].view(2 * ql, hkv, d), pos, rope, q1, k1, q_weight=w, k_weight=w)
        step()
        sess.ctx.query_prefill(aid, 1, q1, k1, qkv[1][2], ql, out[1])
        step()
        cache.append(1, k1, out[1].view(2 * ql, hq, d)[:, :hkv], pos, slots, rope=rope, q=q1, q_out=rot)
        step()
        cache.attend(1, rot[::ql].contiguous(), table, lens, att)
        step()
        cache.copy([3], [39])
        step()
        cache.compact(table, lens, new, kept, ints([20, 20]))
        step()
        return out + [q1, k1, att, rot, k, v], cache

    want, _ = round_(True)
    got = [round_(False) for _ in range(100)]
    torch.cuda.synchronize()
    for tensors, _ in got:
        for a, b in zip(tensors, want):
            assert torch.equal(a, b)
    sess.close()


def test_two_caches_on_two_streams():
    """A cache has its own workspace: split requests of two caches, on a stream each, at the same time."""
    cases = []
    for seed, (hq, hkv, d, dt) in enumerate([(32, 8, 128, torch.bfloat16), (16, 1, 64, torch.bfloat16)]):
        lens = [9000 + 100 * seed, 50, 4000]
        k, v = ref.pages((1, 220, hkv, 64, d), "heads", dt, seed=seed)
        q = torch.randn(3, hq, d, device="cuda").to(dt)
        cases.append((kvp.PagedCache(k, v, hq, max_batch=3), q, table_of(lens, 64, 220), ints(lens)))
    want = []
    for c, q, t, n in cases:
        out = torch.empty_like(q)
        c.attend(0, q, t, n, out)
        want.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.empty_like(w) for _ in range(60)] for w in want]
    for s in streams:
        with torch.cuda.stream(s):
            torch.cuda._sleep(10_000_000)                          # both queues fill up meanwhile
    for i in range(60):
        for (c, q, t, n), s, o in zip(cases, streams, outs):
            c.attend(0, q, t, n, o[i], stream=s)
    torch.cuda.synchronize()
    for w, os in zip(want, outs):
        assert all(torch.equal(o, w) for o in os)


def test_two_graphs_share_a_cache():
    """Calls of one cache recorded into two graphs (batches of two sizes), replayed in turn, with eager calls between."""
    k, v = ref.pages((1, 300, 8, 64, 128), "heads", torch.bfloat16, seed=2)
    c = kvp.PagedCache(k, v, 32, max_batch=4)
    runs = []
    for lens in ([15000], [700, 1, 9000, 0]):
        q = torch.randn(len(lens), 32, 128, device="cuda").bfloat16()
        t, n, out = table_of(lens, 64, 300), ints(lens), torch.empty_like(q)
        c.attend(0, q, t, n, out)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.attend(0, q, t, n, out)
        runs.append((g, q, t, n, out, out.clone()))
    for i in range(30):
        for g, q, t, n, out, want in runs:
            out.zero_()
            g.replay()
            if i % 3 == 0:
                eager = torch.empty_like(out)
                c.attend(0, q, t, n, eager)
                assert torch.equal(eager, want)
            assert torch.equal(out, want)


def test_recorded_copies_compaction_and_norms():
    k, v = ref.pages((2, 30, 2, 16, 64), "tokens", torch.float32, seed=3)
    c = kvp.PagedCache(k, v, 4, order="tokens")
    x, y = torch.randn(40, 4, 64, device="cuda"), torch.empty(40, 4, 64, device="cuda")
    pos, rope = torch.arange(40, device="cuda", dtype=torch.int32), kvp.Rope(64)
    table, new, kept = ints([[0, 1, 2]]), ints([[5, 6]]), torch.arange(1, 41, 2, device="cuda", dtype=torch.int32)[None, None, None]
    n, m = ints([48]), ints([20])

    def calls():
        c.copy([0, 1], [10, 11], rows=[3, 16])
        c.compact(table, n, new, kept, m)
        kvp.norm_rope(x, None, pos, rope, y)

    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for i in range(3):
        k[:, :3].normal_()
        x.normal_()
        m.fill_(20 - i)
        k[:, 5:7] = 7.0
        g.replay()
        z = torch.empty_like(y)
        kvp.norm_rope(x, None, pos, rope, z)
        torch.cuda.synchronize()
        assert torch.equal(y, z) and torch.equal(k[:, 10, :3], k[:, 0, :3]) and torch.equal(k[:, 11], k[:, 1])
        rows = torch.arange(1, 41, 2, device="cuda")[:20 - i]
        assert torch.equal(k[:, 5:7].flatten(1, 2)[:, :20 - i], k[:, rows // 16, rows % 16]) and bool((k[:, 5:7].flatten(1, 2)[:, 20 - i:] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("what", ["layers_inside_pages", "rows_apart", "k_and_v_of_a_token_together", "one_large_page"])
def test_stores_of_other_strides(dtype, what):
    hq, hkv, d, page, P = 8, 2, 64, 16, 30
    lens = [100, 0, 257, 16]
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    order = "tokens"
    if what == "layers_inside_pages":
        k, v = (rnd(P, 3, page, hkv, d).transpose(0, 1) for _ in range(2))
    elif what == "rows_apart":                                     # 16 bytes behind every row that are nobody's
        k, v = (rnd(3, P, page, hkv, d + 16 // dtype.itemsize)[..., :d] for _ in range(2))
    elif what == "k_and_v_of_a_token_together":
        both = rnd(3, P, page, 2, hkv, d)
        k, v = both[:, :, :, 0], both[:, :, :, 1]
    else:
        page, P, order = 300, 4, "heads"
        k, v = (rnd(3, P, hkv, page, d) for _ in range(2))
    q = rnd(4, hq, d)
    table = table_of(lens, page, P)
    was = k.clone(), v.clone()
    for layer in range(3):
        check_attend(k, v, order, hq, q, table, lens, layer=layer)
    c = kvp.PagedCache(k, v, hq, order=order)
    kn, vn = rnd(2, hkv, d), rnd(2, hkv, d)
    spare = P - 1
    c.append(2, kn, vn, None, ints([spare * page + 1, spare * page + page - 1]))
    for t, w, x in ((k, was[0], kn), (v, was[1], vn)):
        for i, r in enumerate((1, page - 1)):
            ref.row_of(w, order, 2, spare, slice(None), r).copy_(x[i])
        assert torch.equal(t, w)
    c.copy([0], [spare], rows=[page - 1])
    for t, w in ((k, was[0]), (v, was[1])):
        row = 3 if order == "heads" else 2
        w[:, spare].narrow(row - 1, 0, page - 1).copy_(w[:, 0].narrow(row - 1, 0, page - 1))
        assert torch.equal(t, w)


def test_shared_tables_and_queries():
    """One list of pages and one query for all requests, by strides of zero: each sees its own length of it."""
    k, v = ref.pages((1, 20, 2, 16, 64), "heads", torch.bfloat16, seed=6)
    lens = [1, 50, 300, 17, 0]
    table = table_of([300], 16, 20).expand(5, -1)
    q = torch.randn(1, 8, 64, device="cuda").bfloat16().expand(5, -1, -1)
    check_attend(k, v, "heads", 8, q, table, lens)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_thousands_of_requests(dtype):
    g = torch.Generator().manual_seed(0)
    lens = torch.randint(0, 40, (3000,), generator=g).tolist()
    need = sum(-(-n // 16) for n in lens)
    k, v = ref.pages((1, need + 1, 1, 16, 64), "heads", dtype, seed=7)
    q = torch.randn(3000, 4, 64, device="cuda").to(dtype)
    check_attend(k, v, "heads", 4, q, table_of(lens, 16, need + 1), lens)


def test_calls_with_nothing_to_do():
    k, v = ref.pages((1, 4, 2, 16, 64), "heads", torch.bfloat16, seed=8)
    was = k.clone()
    c = kvp.PagedCache(k, v, 4)
    e = lambda *s: torch.empty(s, device="cuda", dtype=torch.bfloat16)
    i = lambda *s: torch.empty(s, device="cuda", dtype=torch.int32)
    c.append(0, e(0, 2, 64), e(0, 2, 64), i(0), i(0), rope=kvp.Rope(64), q=e(0, 4, 64), q_out=e(0, 4, 64))
    kvp.norm_rope(e(0, 4, 64), None, i(0), kvp.Rope(64), e(0, 4, 64))
    c.attend(0, e(0, 4, 64), i(0, 3), i(0), e(0, 4, 64))
    c.copy([], [])
    c.compact(i(0, 3), i(0), i(0, 3), i(0, 1, 1, 4), i(0))
    c.compact(i(2, 3), i(2), i(2, 3), i(2, 1, 1, 0), i(2))
    out = torch.full((2, 4, 64), 3.0, device="cuda").bfloat16()
    c.attend(0, torch.randn_like(out), i(2, 0), ints([5, 0]), out)                # tables without a column
    torch.cuda.synchronize()
    assert torch.equal(k, was) and not out.any()


def test_a_cache_that_goes_while_something_is_recorded():
    """Destroying a cache does not wait for the device while a graph is recorded, and leaves the recording whole."""
    k, v = ref.pages((1, 4, 2, 16, 64), "heads", torch.bfloat16, seed=9)
    old, c = kvp.PagedCache(k, v, 4), kvp.PagedCache(k, v, 4)
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    out, want = torch.empty_like(q), torch.empty_like(q)
    t, n = ints([[0, 1]]), ints([20])
    c.attend(0, q, t, n, want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attend(0, q, t, n, out)
        old.close()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype,d", [(torch.float32, 64), (torch.bfloat16, 128), (torch.bfloat16, 64)])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (7, 1), (12, 3), (33, 11), (0, 2)])
@pytest.mark.parametrize("n", [591, 592, 700, 1184, 1185, 5000])
def test_appends_of_every_length(dtype, d, hq, hkv, n):
    """Few tokens, a few thousand, many: each has its own way to share heads out, odd numbers of heads among them."""
    page, n_pages = 16, -(-n // 16) + 1
    k, v = ref.pages((1, n_pages, hkv, page, d), "heads", dtype, seed=n)
    c = kvp.PagedCache(k, v, max(1, hq) * hkv if hq % hkv else max(hq, hkv))
    qkv = torch.randn(n, max(1, c.n_q_heads) + 2 * hkv, d, device="cuda").to(dtype)
    nq = c.n_q_heads if hq else 0
    q, kn, vn = (qkv[:, :nq], qkv[:, nq:nq + hkv], qkv[:, nq + hkv:nq + 2 * hkv])
    g = torch.Generator().manual_seed(n)
    slots = torch.randperm(n_pages * page, generator=g)[:n].int().cuda()
    pos = torch.randint(0, 1 << 17, (n,), generator=g).int().cuda()
    w = (1 + 0.2 * torch.randn(d, device="cuda")).to(dtype)
    q_out = torch.empty(n, nq, d, device="cuda", dtype=dtype) if nq else None
    c.append(0, kn, vn, pos, slots, rope=kvp.Rope(d, rotary_dim=48, theta=1e6), q=q if nq else None, q_out=q_out, q_weight=w if nq else None, k_weight=w)
    f = ref.frequencies(48, 1e6)
    s = slots.long()
    got = [(k[0, s // page, :, s % page], kn)] + ([(q_out, q)] if nq else [])
    for x, src in got:
        want, tol = ref.norm_rotate(src, w, 1e-6, pos, f, 0, 1.0)
        ref.check(x, want, tol + 1.001 * ref.HALF_STEP[dtype] * want.abs())
    assert torch.equal(v[0, s // page, :, s % page], vn)


@pytest.mark.parametrize("batch", [3, 40])
@pytest.mark.parametrize("tokens", [1, 500, 30000])
def test_lengths_written_by_the_call_in_front(batch, tokens):
    """An attend may begin while the kernel in front of it ends.  Here that kernel writes its lengths - rows that norm_rope hands
    through unchanged, whose bits are the lengths - other ones every time."""
    page, hq, hkv, d = 16, 8, 2, 64
    most = [900, 40, 3000] + [20] * (batch - 3)
    n_pages = sum(-(-n // page) for n in most)
    k, v = ref.pages((1, n_pages, hkv, page, d), "heads", torch.bfloat16, seed=1)
    c = kvp.PagedCache(k, v, hq, max_batch=batch)
    q = torch.randn(batch, hq, d, device="cuda").bfloat16()
    table = table_of(most, page, n_pages)
    sets = [most, [1] * batch, [0, 40, 2999] + [0] * (batch - 3), [900, 0, 0] + [19] * (batch - 3), [0] * batch]
    rows, want = [], []
    for lens in sets:
        r = torch.zeros(tokens, 1, d, device="cuda")
        r.view(torch.int32)[-1, 0, :batch] = ints(lens)
        rows.append(r)
        out = torch.empty_like(q)
        c.attend(0, q, table, ints(lens), out)
        want.append(out)
        assert ref.attend(k, v, "heads", 0, q, table, lens, None, page, d ** -0.5)[0].sub(out.double()).abs().max() < 0.02
    written = torch.zeros(tokens, 1, d, device="cuda")
    lens = written.view(torch.int32)[-1, 0, :batch]
    outs = [torch.empty_like(q) for _ in range(200)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        kvp.norm_rope(rows[i % 5], None, None, None, written)
        c.attend(0, q, table, lens, out)
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        assert torch.equal(out, want[i % 5]), i
