"""The paged cache without a GPU: what is refused, who holds which pages, frequencies."""
import ctypes
import math
import random

import pytest
import torch

import paged_reference as ref
from paper_2604_13226_b200 import binding as kvp

INVALID, CAPACITY, STATE = 1, 2, 4


def cache(layers=2, pages=12, heads=2, size=4, d=64, hq=4, dtype=torch.float32, order="heads", **kw):
    shape = (layers, pages, heads, size, d) if order == "heads" else (layers, pages, size, heads, d)
    k = torch.zeros(shape, dtype=dtype)
    return kvp.PagedCache(k, torch.zeros_like(k), hq, order=order, **kw)


def refused(code, call, *a, **kw):
    with pytest.raises(kvp.KvpError) as e:
        call(*a, **kw)
    assert e.value.code == code and len(str(e.value)) > len("KVP_ERR_INVALID: "), e.value
    return str(e.value)


@pytest.mark.parametrize("make", [
    lambda: cache(d=32), lambda: cache(d=96), lambda: cache(hq=3), lambda: cache(hq=0), lambda: cache(max_batch=0), lambda: cache(pages=0),
    lambda: cache(size=0), lambda: cache(softmax_scale=-1.0), lambda: cache(softmax_scale=math.nan), lambda: cache(softmax_scale=math.inf),
    lambda: cache(dtype=torch.float16), lambda: kvp.PagedCache(torch.zeros(2, 3, 2, 4, 64), torch.zeros(2, 3, 2, 5, 64), 4),
    lambda: kvp.PagedCache(torch.zeros(2, 3, 2, 4, 64), torch.zeros(2, 3, 4, 2, 64).transpose(2, 3), 4), lambda: cache(order="rows"),
    lambda: kvp.PagedCache(torch.zeros(3, 2, 4, 64), torch.zeros(3, 2, 4, 64), 4),
    lambda: kvp.PagedCache(*[torch.zeros(1, 1, 1, 4, 64).expand(1, 9, 2, 4, 64) for _ in range(2)], 4),       # pages on top of one another
    lambda: kvp.PagedCache(*[torch.zeros(2, 3, 2, 4, 66)[..., :64] for _ in range(2)], 4),                     # rows of 264 bytes
    lambda: kvp.PagedCache(*[torch.zeros(2, 3, 2, 4, 128)[..., ::2] for _ in range(2)], 4),
    lambda: kvp.PagedCache(*[torch.zeros(4000).as_strided((2, 3, 2, 4, 64), (1024, 256, 128, 64, 1)) for _ in range(2)], 4),    # heads over one another
    lambda: kvp.PagedCache(*[torch.zeros(4000).as_strided((2, 3, 2, 4, 64), (512, 512, 256, 64, 1)) for _ in range(2)], 4),     # layers over pages
])
def test_configurations_that_are_refused(make):
    refused(INVALID, make)


def test_counts_beyond_32_bits_are_refused():
    c = cache().cfg
    size = lambda **kw: kvp.lib().kvp_cache_workspace_bytes(ctypes.byref(type(c).from_buffer_copy(bytes(c)))) if not kw else _with(c, kw)
    assert size() > 0
    for kw in (dict(n_pages=1 << 20, page_size=1 << 12), dict(page_size=1 << 24), dict(n_layers=40000), dict(max_batch=1 << 20),
               dict(struct_bytes=8), dict(row_stride=-64), dict(row_stride=66), dict(page_stride=0), dict(head_stride=1 << 60)):
        assert size(**kw) == 0, kw


def _with(c, kw):
    x = type(c).from_buffer_copy(bytes(c))
    for k, v in kw.items():
        setattr(x, k, v)
    return kvp.lib().kvp_cache_workspace_bytes(ctypes.byref(x))


def test_null_pointers():
    L = kvp.lib()
    assert L.kvp_cache_create(None, None) == INVALID
    h = ctypes.c_void_p()
    assert L.kvp_cache_create(None, ctypes.byref(h)) == INVALID and not h and L.kvp_cache_last_error(None)
    for call in (lambda: L.kvp_cache_destroy(None), lambda: L.kvp_cache_take(None, 1, None), lambda: L.kvp_cache_append(None, 0, None, None, None),
                 lambda: L.kvp_cache_copy(None, 0, None, None, None, None), lambda: L.kvp_cache_free_pages(None, None),
                 lambda: L.kvp_cache_fork(None, 0, None, 0, None, None), lambda: L.kvp_cache_share(None, 0, None),
                 lambda: L.kvp_cache_release(None, 0, None), lambda: L.kvp_rope_frequencies(None, None),
                 lambda: L.kvp_cache_attend(None, 0, 0, None, None, None, 0, 0, None, None, None, None, None, None),
                 lambda: L.kvp_cache_compact(None, 0, None, 0, 0, None, None, 0, 0, None, None, 0, None, None)):
        assert call() == INVALID
    assert L.kvp_cache_workspace_bytes(None) == 0
    c = cache()
    for rc in (L.kvp_cache_take(c._h, 1, None), L.kvp_cache_take(c._h, -1, None), L.kvp_cache_share(c._h, 1, None), L.kvp_cache_release(c._h, 1, None),
               L.kvp_cache_copy(c._h, 1, None, None, None, None), L.kvp_cache_copy(c._h, -1, None, None, None, None),
               L.kvp_cache_free_pages(c._h, None), L.kvp_cache_append(c._h, 0, None, None, None),
               L.kvp_cache_attend(c._h, 0, 1, None, None, None, 0, 1, None, None, None, None, None, None),
               L.kvp_cache_attend(c._h, 0, -1, None, None, None, 0, 1, None, None, None, None, None, None),
               L.kvp_cache_compact(c._h, 1, None, 0, 1, None, None, 0, 1, None, None, 1, None, None)):
        assert rc == INVALID
        assert L.kvp_cache_last_error(c._h)


# ---- pages --------------------------------------------------------------------------------------------------------

def test_pages_are_held_as_a_model_holds_them():
    """Random takes, shares, releases and forks of whole pages against a dictionary of counts; refused calls change nothing."""
    rng = random.Random(5)
    c = cache(pages=40, size=4)
    held = [0] * 40
    for step in range(3000):
        what = rng.choice(["take", "share", "release", "release", "fork", "bad"])
        mine = [p for p in range(40) if held[p]]
        if what == "take":
            n = rng.randint(0, 12)
            if n > held.count(0):
                refused(CAPACITY, c.take, n)
            else:
                got = c.take(n)
                assert len(set(got)) == n and all(held[p] == 0 for p in got)
                for p in got:
                    held[p] = 1
        elif what == "share" and mine:
            some = [rng.choice(mine) for _ in range(rng.randint(1, 4))]
            c.share(some)
            for p in some:
                held[p] += 1
        elif what == "release" and mine:
            some = [rng.choice(mine) for _ in range(rng.randint(1, 6))]
            if all(some.count(p) <= held[p] for p in some):
                c.release(some)
                for p in some:
                    held[p] -= 1
            else:
                refused(STATE, c.release, some)
        elif what == "fork" and mine:
            some = rng.sample(mine, rng.randint(1, min(3, len(mine))))
            for f in c.fork(some, 4 * len(some), 2):
                assert f == some
                for p in some:
                    held[p] += 1
        else:
            free = [p for p in range(40) if not held[p]]
            if free:
                refused(STATE, c.share, mine[:1] + free[:1])
                refused(STATE, c.release, mine[:1] + free[:1])
                refused(STATE, c.fork, free[:1], 4)
            refused(INVALID, c.release, mine[:1] + [40])
            refused(INVALID, c.share, mine[:1] + [-1])
        assert c.free_pages == held.count(0)
    for p in range(40):
        c.release([p] * held[p])
    assert c.free_pages == 40 and sorted(c.take(40)) == list(range(40))


def test_forks_that_are_refused():
    c = cache(pages=8, size=4)
    p = c.take(3)
    assert c.fork(p, 0, 2) == [[], []] and c.fork(p, 8, 0) == []
    refused(INVALID, c.fork, p, 13)                        # more tokens than pages
    refused(INVALID, c.fork, p, -1)
    refused(INVALID, c.fork, p, 8, -1)
    refused(INVALID, c.fork, [0, 99], 8)
    refused(STATE, c.fork, p, 9)                           # a part of a page has to be copied, and nothing runs here
    assert c.free_pages == 5
    assert c.fork(p, 12, 1) == [p] and c.free_pages == 5   # whole pages are only shared


def test_copies_that_are_refused():
    c = cache(pages=8, size=4)
    for src, dst, rows in (([0], [8], None), ([-1], [1], None), ([0], [1], [5]), ([0], [1], [-1]), ([0, 2], [1, 1], None), ([0, 1], [1, 2], None),
                           ([3], [3], None), ([0], [2 ** 31 - 1], None)):
        refused(INVALID, c.copy, src, dst, rows)
    refused(INVALID, c.copy, [0], [1, 2])
    refused(INVALID, c.copy, [0], [1], [1, 2])
    p = c.take(2)
    c.share(p[:1])
    assert "shared" in refused(STATE, c.copy, [p[1]], [p[0]])
    refused(STATE, c.copy, [p[0]], [p[1]])                 # allowed, but host only
    refused(INVALID, c.copy, [0, 1], [2, 2])               # the marks of refused calls are gone
    refused(STATE, c.copy, [4], [5])


# ---- arguments of the calls that run ----------------------------------------------------------------------------------

def test_append_arguments():
    c = cache(heads=2, hq=4)
    t = lambda *s: torch.zeros(s)
    i = lambda n: torch.zeros(n, dtype=torch.int32)
    k, q = t(3, 2, 64), t(3, 4, 64)
    bad = [dict(k=None), dict(v=None), dict(slots=None), dict(k=t(3, 3, 64), v=t(3, 3, 64)), dict(v=t(2, 2, 64)), dict(k=t(3, 2, 32), v=t(3, 2, 32)), dict(q=q),
           dict(q_out=q), dict(q=t(3, 2, 64), q_out=t(3, 2, 64)), dict(q=q, q_out=t(2, 4, 64)), dict(k=k.bfloat16(), v=k.bfloat16()),
           dict(slots=torch.zeros(3, dtype=torch.int64)), dict(slots=i(2)), dict(positions=i(4)), dict(positions=None), dict(k=t(3, 2, 128)[..., ::2]),
           dict(k=t(3, 2, 65)[..., 1:]), dict(k=t(3, 2, 66)[..., :64]), dict(k_weight=t(32)), dict(q_weight=t(64)), dict(k_weight=t(64), eps=-1.0),
           dict(k_weight=t(64), eps=math.nan), dict(q=q, q_out=t(3, 4, 64)[:1].expand(3, 4, 64)), dict(k_out=t(3, 1, 64).expand(3, 2, 64)),
           dict(k_out=t(4, 64).as_strided((3, 2, 64), (64, 64, 1))), dict(k_out=t(8, 64).as_strided((3, 2, 64), (128, 192, 1))),
           dict(q=q, q_out=q.as_strided((3, 4, 64), (64, 192, 1))), dict(slots=i(6)[::2])]
    for kw in bad:
        a = dict(k=k, v=t(3, 2, 64), positions=i(3), slots=i(3), rope=kvp.Rope(64))
        a.update(kw)
        refused(INVALID, c.append, 0, **a)
    refused(INVALID, c.append, 0, k, k, i(3), i(3), rope=kvp.Rope(128))
    refused(STATE, c.append, 0, k, k, i(3), i(3), rope=kvp.Rope(64))
    refused(STATE, c.append, 9, k, k, None, i(3))
    refused(INVALID, kvp.norm_rope, q, k, i(3), None, q, k)           # CPU tensors


def test_norm_rope_arguments():
    """Refused before anything is launched: addresses here are numbers, nothing reads them."""
    L = kvp.lib()

    def call(dtype=0, d=64, rope=None, device=0, **kw):
        a = kvp.kvp_tokens()
        a.struct_bytes, a.n_tokens, a.n_q_heads, a.n_kv_heads = ctypes.sizeof(a), 2, 4, 2
        a.q = a.q_out = 1 << 20
        a.k = a.k_out = 1 << 24
        a.positions = 1 << 28
        for s in (a.q_stride, a.q_out_stride):
            s[0], s[1] = 256, 64
        for s in (a.k_stride, a.k_out_stride):
            s[0], s[1] = 128, 64
        for k, v in kw.items():
            if isinstance(v, tuple):
                getattr(a, k)[0], getattr(a, k)[1] = v
            else:
                setattr(a, k, v)
        return L.kvp_norm_rope(device, dtype, d, ctypes.byref(a), None if rope is None else rope.address, None)

    r = kvp.Rope(64)
    for kw in (dict(d=80), dict(dtype=2), dict(device=-1), dict(struct_bytes=4), dict(n_tokens=-1), dict(n_q_heads=0), dict(n_kv_heads=-2), dict(q_out=None),
               dict(k_out=None), dict(q=None), dict(v=64), dict(slots=64), dict(q=8 + (1 << 20), q_out=8 + (1 << 20)), dict(q_stride=(255, 64)),
               dict(q_stride=(256, 32)), dict(k_out_stride=(128, 16)), dict(q_weight=24), dict(positions=None, rope=r), dict(positions=2, rope=r),
               dict(k_weight=1 << 16, eps=-1.0), dict(k=None, k_out=None, k_weight=1 << 16), dict(n_q_heads=70000)):
        assert call(**kw) == INVALID, kw
        assert L.kvp_cache_last_error(None)
    assert call(n_tokens=0) == 0 and call(q=None, q_out=None, k=None, k_out=None) == 0       # nothing to do, nothing touched


def test_rope_arguments():
    for kw in (dict(rotary_dim=24), dict(rotary_dim=-16), dict(pairing=2), dict(theta=0.0), dict(theta=math.inf), dict(scale=0.5), dict(scale=0.0),
               dict(scale=math.nan), dict(magnitude=0.0), dict(magnitude=math.inf), dict(original_positions=-1.0),
               dict(original_positions=8192, low_rotations=4.0, high_rotations=4.0), dict(inv_freq=[math.nan] * 32), dict(inv_freq=[1.0] * 31)):
        refused(INVALID, kvp.Rope, 64, **kw)
    k = torch.zeros(3, 2, 64)
    i = torch.zeros(3, dtype=torch.int32)
    refused(INVALID, cache().append, 0, k, k, i, i, rope=kvp.Rope(64, rotary_dim=80))       # more than a head has
    r = kvp.Rope(64)
    r.struct.struct_bytes = 8
    refused(INVALID, cache().append, 0, k, k, i, i, rope=r)
    r = kvp.Rope(64)
    r.struct.reserved = 1
    refused(INVALID, cache().append, 0, k, k, i, i, rope=r)


@pytest.mark.parametrize("r,theta,scale,original,low,high", [(128, 500000.0, 8.0, 8192, 1.0, 4.0), (64, 10000.0, 4.0, 32768, 1.0, 32.0),
                                                              (48, 1e6, 2.0, 0, 1.0, 4.0), (16, 10000.0, 1.0, 0, 1.0, 4.0), (0, 1e4, 1.0, 0, 1.0, 4.0)])
def test_frequencies(r, theta, scale, original, low, high):
    got = kvp.Rope(128, rotary_dim=r, theta=theta, scale=scale, original_positions=original, low_rotations=low, high_rotations=high).frequencies()
    want = ref.frequencies(r, theta, scale, original, low, high)
    assert len(got) == r // 2 and all(abs(a - b) <= 1e-14 * b for a, b in zip(got, want))
    if original:
        assert got[0] == 1.0 and abs(got[-1] * scale * theta ** ((r - 2) / r) - 1) < 1e-12   # the fastest as they were, the slowest scaled


def test_frequencies_reach_a_context():
    """What a context re-bases packets with is what the rotation of new tokens uses."""
    f = kvp.Rope(64, theta=500000.0, scale=8.0, original_positions=8192).frequencies()
    ctx = kvp.Context(1, 4, 2, 64, "f32", inv_freq=f, device=-1)
    ctx.close()
    g = kvp.Rope(64, inv_freq=f).frequencies()
    assert f == g


def test_attend_arguments():
    c = cache(heads=2, hq=4, max_batch=3)
    t = lambda *s: torch.zeros(s)
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    good = dict(q=t(2, 4, 64), table=i(2, 3), lens=i(2), out=t(2, 4, 64))
    for kw in (dict(q=t(2, 2, 64)), dict(q=t(2, 4, 32)), dict(q=t(2, 4, 64).bfloat16()), dict(out=t(1, 4, 64)), dict(out=t(2, 4, 64).double()),
               dict(table=i(3, 3)), dict(table=i(2, 3).long()), dict(table=i(2, 6)[:, ::2]), dict(lens=i(3)), dict(lens=t(2)), dict(first=i(1)),
               dict(lse=t(2, 3)), dict(lse=t(4, 2).T), dict(lse=t(2, 4).double()), dict(q=t(2, 4, 65)[..., 1:]), dict(q=t(2, 4, 66)[..., :64]),
               dict(out=t(1, 4, 64).expand(2, 4, 64)), dict(out=t(2, 1, 64).expand(2, 4, 64)), dict(lens=i(4)[::2]),
               dict(out=t(6, 64).as_strided((2, 4, 64), (128, 64, 1)))):
        refused(INVALID, c.attend, 0, **dict(good, **kw))
    refused(STATE, c.attend, 0, **good)
    refused(STATE, c.attend, 0, **dict(good, out=t(8, 64).as_strided((2, 4, 64), (64, 128, 1))))          # heads outermost: rows lie apart
    # tables that could hold more tiles than are counted; nothing reads the addresses
    wide = cache(heads=8, hq=8, max_batch=3)
    strides = (ctypes.c_int64 * 2)(512, 64)
    call = lambda cols: kvp.lib().kvp_cache_attend(wide._h, 0, 3, 1 << 20, strides, 1 << 20, cols, cols, 1 << 20, None, 1 << 20, strides, None, None)
    assert call(2 ** 29) == CAPACITY and call(2 ** 20) == STATE
    refused(CAPACITY, c.attend, 0, t(4, 4, 64), i(4, 3), i(4), t(4, 4, 64))


def test_compact_arguments():
    c = cache(layers=2, heads=2)
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    good = dict(table=i(2, 3), lens=i(2), new_table=i(2, 2), kept=i(2, 2, 2, 5), n_kept=i(2))
    for kw in (dict(table=i(1, 3)), dict(lens=i(1)), dict(new_table=i(3, 2)), dict(kept=i(2, 3, 2, 5)), dict(kept=i(2, 2, 3, 5)), dict(kept=i(2, 5)),
               dict(kept=i(1, 2, 2, 5)), dict(n_kept=i(3)), dict(kept=i(2, 2, 2, 10)[..., ::2]), dict(kept=i(2, 2, 2, 5).long())):
        refused(INVALID, c.compact, **dict(good, **kw))
    refused(STATE, c.compact, **good)


def test_tensors_that_fit_go_straight_to_the_library():
    """The module that marshals calls hands on what fits (the library then says that nothing runs here) and gives back what does
    not; a closed cache says so."""
    c, m = cache(heads=2, hq=4), kvp.calls()
    t, i = (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.int32))
    k, q = t(3, 2, 64), t(3, 4, 64)
    append = lambda *a: m.append(c._h.value, 0, kvp.DTYPE_F32, -1, 64, *a, 1e-6, None)
    assert append(k, k, None, i(3), None, None, None, None, None, None) == STATE
    assert append(k, k, i(3), i(3), kvp.Rope(64).address, q, q, k, t(64), t(64)) == STATE
    for a in ((k, t(2, 2, 64), None, i(3), None, None, None, None, None, None), (k, k, None, i(3).long(), None, None, None, None, None, None),
              (k, k, None, i(3), None, q, t(3, 2, 64), None, None, None), (k, 7, None, i(3), None, None, None, None, None, None),
              (k, k, None, i(3), None, None, None, None, None, t(32)), (k.to("meta"), k, None, i(3), None, None, None, None, None, None),
              (torch.zeros(3, 2, 64).to_sparse(), k, None, i(3), None, None, None, None, None, None)):
        assert append(*a) == -1
    attend = lambda *a: m.attend(c._h.value, 0, kvp.DTYPE_F32, -1, 64, 4, *a, None)
    assert attend(q, q, i(3, 5), i(3), i(3), t(3, 4)) == STATE
    for a in ((q, q, i(2, 5), i(3), None, None), (q, q, i(3, 5), i(3), None, t(4, 3).T), (q, q.double(), i(3, 5), i(3), None, None), (None, q, i(3, 5), i(3), None, None)):
        assert attend(*a) == -1
    assert m.compact(c._h.value, -1, 2, 2, i(2, 3), i(2), i(2, 2), i(2, 2, 1, 5), i(2), None) == STATE
    assert m.compact(c._h.value, -1, 2, 2, i(2, 3), i(2), i(2, 2), i(2, 3, 1, 5), i(2), None) == -1
    assert m.norm_rope(-1, q, None, i(3), None, q, None, None, None, 1e-6, None) == -1
    with pytest.raises(TypeError):
        m.append(1, 2)
    c.close()
    refused(STATE, c.append, 0, k, k, i(3), i(3))
    refused(STATE, c.attend, 0, q, i(3, 5), i(3), q)
    c.close()
