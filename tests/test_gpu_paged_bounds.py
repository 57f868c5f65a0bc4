"""The paged cache's calls at the ends of their ranges on the GPU."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2604_13226_b200 import binding as kvp
from test_gpu_paged import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64), (torch.float32, 128)])
@pytest.mark.parametrize("hq", [1, 20])
@pytest.mark.parametrize("short", [1, 31, 33])
def test_the_longest_lengths(dtype, d, hq, short):
    """Lengths within a tile of 2^31 over lists of absent pages: only the first and the last one are there."""
    page, cols = 64, 1 << 25
    k, v = ref.pages((1, 3, 1, page, d), "heads", dtype, seed=d + hq)
    c = kvp.PagedCache(k, v, hq, max_batch=2)
    g = torch.Generator(device="cuda").manual_seed(hq)
    q = torch.randn(2, hq, d, generator=g, device="cuda").to(dtype)
    table = torch.full((2, cols), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, -1], table[1, 0] = 2, 0, 1
    out, lse = torch.full_like(q, 7.0), torch.full((2, hq), 7.0, device="cuda")
    lens = [2 ** 31 - short, 5]
    c.attend(0, q, table, ints(lens), out, lse=lse, first=ints([10, 0]))
    want = ref.attend(k, v, "heads", 0, q, ints([[2, 0], [1, -1]]), [2 * page - short, 5], [10, 0], page, d ** -0.5)
    ref.check(out, want[0], want[2], "out")
    ref.check(lse, want[1], want[3], "lse")
    if short == 1:                                                 # a list that ends later than lengths can say
        wide = torch.full((1, cols + 9), -1, dtype=torch.int32, device="cuda")
        wide[0, :cols] = table[0]
        again = torch.full_like(out[:1], 7.0)
        c.attend(0, q[:1], wide, ints(lens[:1]), again, first=ints([10]))
        ref.check(again, want[0][:1], want[2][:1], "out")
        nothing = torch.full_like(out[:1], 7.0)
        c.attend(0, q[:1], torch.full_like(wide, 3), ints(lens[:1]), nothing, lse=lse[:1])
        assert not nothing.any() and bool((lse[0] == -math.inf).all())


def test_compact_with_counts_below_zero():
    """A count below zero, the lowest number too, keeps nothing: not a row of the later blocks either."""
    k, v = ref.pages((2, 40, 2, 16, 64), "heads", torch.bfloat16, seed=1)
    was = k.clone(), v.clone()
    c = kvp.PagedCache(k, v, 4)
    counts = [-2 ** 31, -2 ** 31 + 31, -1, 0, 35]
    table = torch.arange(20, dtype=torch.int32, device="cuda").view(5, 4)
    kept = torch.arange(60, dtype=torch.int32, device="cuda").add(2).expand(5, 1, 1, 60).contiguous()
    c.compact(table, ints([64] * 5), table + 20, kept, ints(counts))
    torch.cuda.synchronize()
    for t, w in ((k, was[0]), (v, was[1])):
        for i in range(35):
            w[:, 36 + i // 16, :, i % 16] = w[:, 16 + (i + 2) // 16, :, (i + 2) % 16]
        assert torch.equal(t, w)


def test_compaction_of_tables_without_columns():
    """Nothing is kept, or nothing is there to be kept: rows stay as they are."""
    k, v = ref.pages((2, 12, 2, 16, 64), "heads", torch.bfloat16, seed=2)
    was = k.clone(), v.clone()
    c = kvp.PagedCache(k, v, 4)
    i = lambda *n: torch.empty(n, dtype=torch.int32, device="cuda")
    table, kept = ints([[0, 1], [2, 3]]), torch.arange(20, dtype=torch.int32, device="cuda").expand(2, 1, 1, 20)
    c.compact(table, ints([30, 30]), i(2, 0), kept, ints([0, 0]))
    c.compact(table, ints([30, 30]), i(2, 0), kept, ints([20, 3]))
    c.compact(i(2, 0), ints([30, 30]), table + 4, kept, ints([20, 3]))
    c.compact(i(2, 0), ints([30, 0]), i(2, 0), kept, ints([20, 3]))
    torch.cuda.synchronize()
    assert torch.equal(k, was[0]) and torch.equal(v, was[1])


def test_a_workspace_is_not_handed_out_while_calls_use_it():
    """A cache with a call under way on another stream goes while a graph is recorded: its workspace is not handed out again until
    a later close has waited for the device."""
    k, v = ref.pages((1, 300, 2, 16, 128), "heads", torch.bfloat16, seed=3)
    c, other = kvp.PagedCache(k, v, 8), kvp.PagedCache(k, v, 8)
    q = torch.randn(1, 8, 128, device="cuda").bfloat16()
    out, want, n = torch.empty_like(q), torch.empty_like(q), ints([4800])
    table = torch.arange(300, dtype=torch.int32, device="cuda")[None]
    other.attend(0, q, table, n, want)
    torch.cuda.synchronize()
    side, g, size = torch.cuda.Stream(), torch.cuda.CUDAGraph(), c.workspace.numel()
    at = c.workspace.data_ptr()
    x = torch.zeros(1, device="cuda")
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    c.attend(0, q, table, n, out, stream=side)
    with torch.cuda.graph(g):
        x += 1
        c.close()
        del c
    blocks = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
    assert all(b.data_ptr() != at for b in blocks)
    other.close()
    assert side.query() and torch.equal(out, want)
    assert not any(w.data_ptr() == at for _, w in kvp._unwaited.values())


def test_python_marshals_the_same_calls(monkeypatch):
    """The bits of every call do not depend on who marshals it."""
    def run():
        k, v = ref.pages((2, 40, 2, 16, 64), "heads", torch.bfloat16, seed=4)
        c = kvp.PagedCache(k, v, 8, max_batch=2)
        g = torch.Generator(device="cuda").manual_seed(4)
        x = torch.randn(5, 12, 64, generator=g, device="cuda").bfloat16()
        q, kn, vn = x[:, :8], x[:, 8:10], x[:, 10:]
        w, rope, pos = (1 + torch.rand(64, generator=g, device="cuda")).bfloat16(), kvp.Rope(64, rotary_dim=48, theta=1e6), ints([9, 1 << 30, 0, 7, 300])
        q1, k1, q2, out = (torch.empty(5, h, 64, device="cuda", dtype=torch.bfloat16) for h in (8, 2, 8, 8))
        lse, table = torch.empty(2, 8, device="cuda"), torch.arange(16, dtype=torch.int32, device="cuda").view(2, 8)
        c.append(1, kn, vn, pos, ints([3, 40, 41, 42, 99]), rope=rope, q=q, q_out=q1, k_out=k1, q_weight=w, k_weight=w)
        c.append(0, kn, vn, None, ints([3, 40, 41, 42, 99]))
        kvp.norm_rope(q, None, pos, rope, q2, q_weight=w)
        c.attend(1, q1[:2], table, ints([128, 77]), out[:2], lse=lse, first=ints([0, 40]))
        c.attend(0, q1[2:4], table, ints([128, 77]), out[2:4])
        c.compact(table, ints([128, 77]), table + 16, torch.arange(1, 31, dtype=torch.int32, device="cuda").expand(2, 1, 2, 30).contiguous(), ints([30, 4]))
        return k, v, q1, k1, q2, out[:4], lse

    want = run()
    assert hasattr(kvp.calls(), "bind")
    monkeypatch.setattr(kvp, "_calls", kvp._NoModule)
    for a, b in zip(run(), want):
        assert torch.equal(a, b)
