"""The paged cache's calls at the ends of their ranges, and what surrounds them, without a GPU."""
import ctypes
import gc
import os
import subprocess
import sys
import sysconfig
import weakref

import pytest
import torch

from paper_2604_13226_b200 import binding as kvp
from paper_2604_13226_b200 import build
import test_paged_cpu
from test_paged_cpu import INVALID, STATE, cache, refused


def test_tiles_of_the_longest_lists(tmp_path):
    """Rows are cut into tiles without the count passing 31 bits, whatever the length."""
    src = tmp_path / "tiles.cpp"
    src.write_text(f'#include "{build.CSRC}/kvp_paged.h"\nextern "C" int32_t tiles(int32_t rows, int32_t keys) {{ return kvp_tiles(rows, keys); }}\n')
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-fPIC", "-shared", "-fwrapv", f"-I{cuda}/include", str(src), "-o", str(tmp_path / "tiles.so")])
    tiles = ctypes.CDLL(str(tmp_path / "tiles.so")).tiles
    for keys in (8, 16, 32):
        for rows in [*range(100), *range(2 ** 30 - 40, 2 ** 30 + 40), *range(2 ** 31 - 100, 2 ** 31)]:
            assert tiles(rows, keys) == -(-rows // keys), (rows, keys)


def test_compaction_of_tables_without_columns():
    """Requests that keep nothing have no new pages, and those without rows no old ones: tables of [n][0] have no address."""
    c = cache(layers=2, heads=2)
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    good = dict(table=i(2, 3), lens=i(2), new_table=i(2, 2), kept=i(2, 1, 1, 5), n_kept=i(2))
    for kw in (dict(new_table=i(2, 0)), dict(table=i(2, 0)), dict(table=i(2, 0), new_table=i(2, 0))):
        refused(STATE, c.compact, **dict(good, **kw))              # it would run where something runs
    one, zero = (ctypes.c_int32 * 8)(), (ctypes.c_int64 * 3)()
    call = lambda table, cols, new, new_cols: kvp.lib().kvp_cache_compact(c._h, 2, table, 4, cols, one, new, 4, new_cols, one, zero, 1, one, None)
    assert call(None, 0, None, 0) == STATE and call(None, 1, one, 1) == INVALID and call(one, 1, None, 1) == INVALID


def test_outputs_are_separated_from_what_they_were_cloned_from():
    """A lazily cloned output has its original's memory until something asks to write to it: taking its address does."""
    lazy = getattr(torch, "_lazy_clone", None)
    if lazy is None:
        pytest.skip("this PyTorch has no lazy clones")
    c, rope = cache(heads=2, hq=4), kvp.Rope(64)
    t, i = (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.int32))
    k, q = t(3, 2, 64), t(3, 4, 64)
    outs = [lazy(q), lazy(k), lazy(q), lazy(t(3, 4))]
    assert all(torch._C._is_cow_tensor(o) for o in outs)
    refused(STATE, c.append, 0, k, k, i(3), i(3), rope=rope, q=q, q_out=outs[0], k_out=outs[1])
    refused(STATE, c.attend, 0, q, i(3, 2), i(3), outs[2], lse=outs[3])
    assert not any(torch._C._is_cow_tensor(o) for o in outs)
    inputs = [lazy(k), lazy(k), lazy(q)]                           # what is only read stays shared
    refused(STATE, c.append, 0, inputs[0], inputs[1], i(3), i(3), rope=rope, q=inputs[2], q_out=q)
    assert all(torch._C._is_cow_tensor(x) for x in inputs)


class _Recording:
    """Stands in for the device of a host-only cache: whether something is recorded, and who waited for it."""

    def __init__(self, monkeypatch):
        self.recording, self.fails, self.waits = False, False, 0
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.recording)
        monkeypatch.setattr(torch.cuda, "synchronize", self.wait)

    def wait(self, device):
        assert device == self.device and not self.recording
        if self.fails:
            raise RuntimeError("another thread records")
        self.waits += 1

    device = 99

    def cache(self):
        c = cache()
        c.device, c.workspace = self.device, torch.zeros(8)
        c.workspace.gone = weakref.ref(c.workspace)
        return c, c.workspace.gone


def test_a_workspace_outlives_calls_that_nobody_waited_for(monkeypatch):
    """A cache that is closed, or dropped, while something is recorded cannot wait for its attend calls on other streams: its
    workspace stays until somebody has waited for the device."""
    dev = _Recording(monkeypatch)
    closed, a = dev.cache()
    dropped, b = dev.cache()
    late, _ = dev.cache()
    dev.recording = True
    closed.close()
    del closed, dropped
    gc.collect()
    assert a() is not None and b() is not None and dev.waits == 0
    dev.recording = False
    late.close()
    gc.collect()
    assert dev.waits == 1 and a() is None and b() is None


def test_a_wait_that_fails_ends_the_cache_but_not_its_workspace(monkeypatch):
    dev = _Recording(monkeypatch)
    c, a = dev.cache()
    dev.fails = True
    with pytest.raises(RuntimeError):
        c.close()
    assert not c._h
    c.close()                                              # there is nothing more to close
    del c
    gc.collect()
    assert a() is not None
    dev.fails = False
    other, _ = dev.cache()
    other.close()
    gc.collect()
    assert a() is None


@pytest.mark.parametrize("module", [True, False])
def test_numbers_beyond_32_bits_are_not_cut_to_them(monkeypatch, module):
    """2^32 + 1 is not 1: layers, pages, rows, counts and sizes."""
    if not module:
        monkeypatch.setattr(kvp, "_calls", kvp._NoModule)
    far = (2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 31)
    c = cache(layers=2, heads=2, hq=4, pages=8, size=4)
    t, i = (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.int32))
    k, q, p = t(3, 2, 64), t(3, 4, 64), c.take(2)
    for x in far:
        refused(INVALID, c.append, x, k, k, None, i(3))
        refused(INVALID, c.attend, x, q, i(3, 2), i(3), q)
        refused(INVALID, c.copy, [x], [3])
        refused(INVALID, c.copy, [3], [x])
        refused(INVALID, c.copy, [3], [4], [x])
        refused(INVALID, c.share, [x + p[0]])
        refused(INVALID, c.release, [x + p[0]])
        refused(INVALID, c.fork, [x + p[0]], 4)
        refused(INVALID, c.fork, p, 4, x)
        refused(INVALID, c.take, x)
        refused(INVALID, cache, hq=4 + x)
        refused(INVALID, cache, max_batch=4 + x)
        refused(INVALID, kvp.Rope, 64, rotary_dim=x + 64)
        refused(INVALID, kvp.Rope, 64, pairing=x)
    refused(INVALID, c.fork, p, 2 ** 32)
    assert c.free_pages == 6
    refused(STATE, c.append, 1, k, k, None, i(3))


# ---- what is built ------------------------------------------------------------------------------------------------------

@pytest.fixture
def compilers(monkeypatch, tmp_path):
    """Compilers that note how they were called and leave an empty file."""
    seen = []

    def run(cmd, **kw):
        seen.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(build.subprocess, "check_call", run)
    monkeypatch.setattr(build, "_HERE", str(tmp_path))
    monkeypatch.setattr(build, "CSRC", str(tmp_path / "csrc"))
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "libkvp.so"))
    (tmp_path / "csrc").mkdir()
    (tmp_path.parent / "include").mkdir(exist_ok=True)
    for f in (tmp_path / "csrc" / "kvp_calls.cpp", tmp_path.parent / "include" / "kvp.h"):
        f.write_text("")
        os.utime(f, (1, 1))
    return seen


def test_the_library_builds_without_pytorch(compilers, monkeypatch):
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build(force=True) == build.LIB_PATH and os.path.exists(build.LIB_PATH)
    assert not any("kvp_calls" in str(x) for cmd in compilers for x in cmd)


def test_another_pytorch_gets_a_module_of_its_own(compilers, monkeypatch):
    first = build.build_calls()
    assert os.path.exists(first) and len(compilers) == 1 and build.build_calls() == first and len(compilers) == 1
    monkeypatch.setattr(torch, "__version__", "9.9.9+test")
    second = build.build_calls()
    assert second != first and os.path.exists(second) and len(compilers) == 2
    assert sysconfig.get_config_var("EXT_SUFFIX") in first          # and another Python
    os.utime(os.path.join(build.CSRC, "kvp_calls.cpp"))
    os.utime(second, (2, 2))
    assert build.build_calls() == second and len(compilers) == 3    # newer sources


def _no_compiler(force=False):
    raise subprocess.CalledProcessError(1, ["g++"])


def _cut_short(force=False):
    path = build.calls_path()
    open(path, "wb").write(b"\x7fELF")
    return path


@pytest.mark.parametrize("why", [_no_compiler, _cut_short])
def test_python_marshals_where_the_module_is_not(monkeypatch, tmp_path, why):
    """What the module refuses, and what it hands on, does not depend on its being there."""
    monkeypatch.setattr(kvp, "_calls", None)
    monkeypatch.setattr(build, "calls_path", lambda: str(tmp_path / "none.so"))
    monkeypatch.setattr(build, "build_calls", why)
    with pytest.warns(RuntimeWarning, match="marshalled in Python"):
        cache().close()
    assert kvp.calls() is kvp._NoModule
    for test in (test_paged_cpu.test_append_arguments, test_paged_cpu.test_attend_arguments, test_paged_cpu.test_compact_arguments,
                 test_paged_cpu.test_rope_arguments, test_compaction_of_tables_without_columns):
        test()
    c = cache()
    c.close()
    i = torch.zeros(3, dtype=torch.int32)
    refused(STATE, c.append, 0, torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), i, i)
