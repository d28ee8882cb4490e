"""Sequence tables when the host has no memory left: each call either does what
it says or changes nothing and returns an error; no C++ exception leaves a C
entry.  A preloaded operator new fails from its n-th call on."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include <cstdlib>
#include <new>
static long left = -1;
extern "C" void new_fails_after(long n) { left = n; }
void *operator new(std::size_t n)
{
    if (left == 0) throw std::bad_alloc();
    if (left > 0) --left;
    if (void *p = std::malloc(n ? n : 1)) return p;
    throw std::bad_alloc();
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
"""

SCRIPT = r"""
import ctypes, sys
import numpy as np
from paper_2606_12950_gb300 import kvpool as K

shim = ctypes.CDLL(sys.argv[1])
shim.new_fails_after.argtypes = [ctypes.c_long]
L = K.lib()
LAYOUTS = [(2, 64), (4, 64)]


def setup():
    h = K.kv_pool_create(1 << 40, 256 * 2 * 2 * 16 * 64 * 2, 16, LAYOUTS, (1 << 40) + (1 << 30))
    t = K.SeqTab(h, 0, 4, 100)
    t.reserve(0, 1500)
    t.set_len(0, 1400)
    t.evict(0, 300, 40)   # a hole in its row
    t.reserve(1, 640)
    t.set_len(1, 320)
    return h, t


def state(h, t):
    tab, lens = t.host()
    c = t.counters()
    return tab.copy().tolist(), lens.copy().tolist(), c["blocks_held"], c["releases"], K.kv_pool_stats(h)


dst, status = np.array([2, 3], np.int32), np.zeros(1, np.int32)
one, tokens, lens1 = np.array([1], np.int32), np.array([100], np.int64), np.array([50], np.int32)
n32 = ctypes.c_int32(0)
OPS = {
    "release with a hole": lambda h, t: L.kv_seq_release(t.handle, 0),
    "release": lambda h, t: L.kv_seq_release(t.handle, 1),
    "trim": lambda h, t: L.kv_seq_trim(t.handle, 1),
    "evict": lambda h, t: L.kv_seq_evict(t.handle, 0, 100, 0, ctypes.byref(n32)),
    "reserve": lambda h, t: L.kv_seq_reserve(t.handle, 2, 800),
    "advance": lambda h, t: L.kv_seq_advance(t.handle, 0, None, ctypes.byref(n32)),
    "fork": lambda h, t: L.kv_seq_fork(t.handle, 1, 2, dst.ctypes.data, None),
    "share": lambda h, t: L.kv_seq_share_prefix(t.handle, 2, 1, 20),
    "replace": lambda h, t: L.kv_seq_replace(t.handle, 1, one.ctypes.data, tokens.ctypes.data, lens1.ctypes.data,
                                             status.ctypes.data),
}
for name, op in OPS.items():
    failed = 0
    for n in range(12):
        h, t = setup()
        before = state(h, t)
        shim.new_fails_after(n)
        rc = op(h, t)
        shim.new_fails_after(-1)
        assert rc in (K.KV_OK, K.KV_ERR_OUT_OF_BLOCKS), (name, n, rc)
        if rc:
            failed += 1
            assert state(h, t) == before, (name, n)
            assert op(h, t) == K.KV_OK, (name, n)
        shim.new_fails_after(0)
        rc = L.kv_seqtab_destroy(t.handle)
        shim.new_fails_after(-1)
        t.handle = None
        assert rc == K.KV_OK and K.kv_pool_stats(h)["blocks_used"][0] == 0, (name, n, rc)
        K.kv_pool_destroy(h)
    print(name, failed)
h = K.kv_pool_create(1 << 40, 256 * 8192, 16, LAYOUTS, (1 << 40) + (1 << 30))
out = ctypes.c_void_p()
for n in range(12):
    shim.new_fails_after(n)
    rc = L.kv_seqtab_create(h, 0, 4, 100, ctypes.byref(out))
    shim.new_fails_after(-1)
    assert rc in (K.KV_OK, K.KV_ERR_OUT_OF_BLOCKS), (n, rc)
    if rc == K.KV_OK:
        L.kv_seqtab_destroy(out)
print("done")
"""


def test_no_host_memory(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, shim = tmp_path / "shim.cpp", tmp_path / "shim.so"
    src.write_text(SHIM)
    subprocess.run([gxx, "-O1", "-shared", "-fPIC", "-o", str(shim), str(src)], check=True)
    env = {**os.environ, "LD_PRELOAD": str(shim), "PYTHONPATH": ROOT}
    r = subprocess.run([sys.executable, "-c", SCRIPT, str(shim)], cwd=ROOT, env=env, capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout[-800:], r.stderr[-2000:])
    assert r.stdout.split()[-1] == "done"
