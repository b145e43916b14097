"""Calls through the C ABI while the host has no memory left: they come back with a status, and throw nothing through a C entry.  In a process of
its own, with an operator new that fails on request in the thread that asks."""
import os
import subprocess
import sys

import pytest

from paper_2410_15352_b200.build import build_library

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

ALLOCATOR = r"""
#include <cstdlib>
#include <new>
static thread_local bool failing = false;
static thread_local int refused = 0;
extern "C" void set_failing(int f) { failing = f != 0; }
extern "C" int count_refused() { return refused; }
void* operator new(std::size_t n) {
  if (failing) { ++refused; throw std::bad_alloc(); }
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
"""

PROGRAM = r"""
import ctypes as C, sys, torch
from paper_2410_15352_b200 import binding as cb, block
alloc = C.CDLL(sys.argv[1])
L = block.lib()
dev = lambda t: C.c_void_p(t.data_ptr())
t, n, m = 200, 256, 128
x, w, dy = torch.randn(t, n, device="cuda").bfloat16(), torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.randn(t, n, device="cuda").bfloat16()
W = torch.randn(m, n, device="cuda").bfloat16()
a8, b8, bt8 = block.new_fp8(t, n), block.new_fp8(m, n), block.new_fp8(n, m)
rstd, dx, dw, c = torch.empty(t, device="cuda"), torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(t, m, dtype=torch.bfloat16, device="cuda")
need = L.compact_rms_norm_bwd_workspace_bytes(cb.BF16, t, n)
ws = torch.empty(need, dtype=torch.uint8, device="cuda")
product, rotary = block.Fp8Product(), block.Rotary(64)
cfg = block.RotaryConfig(64, 64, 0, 0, 1e4, 1.0, 1.0, 4.0, 8192.0, 1.0)
out = C.c_void_p()
s = None
def later(f, *args):      # torch's own calls, which allocate, are made before
    return lambda: f(*args)
run = later(L.compact_fp8_product_run, product._h, t, m, n, 0, dev(a8.data), a8.data.stride(0), dev(a8.scales), t, 0, dev(b8.data), b8.data.stride(0),
                                        dev(b8.scales), m, cb.BF16, dev(c), m, s)
calls = [
    ("quantize_rows", later(L.compact_quantize_rows, cb.BF16, t, n, dev(x), n, 0, dev(a8.data), a8.data.stride(0), dev(a8.scales), t, s)),
    ("quantize_blocks", later(L.compact_quantize_blocks, cb.BF16, m, n, dev(W), n, 0, dev(b8.data), b8.data.stride(0), dev(b8.scales), m, dev(bt8.data),
                                                          bt8.data.stride(0), dev(bt8.scales), n, s)),
    ("norm", later(L.compact_rms_norm_fwd, cb.BF16, t, n, 1e-6, dev(x), n, None, 0, dev(w), None, 0, dev(dx), n, dev(rstd), 0, None, 0, None, 0, s)),
    ("norm backward", later(L.compact_rms_norm_bwd, cb.BF16, t, n, dev(dy), n, dev(x), n, dev(w), dev(rstd), None, 0, dev(dx), n, dev(dw), 0, dev(ws), need, s)),
    ("rotary", later(L.compact_rotary_apply, rotary._h, cb.BF16, t, 4, 0, dev(x), n, 64, None, 0, 0, None, 64, 0, 0, dev(dx), n, 64, None, 0, 0, s)),
]
status = {}
def without_memory(call):
    alloc.set_failing(1)
    try:
        return call()
    finally:
        alloc.set_failing(0)
for name, call in calls:
    status[name] = without_memory(call)
for which in (1, 2):
    block.set_product_kernel(which)
    status["product %d" % which] = without_memory(run)
block.set_product_kernel(0)
assert all(v == cb.OK for v in status.values()), status
assert alloc.count_refused() > 0
torch.cuda.synchronize()
assert product.status() == cb.OK
got = c.clone()
assert run() == cb.OK
torch.cuda.synchronize()
assert torch.equal(got, c) and bool(c.isfinite().all())
# what needs memory says so
assert without_memory(lambda: L.compact_rotary_create(C.byref(cfg), C.byref(out))) != cb.OK and not out.value
assert without_memory(lambda: L.compact_fp8_product_create(C.byref(out))) != cb.OK and not out.value
print("came back")
"""


@pytest.mark.gpu
def test_no_exception_leaves_a_c_entry(tmp_path):
    build_library()
    lib = str(tmp_path / "libfailing.so")
    (tmp_path / "failing.cpp").write_text(ALLOCATOR)
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-fPIC", "-shared", str(tmp_path / "failing.cpp"), "-o", lib], check=True)
    env = dict(os.environ, LD_PRELOAD=lib, PYTHONPATH=ROOT)
    done = subprocess.run([sys.executable, "-c", PROGRAM, lib], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "came back" in done.stdout, done.stdout + done.stderr
