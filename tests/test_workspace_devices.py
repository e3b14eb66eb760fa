"""A workspace belongs to the device it was made on, whichever is current when it is given back: libef.so over a runtime of two devices that notes
what it is asked for (no GPU)."""
import os
import subprocess
import sys

import paper_1905_10936_amd as ef

RUNTIME = r"""
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
static int current, malloc_fails;
static char log_[4096];
static void note(const char *what) { sprintf(log_ + strlen(log_), "%s%d ", what, current); }
const char *fake_log(void) { return log_; }
void fake_begin(int device, int fails) { current = device; malloc_fails = fails; log_[0] = 0; }
int fake_current(void) { return current; }
int hipGetDevice(int *d) { *d = current; return 0; }
int hipSetDevice(int d) { current = d; return 0; }
int hipDeviceSynchronize(void) { note("wait"); return 0; }
int hipMalloc(void **p, size_t n) { note("malloc"); if (malloc_fails) return 2; *p = malloc(64); return 0; }
int hipFree(void *p) { note("free"); free(p); return 0; }
int hipGetLastError(void) { return 0; }
const char *hipGetErrorString(int e) { return "made to fail"; }
"""

DRIVER = r"""
import ctypes, sys
fake, L = ctypes.CDLL(sys.argv[1]), ctypes.CDLL(sys.argv[2])
fake.fake_log.restype = ctypes.c_char_p
w = ctypes.c_void_p()
for made, current in ((0, 0), (1, 0), (0, 1)):
    fake.fake_begin(made, 0)
    assert L.ef_workspace_create(ctypes.byref(w), ctypes.c_int64(100), None) == 0
    assert fake.fake_log().decode().split() == ["malloc%d" % made]
    fake.fake_begin(current, 0)
    assert L.ef_workspace_destroy(w) == 0
    assert fake.fake_log().decode().split() == ["wait%d" % made, "free%d" % made], fake.fake_log()
    assert fake.fake_current() == current
fake.fake_begin(0, 1)
assert L.ef_workspace_create(ctypes.byref(w), ctypes.c_int64(100), None) == -5 and not w.value
print("workspaces ok")
"""


def test_a_workspace_is_given_back_on_its_device(tmp_path):
    ef.lib()
    source, fake = tmp_path / "runtime.c", str(tmp_path / "runtime.so")
    source.write_text(RUNTIME)
    subprocess.run([os.environ.get("CC", "gcc"), "-O1", "-shared", "-fPIC", "-w", "-o", fake, str(source)], check=True)
    run = subprocess.run([sys.executable, "-c", DRIVER, fake, ef.LIB_PATH], capture_output=True, text=True, timeout=120,
                         env=dict(os.environ, LD_PRELOAD=fake))
    assert run.returncode == 0, run.stdout + run.stderr
    assert "workspaces ok" in run.stdout
