"""The launches of the gated block's products at the largest sizes, on the host alone: libef.so over a runtime that keeps each launch's grid and arguments instead of
running it (fake_hip_grids.c)."""
import os
import subprocess
import sys

import pytest

import paper_1905_10936_amd as ef

HERE = os.path.dirname(os.path.abspath(__file__))

DRIVER = r"""
import ctypes, struct, sys
fake, L = ctypes.CDLL(sys.argv[1]), ctypes.CDLL(sys.argv[2])
fake.fake_launched.restype = ctypes.c_char_p
vp, i64 = ctypes.c_void_p, ctypes.c_int64
class Kept(ctypes.Structure):
    _fields_ = [("grid", ctypes.c_uint), ("threads", ctypes.c_uint), ("argument", ctypes.c_ubyte * 128)]
X, W, Z, ACT, DZ, PRE, DPRE, DX = (vp(i << 46) for i in range(1, 9))

def launches(call):
    fake.fake_begin(-1)
    kept = (Kept * 256)()
    fake.fake_kept(kept)
    assert call() == 0
    n = fake.fake_kept(kept)
    names = fake.fake_launched().decode().split("\n")[:n]
    assert all(k.grid * k.threads < 2 ** 32 and k.grid > 0 for k in kept[:n]), [(k.grid, k.threads) for k in kept[:n]]
    return [(name, k.grid, bytes(k.argument)) for name, k in zip(names, kept)]

def numbers(argument, at, kinds):
    return struct.unpack_from("=" + kinds, argument, at)

def forward(rows, width, inner, z, act):
    first = 0
    for name, grid, a in launches(lambda: L.ef_gated_forward(i64(rows), i64(width), i64(inner), 1, X, i64(width), W, i64(width), 0, None, i64(0), Z if z else None,
                                                             i64(inner), ACT if act else None, None)):
        assert "k_gated" in name
        n, _, f, x, = numbers(a, 0, "qqqQ")
        to, _, codes, scales, groups, tiles_t, tiles_c = numbers(a, 80, "QqQQqii")
        assert f == inner and grid == tiles_t * tiles_c and x == X.value + first * width * 2
        assert to == (Z.value + first * inner * 2 if z else 0)
        padded = (inner + 31) // 32 * 32
        assert not act or (groups == padded // 32 and codes == ACT.value + first * padded and scales - first * padded // 32 >= ACT.value + rows * padded)
        # the tiles are as many as the tokens and the channels take, of 32 to 256 and 16 to 128
        assert n / tiles_t <= 256 and inner / tiles_c <= 128 and n > (tiles_t - 1) * 32 and inner > (tiles_c - 1) * 16
        first += n
    assert first == rows

def backward(workspace, rows, width, inner):
    first = 0
    for name, grid, a in launches(lambda: L.ef_gated_backward(workspace, i64(rows), i64(width), i64(inner), 1, DZ, i64(inner), PRE, i64(2 * inner), W, i64(width), 0, DPRE,
                                                              i64(2 * inner), DX, i64(width), None)):
        if "k_input_grad" not in name:
            continue
        n, channels, k, dpre = numbers(a, 0, "qqqQ")
        dx, _, tiles_t, tiles_c, splits = numbers(a, 56, "Qqiii")
        assert channels == width and k == 2 * inner and splits >= 1 and grid == tiles_t * tiles_c * splits
        assert dpre == DPRE.value + first * 4 * inner and dx == DX.value + first * 2 * width
        assert n / tiles_t <= 256 and width / tiles_c <= 256 and n > (tiles_t - 1) * 64 and width > (tiles_c - 1) * 64
        first += n
    assert first == rows

workspace = vp()
assert L.ef_workspace_create(ctypes.byref(workspace), i64(1 << 23), None) == 0
"""

SIZES = DRIVER + r"""
for z, act in ((True, True), (False, True), (True, False)):
    for rows, inner in ((100, 1 << 24), (8192, 1 << 24), (8193, 1 << 24), (20000, (1 << 24) - 1), (1 << 22, 32768), (1 << 22, 32769), ((1 << 22) + 1, 40000), (5 << 22, 300)):
        forward(rows, 1, inner, z, act)
for rows, width in ((100, 1 << 24), (8192, 1 << 24), (20000, (1 << 24) - 1), (1 << 22, 32768), (1 << 22, 32769), ((1 << 22) + 1, 40000), (1 << 23, 300)):
    backward(workspace, rows, width, 1)
print("launches ok")
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    ef.lib()
    fake = str(tmp_path_factory.mktemp("fake") / "fake_hip_grids.so")
    subprocess.run([os.environ.get("CC", "gcc"), "-O1", "-shared", "-fPIC", "-w", "-I", HERE, "-o", fake, os.path.join(HERE, "fake_hip_grids.c")], check=True)

    def run(driver):
        done = subprocess.run([sys.executable, "-c", driver, fake, ef.LIB_PATH], capture_output=True, text=True, timeout=120, env=dict(os.environ, LD_PRELOAD=fake))
        assert done.returncode == 0, done.stdout + done.stderr
        assert "launches ok" in done.stdout
    return run


def test_every_width_is_taken(run):
    """Widths up to 2^24 with any number of tokens: in launches of as many tokens as their grid takes."""
    run(SIZES)


KERNELS = DRIVER + r"""
for kernel in range(4):
    assert L.ef_gated_kernels(kernel, kernel, 0) == 0
    for rows, channels in ((1, 1), (100, 1 << 24), (8192, 1 << 24), (1 << 22, 32768), (1 << 23, 300)):
        forward(rows, 1, channels, True, True)
        backward(workspace, rows, channels, 1)
print("launches ok")
"""


def test_kernels_that_are_asked_for(run):
    """Where a grid does not hold their tiles another one is taken."""
    run(KERNELS)
