"""pair_verify_drafts on two devices of one process, with a stand-in for the CUDA
runtime's launch calls (no GPU): each device gets its own attribute for large
clusters and its own count of clusters that fit."""
import os
import subprocess
import sys

from paper_2608_11368_gb300 import build

HERE = os.path.dirname(os.path.abspath(__file__))

CHILD = """
import ctypes, sys
fake, lib = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL), ctypes.CDLL(sys.argv[2])
P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
lib.pair_verify_drafts.argtypes = [I64, I32, I32, I32, P, I64, P, I64] + [P] * 9
one, R, V = P(1 << 20), 4, 151936
for dtype in (0, 1):
    for k, device in enumerate((0, 1, 0, 1)):
        fake.fake_set_device(device)
        before = fake.fake_launches()
        st = lib.pair_verify_drafts(8, R, V, dtype, one, V, one, V, one, one, one, one, one, one,
                                    one, None, None)
        fits = (9, 2)[device]
        print(st, fake.fake_launches() - before, fake.fake_cluster(), fake.fake_grid(),
              16 * min(R, fits))
"""


def test_clusters_of_two_devices(tmp_path):
    lib, fake = build.build(), str(tmp_path / "fake_cudart.so")
    include = os.path.join(os.path.dirname(os.path.dirname(build.nvcc())), "include")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", include, "-o", fake,
                    os.path.join(HERE, "fake_cudart.cpp")], check=True)
    env = dict(os.environ, LD_PRELOAD=fake, CUDA_VISIBLE_DEVICES="")
    res = subprocess.run([sys.executable, "-c", CHILD, fake, lib], env=env, capture_output=True,
                         text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-2000:]
    rows = [[int(x) for x in line.split()] for line in res.stdout.splitlines()]
    assert len(rows) == 8
    for st, launched, cluster, grid, want in rows:
        assert (st, launched, cluster, grid) == (0, 1, 16, want)
