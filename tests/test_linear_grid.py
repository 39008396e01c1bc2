"""Products and passes over rows of the linear layer fit the grid of one launch, or are refused before anything is sent."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LIMIT = (1 << 32) // 256  # workgroups of 256 threads: a grid has fewer than 2^32 threads


@pytest.mark.skipif(not os.path.exists(HIPCC) and not shutil.which(HIPCC), reason="no hipcc")
def test_workgroups_of_every_size_that_is_taken(tmp_path):
    exe = str(tmp_path / "host_linear_grid_check")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", os.path.join(ROOT, "tests", "host_linear_grid_check.cpp"), "-o", exe], check=True, stderr=subprocess.PIPE)
    rng = random.Random(2)
    sizes = [(1 << 30, 8, 8), (1 << 30, 64, 64), (1_200_000_000, 8, 16), (2147483647, 8, 8), (2147483647, 504, 8), (1 << 30, 1016, 8), (1 << 30, 1008, 8), (8, 8, 2147483647),
             (1 << 20, (1 << 20) - 8, 64), (8, (1 << 23) - 8, 8), (80640, 5120, 5120), (1, 8, 8)]
    while len(sizes) < 400:
        M, N, K = round(2 ** rng.uniform(0, 31)), 8 * round(2 ** rng.uniform(0, 20)), 8 * round(2 ** rng.uniform(0, 20))
        if M < 1 << 31 and N < 1 << 23 and K < 1 << 23 and M * N < 1 << 40 and M * K < 1 << 40 and N * K < 1 << 40:
            sizes.append((M, N, K))
    done = subprocess.run([exe], input="".join("%d %d %d\n" % s for s in sizes), stdout=subprocess.PIPE, text=True, check=True)
    fits = 0
    for (M, N, K), line in zip(sizes, done.stdout.splitlines()):
        fit, products, per, rows = map(int, line.split())
        assert fit == (-(-M // 256) * -(-N // 256) < LIMIT), (M, N, K)
        assert not fit or 0 < products < LIMIT, (M, N, K, products)
        assert rows == -(-M // per) * -(-N // 256) < LIMIT, (M, N, K, per)
        assert per >= (32 if M < 32768 else 128) and (per <= 128 or -(-M // (per // 2)) * -(-N // 256) >= LIMIT), (M, N, per)  # no longer than need be
        fits += fit
    assert fits > 300 and fits < len(sizes)


def test_results_beyond_one_launch_are_refused_first():
    """With ESHAPE, where the pass over rows or another product of the call would have been sent already."""
    import paper_2605_28691_amd as sk

    L = sk.lib()
    at = [ctypes.c_void_p(0x10000 + i * (1 << 44)) for i in range(8)]  # never dereferenced
    big, wide = 1 << 30, 1016

    def fwd(K, N):
        return L.skiparse_linear_fwd(at[0], at[1], None, None, at[2], None, None, 1, 1, 1, big, K, N, 1, 0, 0, 0, 0, at[3], 1 << 43, None)

    def bwd(K, N, dx=at[4], dw=at[5], db=at[6]):
        return L.skiparse_linear_bwd(at[0], at[1], None, at[2], None, None, None, dx, dw, db, 1, 1, 1, big, K, N, 1, 0, 0, 0, 0, at[7], 1 << 43, None)

    assert fwd(8, wide) == -2
    assert bwd(wide, 8) == -2 and bwd(wide, 8, dw=None) == -2
