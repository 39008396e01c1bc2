"""How products in 8-bit integers are cut, on the host: every part of every tile once, one workspace for every epilogue, and GPU tests that reach every kernel."""
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_linear_int8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC) and not shutil.which(HIPCC), reason="no hipcc")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("linear8_plan") / "host_linear8_plan_check")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", os.path.join(ROOT, "tests", "host_linear8_plan_check.cpp"), "-o", exe], check=True, stderr=subprocess.PIPE)

    def run(sizes):  # (M, K, N)
        done = subprocess.run([exe], input="".join("%d %d %d\n" % (m, n, k) for m, k, n in sizes), stdout=subprocess.PIPE, text=True, check=True)
        got = []
        for line in done.stdout.splitlines():
            w = line.split()
            assert w[4] == w[8] == "ok", line
            got.append((int(w[0]), tuple(map(int, w[1:4])), tuple(map(int, w[5:8]))))
        return got

    return run


def test_every_part_of_every_tile_once(plans):
    import paper_2605_28691_amd as sk

    rng = random.Random(2)
    sizes = [(1, 16, 8), (33, 16, 8), (33, 131056, 8), (80640, 5120, 20480), (32760, 1536, 1536), (6426, 1008, 4008), (65536, 64, 64), (300000, 16, 8), (17, 256, 72), (40, 131056, 72)]
    sizes += [(round(2 ** rng.uniform(0, 16)), 16 * round(2 ** rng.uniform(0, 12)), 8 * round(2 ** rng.uniform(0, 11))) for _ in range(300)]
    for (m, k, n), (few, *cuts) in zip(sizes, plans(sizes)):
        space = sk.skiparse_linear_fwd_int8_workspace_bytes(m, k, n)
        if few:
            assert space == 0
            continue
        for tm, tn, parts in cuts:
            tiles = -(-m // tm) * -(-n // tn)
            slots = 256 * {(256, 256): 1, (128, 128): 2, (64, 64): 4}[tm, tn]
            assert space >= (tiles % slots * parts * tm * tn * 4 if parts > 1 else 0)


def test_the_gpu_tests_reach_every_kernel(plans):
    got = plans(test_gpu_linear_int8.SIZES)
    assert {few for few, *_ in got} == {0, 1, 3, 4, 5, 6}
    reached = [{(tm, tn, parts > 1) for few, *cuts in got if not few for tm, tn, parts in (cuts[act],)} for act in (0, 1)]
    assert reached[0] == reached[1] == {(n, n, cut) for n in (256, 128, 64) for cut in (False, True)}
