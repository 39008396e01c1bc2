"""How the passes over rows are cut, on the host: every channel of every row has a lane, every shape has a kernel, and the GPU tests reach each of them; and what the compiler makes of the 8-bit products."""
import os
import random
import re
import shutil
import subprocess

import pytest

import test_gpu_norm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_28691_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
needs_hipcc = pytest.mark.skipif(not os.path.exists(HIPCC) and not shutil.which(HIPCC), reason="no hipcc")
LANES, WAVE, GROUP = range(3)
FORWARD = {(LANES, 1), (WAVE, 1), (WAVE, 2), (WAVE, 3), (GROUP, 1), (GROUP, 2), (GROUP, 4)}
BACKWARD = {(LANES, 1), (WAVE, 1), (WAVE, 2), (GROUP, 1), (GROUP, 2), (GROUP, 4)}


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("norm_shape") / "host_norm_shape_check")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", os.path.join(ROOT, "tests", "host_norm_shape_check.cpp"), "-o", exe], check=True, stderr=subprocess.PIPE)

    def run(sizes):
        done = subprocess.run([exe], input="".join("%d %d\n" % s for s in sizes), stdout=subprocess.PIPE, text=True, check=True)
        got = [list(map(int, line.split())) for line in done.stdout.splitlines()]
        return [[tuple(g[0:4]), tuple(g[4:8]), tuple(g[8:12])] for g in got], [tuple(g[12:]) for g in got]

    return run


def _holds(span, ch, lanes, threads, cols):
    pieces = -(-cols // 8)
    if span == LANES:
        return ch == 1 and lanes in (1, 2, 4, 8, 16, 32) and pieces <= lanes and (lanes == 1 or pieces > lanes // 2) and threads == 256
    if span == WAVE:
        return pieces <= 64 * ch and threads == 256
    return pieces <= threads * ch and threads % 64 == 0 and threads <= 1024


@needs_hipcc
def test_every_channel_has_a_lane_and_every_shape_a_kernel(shapes):
    rng = random.Random(3)
    sizes = [(r, 8 * c) for r in (1, 2, 255, 256, 1023, 1024, 2048, 100_000, 2147483647) for c in (1, 2, 3, 4, 32, 33, 64, 65, 128, 129, 192, 193, 1024, 1025, 2048, 2049, 4096)]
    sizes += [(round(2 ** rng.uniform(0, 30)), 8 * round(2 ** rng.uniform(0, 12))) for _ in range(500)]
    forward, backward = shapes(sizes)
    seen = set(), set()
    for (rows, cols), fs, (span, ch, lanes, threads, parts) in zip(sizes, forward, backward):
        for f in fs:
            assert (f[0], f[1]) in FORWARD and _holds(*f, cols), (rows, cols, f)
            seen[0].add(f[:2])
        assert (span, ch) in BACKWARD and _holds(span, ch, lanes, threads, cols), (rows, cols, span, ch)
        at_once = threads // lanes if span == LANES else threads // 64 if span == WAVE else 1
        assert 1 <= parts <= -(-rows // at_once) and parts <= 2048, (rows, cols, parts)
        seen[1].add((span, ch))
    assert seen[0] == FORWARD and seen[1] == BACKWARD


@needs_hipcc
def test_the_gpu_tests_reach_every_kernel(shapes):
    forward, backward = shapes(test_gpu_norm.SIZES)
    # what is read of a channel: bf16 2, or 4 with a residual; float32 4 or 8
    assert {f[:2] for fs in forward for f in fs} == FORWARD and {fs[0][:2] for fs in forward} >= {(WAVE, 3), (GROUP, 2)}
    assert {b[:2] for b in backward} == BACKWARD


@needs_hipcc
def test_accumulators_of_the_8_bit_products(tmp_path):
    """The products are asm, and the compiler does not wait for them by itself: between a walk's last product and anything else that touches an accumulation register stands the wait (s_nop 15), whichever
    way control goes; and no vector instruction writes what one of the next two products reads."""
    out = str(tmp_path / "linear_int8.s")
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "--cuda-device-only", "-S"]
    subprocess.run([HIPCC, *flags, os.path.join(CSRC, "linear_int8.hip"), "-o", out], check=True, stderr=subprocess.PIPE)
    kernels = re.findall(r"^(_ZN8skiparse13linear_kernel\w+):(.*?)\.Lfunc_end", open(out).read(), re.S | re.M)
    assert len(kernels) == 6
    number = r"(0x[0-9a-f]+|\d+)"

    def registers(x):  # v[8:11], a[0x41], a7
        found = {(kind, int(n, 0)) for kind, n in re.findall(r"\b([va])(\d+)\b", x)}
        for kind, first, last in re.findall(r"\b([va])\[" + number + "(?::" + number + r")?\]", x):
            found |= {(kind, i) for i in range(int(first, 0), int(last or first, 0) + 1)}
        return found

    for name, body in kernels:
        lines = [x.split(";")[0].strip() for x in body.split("\n")]
        lines = [x for x in lines if x and (not x.startswith(".") or x.startswith(".LBB"))]
        label = {x.rstrip(":"): i for i, x in enumerate(lines) if x.startswith(".LBB")}
        products = [i for i, x in enumerate(lines) if x.startswith("v_mfma_i32_16x16x64_i8")]
        tile = int(re.search(r"ILi(\d+)ELi", name).group(1)) * int(re.search(r"ELi(\d+)ELi3E", name).group(1))
        # the accumulators are the program's: cleared once, read in both ways out, and the compiler has no use for them
        moved = [x for x in lines if x.startswith("v_accvgpr")]
        mine = [x for x in moved if all(i < tile // 256 for kind, i in registers(x) if kind == "a")]
        assert sum(x.startswith("v_accvgpr_write") for x in mine) == tile // 256 and sum(x.startswith("v_accvgpr_read") for x in mine) == 2 * tile // 256 and not any("mov" in x for x in mine), name
        assert len(products) > 4 and not any(x.startswith("v_mfma") and i not in products for i, x in enumerate(lines))
        # from behind every product along all ways: other products, or the wait first
        seen, todo = set(), [i + 1 for i in products]
        while todo:
            i = todo.pop()
            if i in seen or i >= len(lines):
                continue
            seen.add(i)
            x = lines[i]
            if x.startswith("s_nop 15") or x.startswith("s_endpgm"):
                continue
            if not x.startswith("v_mfma"):
                assert not any(r == "a" for r, _ in registers(x)), (name, x)
            m = re.match(r"s_c?branch\w*\s+(\.LBB\w+)", x)
            if m:
                todo.append(label[m.group(1)])
            if not x.startswith("s_branch"):
                todo.append(i + 1)
        assert set().union(*(registers(lines[i].split(None, 1)[1].split(",")[0]) for i in products)) == {("a", i) for i in range(tile // 256)}
        for i in products:
            reads = set().union(*(registers(a) for a in lines[i].split(None, 1)[1].split(",")[1:]))
            for x in lines[max(0, i - 2):i]:
                if x.startswith("v_") and not x.startswith("v_mfma"):
                    assert not reads & registers(x.split(None, 1)[1].split(",")[0]), (name, lines[i], x)
