"""How products of the linear layer are cut into workgroups: every part of every tile once, sums that fit the workspace; and what the compiler makes of the products."""
import os
import random
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
needs_hipcc = pytest.mark.skipif(not os.path.exists(HIPCC) and not shutil.which(HIPCC), reason="no hipcc")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("linear_plan") / "host_linear_plan_check")
    src = os.path.join(ROOT, "tests", "host_linear_plan_check.cpp")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", src, "-o", exe], check=True, stderr=subprocess.PIPE)

    def run(sizes):
        done = subprocess.run([exe], input="".join("%d %d %d\n" % s for s in sizes), stdout=subprocess.PIPE, text=True, check=True)
        return [line.split() for line in done.stdout.splitlines()]

    return run


@needs_hipcc
def test_every_part_of_every_tile_once(plans):
    rng = random.Random(1)
    sizes = [(1, 8, 8), (1, 5120, 5120), (128, 128, 128), (129, 8, 64), (80640, 5120, 5120), (1536, 1536, 32760), (3840, 5120, 5120), (6426, 4008, 1000), (257, 257 * 8, 100000),
             (5120, 5120, 80640), (8, 8, 2000000), (65536, 64, 64)]
    sizes += [(round(2 ** rng.uniform(0, 16)), 8 * round(2 ** rng.uniform(0, 11)), 8 * round(2 ** rng.uniform(0, 12))) for _ in range(300)]
    for size, got in zip(sizes, plans(sizes)):
        assert got[-1] == "ok", (size, got)


@needs_hipcc
def test_both_ends_of_the_rule(plans):
    """Large products take the largest tiles, small ones the smallest; a last round that would leave most of the chip idle is cut, a full one is not."""
    m, n, whole, rest, parts, size, _ = (int(x) if x.isdigit() else x for x in plans([(32768, 2048, 4096)])[0])
    assert (m, n, whole, rest, parts, size) == (256, 256, 1024, 0, 1, 0)
    m, n, whole, rest, parts, size, _ = (int(x) if x.isdigit() else x for x in plans([(1536, 1536, 32760)])[0])
    assert whole == 0 and rest == 1536 // m * (1536 // n) and parts > 2 and size == rest * parts * m * n * 4
    assert plans([(256, 256, 256)])[0][0] in ("64", "128")


# products (rows, channels, sum) that take tiles of 128 x 256, one not cut and one cut; tests/test_gpu_linear.py has them in each form
WIDE = [(6566, 536, 2056), (528, 3616, 4008)]


@needs_hipcc
def test_wide_tiles(plans):
    """Where 128 x 128 would leave a fifth of a round empty, and 256 x 256 most of one."""
    for size, got in zip(WIDE, plans(WIDE)):
        assert got[:2] == ["128", "256"] and (got[4] == "1") == (size == WIDE[0]), (size, got)


def test_workspace_is_what_the_plan_says():
    import paper_2605_28691_amd as sk

    assert sk.skiparse_linear_workspace_bytes(0, 64, 64) == 0 and sk.skiparse_linear_workspace_bytes(64, -1, 64) == 0
    assert sk.skiparse_linear_workspace_bytes(32768, 4096, 2048) == 0
    # dw of 32,760 rows is cut along the rows
    assert sk.skiparse_linear_bwd_workspace_bytes(32760, 1536, 1536) > 2 * 1536 * 1536 * 4


@needs_hipcc
def test_accumulators_are_not_read_before_they_are_written(tmp_path):
    """The products are asm, so the compiler does not wait for them by itself.  In the code that it makes: a walk's last product is followed by its wait (s_nop 15) before anything
    that reads an accumulation register other than a product, and what a product multiplies is nothing that a vector instruction has just written."""
    out = str(tmp_path / "linear.s")
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "--cuda-device-only", "-S"]
    subprocess.run([HIPCC, *flags, os.path.join(ROOT, "paper_2605_28691_amd", "csrc", "linear.hip"), "-o", out], check=True, stderr=subprocess.PIPE)
    text = open(out).read()
    kernels = re.findall(r"^(_ZN8skiparse13linear_kernel\w+):(.*?)\.Lfunc_end", text, re.S | re.M)
    assert len(kernels) >= 9
    for name, body in kernels:
        # blocks, and where each goes
        blocks, label = {}, "entry"
        order = [label]
        blocks[label] = []
        for line in body.split("\n"):
            m = re.match(r"(\.LBB\w+):", line)
            if m:
                label = m.group(1)
                blocks[label] = []
                order.append(label)
                continue
            line = line.strip()
            if line and line[0] not in ";.":
                blocks[label].append(line)
        following = {a: b for a, b in zip(order, order[1:])}

        # is an unfinished product possible where a block begins?
        pending = {at: False for at in order}

        def walk(at, state, report=None):
            """Where control goes from the block, and whether a product is unfinished then."""
            to = []
            for line in blocks[at]:
                m = re.match(r"s_c?branch\w*\s+(\.LBB\w+)", line)
                if m:
                    to.append((m.group(1), state))
                elif line.startswith("v_mfma"):
                    state = True
                elif line.startswith("s_nop 15"):
                    state = False
                elif state and report is not None and re.search(r"[\s,]a(\d|\[)", line):
                    report.append(line)
            if at in following and not (blocks[at] and blocks[at][-1].startswith(("s_branch", "s_endpgm"))):
                to.append((following[at], state))
            return to

        changed = True
        while changed:
            changed = False
            for at in order:
                for to, state in walk(at, pending[at]):
                    if state and not pending[to]:
                        pending[to] = changed = True
        found = []
        for at in order:
            walk(at, pending[at], found)
        assert not found, (name, found[:5])
        # vector instructions that write what a product reads, without two instructions between
        for at in order:
            recent = []
            for line in blocks[at]:
                op, _, rest = line.partition("\t") if "\t" in line else line.partition(" ")
                args = [x.strip() for x in rest.split(",")]
                if op.startswith("v_mfma"):
                    reads = set()
                    for x in args[1:4]:
                        m = re.match(r"([va])\[(\d+):(\d+)\]", x)
                        reads |= {(m.group(1), i) for i in range(int(m.group(2)), int(m.group(3)) + 1)}
                    assert not reads & {r for rs in recent[-2:] for r in rs}, (name, line)
                    recent.append(set())
                    continue
                writes = set()
                if op.startswith("v_"):
                    m = re.match(r"([va])\[(\d+):(\d+)\]$", args[0]) or re.match(r"([va])(\d+)()$", args[0])
                    if m:
                        lo = int(m.group(2))
                        writes = {(m.group(1), i) for i in range(lo, int(m.group(3) or lo) + 1)}
                recent.append(writes)
