"""The look that a build takes at the accumulators of the 8-bit products: what this compiler makes passes, and each mistake that it could make is found."""
import os
import re
import shutil

import pytest

from paper_2605_28691_amd import accumulators, build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC) and not shutil.which(HIPCC), reason="no hipcc")


@pytest.fixture(scope="module")
def made():
    return build.assembly(accumulators.SOURCE)


def test_what_the_compiler_makes(made):
    accumulators.check(made)


def _changed(made, kernel, change):
    """The assembly with one kernel's body changed: change(lines, indices of its products) -> lines."""
    m = re.search(r"^_ZN8skiparse13linear_kernelILi%dELi%dELi3E\w+:(.*?)\.Lfunc_end" % (kernel, kernel), made, re.S | re.M)
    lines = m.group(1).split("\n")
    products = [i for i, x in enumerate(lines) if x.strip().startswith("v_mfma_i32")]
    return made[:m.start(1)] + "\n".join(change(lines, products)) + made[m.end(1):]


def _insert(at, line):
    return lambda lines, products: lines[:at(lines, products)] + ["\t" + line] + lines[at(lines, products):]


def _first(lines, what):
    return next(i for i, x in enumerate(lines) if x.strip().startswith(what))


BEFORE = lambda lines, products: products[0]  # noqa: E731
WITHIN = lambda lines, products: products[len(products) // 2]  # noqa: E731
WAIT = lambda lines, products: next(i for i, x in enumerate(lines) if x.strip() == "s_nop 15") + 1  # noqa: E731
END = lambda lines, products: _first(lines, "s_endpgm")  # noqa: E731


USES = ["v_accvgpr_write_b32 a3, v7", "v_accvgpr_read_b32 v7, a3", "v_accvgpr_mov_b32 a3, a4", "v_accvgpr_write_b32 a[3], 0", "global_load_dwordx4 a[0:3], v[2:3], off", "ds_read_b128 a[4:7], v1",
        "global_store_dword v[2:3], a5, off", "buffer_load_dword a15, v1, s[0:3], 0 offen", "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]", "v_accvgpr_write_b32 a250, v7",
        "v_mfma_i32_16x16x64_i8 a[0:3], v[0:3], v[4:7], a[4:7]"]


@pytest.mark.parametrize("kernel, at, line", [(64, at, line) for at in (BEFORE, WITHIN, WAIT, END) for line in USES] + [(kernel, at, line) for kernel in (128, 256) for at, line in zip((BEFORE, WITHIN, WAIT, END), USES)])
def test_another_use_of_an_accumulator(made, kernel, at, line):
    with pytest.raises(RuntimeError, match="linear_kernel"):
        accumulators.check(_changed(made, kernel, _insert(at, line)))


@pytest.mark.parametrize("kernel", [64, 128, 256])
def test_a_wait_or_a_sum_that_is_missing(made, kernel):
    waits = [i for i, x in enumerate(made.split("\n")) if x.strip() == "s_nop 15"]
    assert waits
    without = lambda what: lambda lines, products: lines[:what(lines)] + lines[what(lines) + 1:]  # noqa: E731
    for change in (lambda lines, products: [x for x in lines if x.strip() != "s_nop 15"], without(lambda lines: _first(lines, "v_accvgpr_write_b32")), without(lambda lines: _first(lines, "v_accvgpr_read_b32"))):
        with pytest.raises(RuntimeError, match="linear_kernel"):
            accumulators.check(_changed(made, kernel, change))

    def written_in_front(lines, products):
        i = products[len(products) // 2]
        operand = re.search(r"v\[(\d+):", lines[i].split(",", 1)[1]).group(1)
        return lines[:i] + ["\tv_add_u32_e32 v%s, v0, v1" % operand] + lines[i:]

    with pytest.raises(RuntimeError, match="reads"):
        accumulators.check(_changed(made, kernel, written_in_front))


def test_registers_and_kernels_that_are_missing(made):
    m = re.search(r"\.amdhsa_kernel _ZN8skiparse13linear_kernelILi256ELi256ELi3E\w+\s.*?\.amdhsa_next_free_vgpr (\d+)", made, re.S)
    for n in (255, int(m.group(1)) - 256):
        with pytest.raises(RuntimeError, match="fewer"):
            accumulators.check(made[:m.start(1)] + str(n) + made[m.end(1):])
    with pytest.raises(RuntimeError, match="instead of"):
        accumulators.check(made.replace("linear_kernelILi64ELi64ELi3ELb1", "another_kernel"))
    with pytest.raises(RuntimeError, match="instead of"):
        accumulators.check("")


def test_registers():
    assert accumulators.registers("v[8:11], a[0x41], a7, s[2:3], v3") == {("v", 8), ("v", 9), ("v", 10), ("v", 11), ("a", 0x41), ("a", 7), ("v", 3)}


def test_a_build_without_the_check_passed_leaves_no_library(tmp_path, monkeypatch):
    """An older library stays, as after any other failed build."""
    lib = tmp_path / "lib.so"
    lib.write_bytes(b"old")
    seen = []

    def run(cmd, verbose):
        out = cmd[cmd.index("-o") + 1]
        with open(out, "w") as f:
            f.write("")
        seen.append(cmd)

    monkeypatch.setattr(build, "_run", run)
    with pytest.raises(RuntimeError, match="instead of"):
        build._build_one(str(lib), build.SOURCES, False, False)
    assert sorted(p.name for p in tmp_path.iterdir()) == ["lib.so"] and lib.read_bytes() == b"old"
    # the library's own flags, without those of the host's side
    library, kernels = seen
    assert [f for f in build.FLAGS if f != "-shared"] == kernels[1:len(build.FLAGS)] and library[1:len(build.FLAGS) + 1] == build.FLAGS and "--cuda-device-only" in kernels
    assert build._build_one(str(lib), build.PROBE_SOURCES, False, False) == str(lib) and lib.read_bytes() == b""
