"""A look through the assembly of the products in 8-bit integers (csrc/linear_tiles.h).  Their sums are in accumulation registers that the compiler does not know to hold anything, and their products are statements
whose latency it does not see.  So a build compiles them once more to assembly, and fails where that shows one of these:

  - any instruction but their own that names an accumulation register: each is cleared once, in front of all products, and read once in either way out;
  - a way from a product to anything that reads an accumulator without the wait (s_nop 15) in between;
  - a vector instruction that writes what one of the next two products reads;
  - fewer accumulation registers than a tile has sums for a lane.
"""
from __future__ import annotations

import re

SOURCE = "linear_int8.hip"
FORMS = 6  # three tiles, with an epilogue's extras and without
_KERNEL = re.compile(r"^(_ZN8skiparse13linear_kernelILi(\d+)ELi(\d+)ELi3E\w+):(.*?)\.Lfunc_end", re.S | re.M)
_NUMBER = r"(0x[0-9a-f]+|\d+)"
_ONE = re.compile(r"\b([va])(\d+)\b")
_SOME = re.compile(r"\b([va])\[" + _NUMBER + r"(?::" + _NUMBER + r")?\]")
_CLEARED = re.compile(r"v_accvgpr_write_b32 (a\S+), 0$")
_READ = re.compile(r"v_accvgpr_read_b32 v\S+, (a\S+)$")
_PRODUCT = "v_mfma_i32_16x16x64_i8 "
_WAIT = "s_nop 15"


def registers(text: str) -> set:
    """{("v" or "a", number)} of what an instruction names: v[8:11], a[0x41], a7."""
    found = {(kind, int(n)) for kind, n in _ONE.findall(text)}
    for kind, first, last in _SOME.findall(text):
        found |= {(kind, i) for i in range(int(first, 0), int(last or first, 0) + 1)}
    return found


def _operands(line: str) -> list:
    return line.split(None, 1)[1].split(",")


def _accumulators(line: str) -> set:
    return {i for kind, i in registers(line.split(None, 1)[-1]) if kind == "a"}


def check(assembly: str) -> None:
    """Raises RuntimeError where a kernel is not as it has to be."""
    kernels = _KERNEL.findall(assembly)
    if len(kernels) != FORMS:
        raise RuntimeError(f"{len(kernels)} products in 8-bit integers instead of {FORMS}")
    for name, rows, channels, body in kernels:
        _check_kernel(name, int(rows) * int(channels) // 256, body)
        described = re.search(r"\.amdhsa_kernel " + name + r"\b(.*?)\.end_amdhsa_kernel", assembly, re.S)
        size = {key: int(n) for key, n in re.findall(r"\.amdhsa_(next_free_vgpr|accum_offset) (\d+)", described.group(1))} if described else {}
        if size.get("next_free_vgpr", 0) - size.get("accum_offset", 0) < int(rows) * int(channels) // 256:
            raise RuntimeError(f"{name}: fewer accumulation registers than sums: {size}")


def _check_kernel(name: str, sums: int, body: str) -> None:
    def fail(why, line=""):
        raise RuntimeError(f"{name}: {why}: {line}")

    lines = [x.split(";")[0].strip() for x in body.split("\n")]
    lines = [x for x in lines if x and (not x.startswith(".") or x.startswith(".LBB"))]
    label = {x.rstrip(":"): i for i, x in enumerate(lines) if x.startswith(".LBB")}
    products = [i for i, x in enumerate(lines) if x.startswith(_PRODUCT)]
    if not products:
        fail("no products")
    cleared, read, added = [], [], set()
    for i, x in enumerate(lines):
        named = _accumulators(x) if not x.startswith(".LBB") else set()
        if not named:
            continue
        if i in products:
            to, _, _, of = _operands(x)
            if to.strip() != of.strip() or _accumulators("x " + to) != named or len(named) != 4:
                fail("a product that is not added to its own sum", x)
            added |= named
        elif _CLEARED.match(x):
            if i > products[0]:
                fail("cleared behind a product", x)
            cleared += named
        elif _READ.match(x):
            if i < products[-1]:
                fail("read between products", x)
            read += named
        else:
            fail("names an accumulation register", x)
    if added != set(range(sums)) or sorted(cleared) != sorted(added) or sorted(read) != sorted(list(added) * 2):
        fail("not every sum is cleared once, added to, and read in both ways out")
    # in front of the products control goes forward only: what is cleared is so once
    for i, x in enumerate(lines):
        m = re.match(r"s_c?branch\w*\s+(\.LBB\w+)", x)
        if m and i >= products[0] and label[m.group(1)] <= max(j for j, y in enumerate(lines) if _CLEARED.match(y)):
            fail("goes back to where sums are cleared", x)
    # from behind every product along all ways: other products, or the wait first
    seen, todo = set(), [i + 1 for i in products]
    while todo:
        i = todo.pop()
        if i in seen or i >= len(lines):
            continue
        seen.add(i)
        x = lines[i]
        if x.startswith(_WAIT) or x.startswith("s_endpgm"):
            continue
        if not x.startswith(_PRODUCT) and not x.startswith(".LBB") and _accumulators(x):
            fail("comes upon a sum without the wait", x)
        m = re.match(r"s_c?branch\w*\s+(\.LBB\w+)", x)
        if m:
            todo.append(label[m.group(1)])
        if not x.startswith("s_branch"):
            todo.append(i + 1)
    for i in products:
        reads = set().union(*(registers(a) for a in _operands(lines[i])[1:]))
        for x in lines[max(0, i - 2):i]:
            if x.startswith("v_") and not x.startswith("v_mfma") and reads & registers(_operands(x)[0]):
                fail("writes what a product behind it reads", x)
