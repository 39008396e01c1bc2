"""The binding's native module built once more for tensors of the CPU (device -1), with functions of the test's in the place of the library's, so that its whole calls run without a GPU; and with a look at
every tensor that it makes: whether the interpreter's lock is held meanwhile (an allocation can wait for the GPU, and other threads with it)."""
import ctypes
import importlib.machinery
import importlib.util
import os
import shutil

import paper_2605_28691_amd as sk

LAUNCHES = ("skiparse_rmsnorm_fwd", "skiparse_rmsnorm_bwd", "skiparse_quantize_int8", "skiparse_linear_fwd_int8")
SPACE = 48  # bytes that the workspaces need, as the module is told
EMPTY = """
static at::Tensor unlocked_empty(at::IntArrayRef shape, at::TensorOptions options) {
    if (PyGILState_Check()) throw 0;  // the call is not answered then
    return at::empty(shape, options);
}
"""


def build(folder: str) -> str:
    """Compiles the module into `folder`; returns its path."""
    from paper_2605_28691_amd import build as b

    csrc = os.path.join(folder, "package", "csrc")
    os.makedirs(csrc)
    shutil.copytree(os.path.join(os.path.dirname(b.HERE), "include"), os.path.join(folder, "include"))
    with open(os.path.join(b.CSRC, "marshal.cpp")) as f:
        source = f.read()
    assert source.count("is_cuda()") == 2 and source.count("at::empty(") == 10
    source = source.replace("is_cuda()", "is_cpu()").replace("at::empty(", "unlocked_empty(").replace("\nnamespace {\n", EMPTY + "\nnamespace {\n", 1)
    with open(os.path.join(csrc, "marshal.cpp"), "w") as f:
        f.write(source)
    kept = b.CSRC, b.MARSHAL
    b.CSRC, b.MARSHAL = csrc, os.path.join(folder, "_marshal.so")
    try:
        return b._build_marshal(False)
    finally:
        b.CSRC, b.MARSHAL = kept


class Host:
    """The module, and in `calls` (name, arguments) of what it has called; `code` is what those calls answer."""

    def __init__(self, path: str):
        loader = importlib.machinery.ExtensionFileLoader("_marshal", path)
        self.native = importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader))
        loader.exec_module(self.native)
        self.calls, self.code, self._held, L = [], 0, [], sk.lib()
        self.native.set_up(lambda *args: self.calls.append(("general", args)), sk._failed)
        for name in LAUNCHES:
            f = getattr(L, name)
            self._bind(name, f, lambda *args, name=name: self.calls.append((name, args)) or self.code)
        for name in sk._PLAIN_SIZES:
            self._bind(name, getattr(L, name), lambda *args: SPACE)

    def _bind(self, name, f, does):
        self._held.append(ctypes.CFUNCTYPE(f.restype, *f.argtypes)(does))
        self.native.bind(name, ctypes.cast(self._held[-1], ctypes.c_void_p).value)


def device() -> int:
    return -1


def stream(at: int) -> int:
    assert at == -1
    return 5
