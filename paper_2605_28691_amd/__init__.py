"""MI355X-native Skiparse-2D attention: thin Python binding over the C ABI in ``include/skiparse.h``.

Argument marshalling only.  Tensors are ``torch`` CUDA(HIP) tensors used purely as device memory; every step of
the path runs in the library's own kernels on the current torch stream.  There is no CPU fallback: without the
built library, or on a bad argument, a call raises.
"""
from __future__ import annotations

import ctypes
import functools
import importlib
import operator
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libskiparse.so")

TOKEN, GROUP = 0, 1
BF16, FP32, FP8_E4M3 = 0, 1, 2
FUSED = 1
PAD = 2
PATTERNS = {"token": TOKEN, "group": GROUP}
OUT_LAYOUTS = {"same": 0, "other": 1, "original": 2}
ORDERS = {"same": 0, "to_sparse": 1, "to_original": 2, "stay_sparse": 3}
ROPE_LAYOUTS = {"interleaved": 0, "half": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
ACTS = {"none": 0, "gelu_tanh": 1, "silu": 2}
_DTYPES = {torch.bfloat16: BF16, torch.float32: FP32, torch.uint8: FP8_E4M3, torch.float8_e4m3fn: FP8_E4M3}

_lib = None


class SkiparseError(RuntimeError):
    def __init__(self, code: int, what: str):
        msg = lib().skiparse_strerror(code).decode()
        extra = f" [hipError {lib().skiparse_last_hip_error()}]" if code == -5 else ""
        super().__init__(f"{what}: {msg} (code {code}){extra}")
        self.code = code


def lib() -> ctypes.CDLL:
    """Loads libskiparse.so (built by ``paper_2605_28691_amd.build.build()``); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"{_LIB_PATH} is missing: build it first (python -m paper_2605_28691_amd.build); there is no fallback path"
            )
        L = ctypes.CDLL(_LIB_PATH)
        i, vp, f, d, u, sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_float, ctypes.c_double, ctypes.c_uint, ctypes.c_size_t
        L.skiparse_permute.restype = i
        L.skiparse_permute.argtypes = [vp, vp] + [i] * 9 + [vp]
        L.skiparse_unpermute.restype = i
        L.skiparse_unpermute.argtypes = [vp, vp] + [i] * 9 + [vp]
        L.skiparse_switch_pattern.restype = i
        L.skiparse_switch_pattern.argtypes = [vp, vp] + [i] * 9 + [vp]
        L.skiparse_ssp_pack.restype = i
        L.skiparse_ssp_pack.argtypes = [vp, vp] + [i] * 9 + [vp]
        L.skiparse_ssp_unpack.restype = i
        L.skiparse_ssp_unpack.argtypes = [vp, vp] + [i] * 9 + [vp]
        L.dense_attn_fwd.restype = i
        L.dense_attn_fwd.argtypes = [vp] * 4 + [i] * 6 + [f, i, vp]
        L.skiparse_attn_fwd.restype = i
        L.skiparse_attn_fwd.argtypes = [vp] * 4 + [i] * 8 + [f, i, u, vp, sz, vp]
        L.skiparse_attn_fwd_sparse.restype = i
        L.skiparse_attn_fwd_sparse.argtypes = [vp] * 4 + [i] * 9 + [f, i, vp]
        L.skiparse_lse_bytes.restype = sz
        L.skiparse_lse_bytes.argtypes = [i] * 8 + [u]
        L.skiparse_attn_fwd_lse.restype = i
        L.skiparse_attn_fwd_lse.argtypes = [vp] * 5 + [i] * 8 + [f, i, u, vp]
        L.skiparse_bwd_workspace_bytes.restype = sz
        L.skiparse_bwd_workspace_bytes.argtypes = [i] * 8 + [u]
        L.skiparse_bwd_walk_workspace_bytes.restype = sz
        L.skiparse_bwd_walk_workspace_bytes.argtypes = [i] * 8 + [u]
        L.skiparse_attn_bwd.restype = i
        L.skiparse_attn_bwd.argtypes = [vp] * 9 + [i] * 8 + [f, i, u, vp, sz, vp]
        L.skiparse_attn_bwd_static.restype = i
        L.skiparse_attn_bwd_static.argtypes = [vp] * 9 + [i] * 8 + [f, i, u, vp]
        L.skiparse_static_scratch_bytes.restype = sz
        L.skiparse_static_scratch_bytes.argtypes = []
        L.skiparse_workspace_bytes.restype = sz
        L.skiparse_workspace_bytes.argtypes = [i] * 8 + [u]
        L.skiparse_quantize_fp8_ex.restype = i
        L.skiparse_quantize_fp8_ex.argtypes = [vp, vp, vp] + [i] * 8 + [u, vp]
        L.skiparse_attn_fwd_fp8_ex.restype = i
        L.skiparse_attn_fwd_fp8_ex.argtypes = [vp] * 7 + [i] * 8 + [f, u, vp]
        L.skiparse_quantize_fp8.restype = i
        L.skiparse_quantize_fp8.argtypes = [vp, vp, vp] + [i] * 8 + [vp]
        L.skiparse_attn_fwd_fp8.restype = i
        L.skiparse_attn_fwd_fp8.argtypes = [vp] * 7 + [i] * 8 + [f, vp]
        L.skiparse_strerror.restype = ctypes.c_char_p
        L.skiparse_strerror.argtypes = [i]
        L.skiparse_last_hip_error.restype = i
        L.skiparse_last_hip_error.argtypes = []
        L.skiparse_rope_table_bytes.restype = sz
        L.skiparse_rope_table_bytes.argtypes = [i] * 6
        L.skiparse_rope_table.restype = i
        L.skiparse_rope_table.argtypes = [vp] + [i] * 6 + [f, i] + [f] * 3 + [i] * 3 + [f] * 3 + [vp]
        L.skiparse_rope_table_ex.restype = i
        L.skiparse_rope_table_ex.argtypes = [vp] + [i] * 6 + [d, i] + [d] * 3 + [i] * 3 + [d] * 3 + [vp]
        L.skiparse_rope.restype = i
        L.skiparse_rope.argtypes = [vp] * 5 + [i] * 21 + [vp]
        L.skiparse_checkpoint_save.restype = i
        L.skiparse_checkpoint_save.argtypes = [vp] * 3 + [i] * 3 + [vp]
        L.skiparse_checkpoint_load.restype = i
        L.skiparse_checkpoint_load.argtypes = [vp] * 3 + [i] * 3 + [vp]
        L.skiparse_linear_workspace_bytes.restype = sz
        L.skiparse_linear_workspace_bytes.argtypes = [i] * 3
        L.skiparse_linear_fwd.restype = i
        L.skiparse_linear_fwd.argtypes = [vp] * 7 + [i] * 11 + [vp, sz, vp]
        L.skiparse_linear_bwd_workspace_bytes.restype = sz
        L.skiparse_linear_bwd_workspace_bytes.argtypes = [i] * 6
        L.skiparse_linear_bwd.restype = i
        L.skiparse_linear_bwd.argtypes = [vp] * 10 + [i] * 11 + [vp, sz, vp]
        L.skiparse_rmsnorm_fwd.restype = i
        L.skiparse_rmsnorm_fwd.argtypes = [vp] * 6 + [i] * 5 + [f] + [i] * 4 + [vp]
        L.skiparse_rmsnorm_bwd_workspace_bytes.restype = sz
        L.skiparse_rmsnorm_bwd_workspace_bytes.argtypes = [i] * 2
        L.skiparse_rmsnorm_bwd.restype = i
        L.skiparse_rmsnorm_bwd.argtypes = [vp] * 6 + [i] * 5 + [f] + [i] * 4 + [vp, sz, vp]
        L.skiparse_quantize_int8.restype = i
        L.skiparse_quantize_int8.argtypes = [vp] * 3 + [i] * 9 + [vp]
        L.skiparse_linear_fwd_int8_workspace_bytes.restype = sz
        L.skiparse_linear_fwd_int8_workspace_bytes.argtypes = [i] * 3
        L.skiparse_linear_fwd_int8.restype = i
        L.skiparse_linear_fwd_int8.argtypes = [vp] * 7 + [i] * 10 + [vp, sz, vp]
        _bind(L)
        _lib = L
    return _lib


# A small call is bound by what it costs to issue it, so no Stream object is made for it.  torch hands out the bare handle under private names
# only; where a release has no such names the Stream object serves.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    """Handle of torch's current stream on the current device."""
    if _raw_stream is None or _get_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_get_device())


def _forked() -> None:
    """The bare handle is given out without a look at where: in a forked child torch's public call decides, which refuses the GPU to the
    child of a process that has used it."""
    global _raw_stream
    _raw_stream = None


os.register_at_fork(after_in_child=_forked)


def _dev(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    return t.data_ptr()


def _check(code: int, what: str) -> None:
    if code != 0:
        raise SkiparseError(code, what)


# Where the tensors of a call stand in the C function's arguments, and what they are called when one is refused.
_QKVO = ((0, "q"), (1, "k"), (2, "v"), (3, "out"))
_TENSORS = {
    "skiparse_permute": ((0, "x"), (1, "out")),
    "skiparse_unpermute": ((0, "y"), (1, "out")),
    "skiparse_switch_pattern": ((0, "y"), (1, "out")),
    "skiparse_ssp_pack": ((0, "x"), (1, "out")),
    "skiparse_ssp_unpack": ((0, "recv"), (1, "out")),
    "dense_attn_fwd": _QKVO,
    "skiparse_attn_fwd": (*_QKVO, (15, "workspace")),
    "skiparse_attn_fwd_sparse": _QKVO,
    "skiparse_attn_fwd_lse": (*_QKVO, (4, "lse")),
    "skiparse_attn_bwd": (*_QKVO, (4, "dout"), (5, "lse"), (6, "dq"), (7, "dk"), (8, "dv"), (20, "workspace")),
    "skiparse_attn_bwd_static": (*_QKVO, (4, "dout"), (5, "lse"), (6, "dq"), (7, "dk"), (8, "dv")),
    "skiparse_quantize_fp8_ex": ((0, "x"), (1, "x8"), (2, "scales")),
    "skiparse_attn_fwd_fp8_ex": ((0, "q8"), (1, "k8"), (2, "v8"), (3, "sq"), (4, "sk"), (5, "sv"), (6, "out")),
    "skiparse_rope_table_ex": ((0, "table"),),
    "skiparse_rope": ((0, "q"), (1, "k"), (2, "q_out"), (3, "k_out"), (4, "table")),
    "skiparse_checkpoint_save": ((0, "x"), (1, "codes"), (2, "scales")),
    "skiparse_checkpoint_load": ((0, "codes"), (1, "scales"), (2, "out")),
    "skiparse_linear_fwd": ((0, "x"), (1, "w"), (2, "bias"), (3, "residual"), (4, "out"), (5, "pre"), (6, "pre_scales"), (18, "workspace")),
    "skiparse_linear_bwd": ((0, "dy"), (1, "x"), (2, "x_scales"), (3, "w"), (4, "pre"), (5, "pre_scales"), (6, "dx_add"), (7, "dx"), (8, "dw"), (9, "db"),
                            (21, "workspace")),
    "skiparse_rmsnorm_fwd": ((0, "x"), (1, "residual"), (2, "weight"), (3, "total"), (4, "out"), (5, "scales")),
    "skiparse_rmsnorm_bwd": ((0, "dy"), (1, "h"), (2, "weight"), (3, "dx_add"), (4, "dx"), (5, "dw"), (16, "workspace")),
    "skiparse_quantize_int8": ((0, "x"), (1, "codes"), (2, "scales")),
    "skiparse_linear_fwd_int8": ((0, "x"), (1, "x's scales"), (2, "w"), (3, "w's scales"), (4, "bias"), (5, "residual"), (6, "out"), (17, "workspace")),
}
# Those that a call can do without.
_OPTIONAL = {
    "skiparse_attn_fwd": {15},  # the fused form needs no workspace
    "skiparse_rope": {1, 3},
    "skiparse_linear_fwd": {2, 3, 5, 6, 18},
    "skiparse_linear_bwd": {1, 2, 3, 4, 5, 6, 7, 8, 9, 21},
    "skiparse_rmsnorm_fwd": {1, 2, 3, 5},
    "skiparse_rmsnorm_bwd": {2, 3, 4, 5, 16},
    "skiparse_linear_fwd_int8": {4, 5, 17},
}


# What an integer argument holds.  ctypes cuts a larger one to it without a word, so that 2^32 + 1 rows would be one row.
_RANGES = {ctypes.c_int: (-(1 << 31), 1 << 31), ctypes.c_uint: (0, 1 << 32), ctypes.c_size_t: (0, 1 << 64)}


def _fit(name: str, types, args) -> None:
    for i, (t, a) in enumerate(zip(types, args)):
        if t in _RANGES:
            try:
                n = operator.index(a)
            except TypeError:  # no integer: the call says so
                continue
            if not _RANGES[t][0] <= n < _RANGES[t][1]:
                raise ValueError(f"{name}: argument {i}, {n}, does not fit the {8 * ctypes.sizeof(t)} bits that the library has for it")


def _size(name: str, *sizes) -> int:
    """A number of bytes that the library computes."""
    f = getattr(lib(), name)
    _fit(name, f.argtypes, sizes)
    return int(f(*sizes))


def _failed(code: int, name: str) -> None:
    _check(code, name.removesuffix("_ex"))


def _general(name: str, *args) -> None:
    """The call by way of ctypes, which takes every integer-like argument and names what it refuses."""
    f = getattr(lib(), name)
    if len(args) != len(f.argtypes):  # ctypes would pass on what is too many
        raise TypeError(f"{name} takes {len(f.argtypes)} arguments, not {len(args)}")
    _fit(name, f.argtypes, args)
    args = list(args)
    for i, what in _TENSORS[name]:
        if not (args[i] is None and i in _OPTIONAL.get(name, ())):
            args[i] = _dev(args[i], what)
    _failed(f(*args), name)


# The entry points themselves: by ctypes until the library is opened, then natively marshalled where there is a module for this Python and
# this torch.  The module is imported then and not with the package, so that a process that builds first gets what it has built.
for _name in _TENSORS:
    globals()["_" + _name] = functools.partial(_general, _name)


# Calls as a whole, natively: they answer NotImplemented to all but plain arguments, and before the module is there.
_PLAIN = ("rmsnorm_fwd", "rmsnorm_bwd", "quantize_int8", "linear_fwd_int8")
_PLAIN_SIZES = ("skiparse_rmsnorm_bwd_workspace_bytes", "skiparse_linear_fwd_int8_workspace_bytes")


def _not_plain(*args):
    return NotImplemented


for _name in _PLAIN:
    globals()["_plain_" + _name] = _not_plain


def _torch_build() -> str:
    """Which torch this is: the module reads tensors by the layout in the headers that it was built with."""
    return f"{torch.__version__} {torch.version.git_version}"


def _bind(L: ctypes.CDLL) -> None:
    """Looks for the module, and hands it the functions of the library that has been opened."""
    global _marshal
    try:
        native = importlib.import_module(__name__ + "._marshal")
    except ImportError:
        native = None
    if native is not None and getattr(native, "BUILT_FOR", None) != _torch_build():
        native = None
    if native is not None:
        native.set_up(_general, _failed)
        for name in _TENSORS:
            native.bind(name, ctypes.cast(getattr(L, name), ctypes.c_void_p).value)
            globals()["_" + name] = getattr(native, name)
        for name in _PLAIN_SIZES:
            native.bind(name, ctypes.cast(getattr(L, name), ctypes.c_void_p).value)
        for name in _PLAIN:
            globals()["_plain_" + name] = getattr(native, "plain_" + name)
    _marshal = native


def __getattr__(name: str):
    if name == "_marshal":  # the native module, or None: known once the library is open
        lib()
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def _dims(x: torch.Tensor, T: int, H: int, W: int):
    B, N, heads, D = x.shape
    if N != T * H * W:
        raise ValueError("token axis does not match T*H*W")
    return B, heads, D


def skiparse_permute(x: torch.Tensor, T: int, H: int, W: int, s: int, pattern: str, out: torch.Tensor | None = None):
    """[B][N][heads][D] -> [s*s*B][N/s^2][heads][D] (original -> sparse layout), bit-exact row gather."""
    B, heads, D = _dims(x, T, H, W)
    if out is None:
        out = torch.empty((s * s * B, (T * H * W) // (s * s), heads, D), dtype=x.dtype, device=x.device)
    _skiparse_permute(x, out, B, heads, T, H, W, D, s, PATTERNS[pattern], _DTYPES[x.dtype], _stream())
    return out


def skiparse_unpermute(y: torch.Tensor, T: int, H: int, W: int, s: int, pattern: str, out: torch.Tensor | None = None):
    """[s*s*B][N/s^2][heads][D] -> [B][N][heads][D] (sparse -> original layout)."""
    SB, Nsub, heads, D = y.shape
    B = SB // (s * s)
    if SB != B * s * s or Nsub * s * s != T * H * W:
        raise ValueError("sparse-layout shape does not match the grid")
    if out is None:
        out = torch.empty((B, T * H * W, heads, D), dtype=y.dtype, device=y.device)
    _skiparse_unpermute(y, out, B, heads, T, H, W, D, s, PATTERNS[pattern], _DTYPES[y.dtype], _stream())
    return out


def skiparse_switch_pattern(y: torch.Tensor, T: int, H: int, W: int, s: int, from_pattern: str, out: torch.Tensor | None = None):
    """Sparse layout of `from_pattern` -> sparse layout of the other pattern, one row move per token."""
    SB, Nsub, heads, D = y.shape
    B = SB // (s * s)
    if SB != B * s * s or Nsub * s * s != T * H * W:
        raise ValueError("sparse-layout shape does not match the grid")
    if out is None:
        out = torch.empty_like(y)
    _skiparse_switch_pattern(y, out, B, heads, T, H, W, D, s, PATTERNS[from_pattern], _DTYPES[y.dtype], _stream())
    return out


def skiparse_ssp_pack(x: torch.Tensor, T: int, H: int, W: int, s: int, group_size: int, out: torch.Tensor | None = None):
    """One rank's shard [G*b][T*(H/s)*(W/s)][heads][D] (G = s*s/group_size subsequences, batch fastest) -> the all-to-all send buffer
    [group_size][G][G*b][T*(H/s^2)*(W/s^2)][heads][D] of Sparse Sequence Parallelism (chunk r is for rank r)."""
    Bl, n_local, heads, D = x.shape
    G = (s * s) // group_size
    if G < 1 or G * group_size != s * s or Bl % G or n_local * s * s != T * H * W:
        raise ValueError("shard shape does not match the grid and the group")
    if out is None:
        out = torch.empty((group_size, G, Bl, n_local // (s * s), heads, D), dtype=x.dtype, device=x.device)
    _skiparse_ssp_pack(x, out, Bl // G, heads, T, H, W, D, s, group_size, _DTYPES[x.dtype], _stream())
    return out


def skiparse_ssp_unpack(recv: torch.Tensor, T: int, H: int, W: int, s: int, group_size: int, out: torch.Tensor | None = None):
    """The all-to-all receive buffer [group_size][G][G*b][base][heads][D] (chunk r came from rank r) -> the rank's shard
    [G*b][T*(H/s)*(W/s)][heads][D] in the other pattern's sparse layout."""
    gs, G, Bl, base, heads, D = recv.shape
    if gs != group_size or G * group_size != s * s or Bl % G or base * s * s * s * s != T * H * W:
        raise ValueError("receive-buffer shape does not match the grid and the group")
    if out is None:
        out = torch.empty((Bl, base * s * s, heads, D), dtype=recv.dtype, device=recv.device)
    _skiparse_ssp_unpack(recv, out, Bl // G, heads, T, H, W, D, s, group_size, _DTYPES[recv.dtype], _stream())
    return out


def dense_attn_fwd(q, k, v, T: int, H: int, W: int, scale: float = 0.0, out: torch.Tensor | None = None):
    """softmax(q k^T * scale) v over all T*H*W tokens for every (batch, head); bf16 in, bf16 out."""
    B, heads, D = _dims(q, T, H, W)
    if out is None:
        out = torch.empty_like(q)
    _dense_attn_fwd(q, k, v, out, B, heads, T, H, W, D, float(scale), _DTYPES[q.dtype], _stream())
    return out


def skiparse_workspace_bytes(B, heads, T, H, W, D, s, fused: bool) -> int:
    return _size("skiparse_workspace_bytes", B, heads, T, H, W, D, s, BF16, FUSED if fused else 0)


def skiparse_attn_fwd(q, k, v, T: int, H: int, W: int, s: int, pattern: str, scale: float = 0.0, fused: bool = True,
                      out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, pad: bool = False):
    """Skiparse-2D attention, q/k/v/out in the original layout.  The unfused path needs a uint8 device workspace of
    skiparse_workspace_bytes() bytes; one is allocated with torch if none is passed.  pad=True selects the any-resolution
    mode (fused only): H and W arbitrary, end padding to multiples of s*s masked."""
    B, heads, D = _dims(q, T, H, W)
    if out is None:
        out = torch.empty_like(q)
    ws_bytes = 0
    if fused:
        workspace = None
    else:
        need = skiparse_workspace_bytes(B, heads, T, H, W, D, s, False)
        if workspace is None:
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)
        ws_bytes = workspace.numel() * workspace.element_size()
    _skiparse_attn_fwd(q, k, v, out, B, heads, T, H, W, D, s, PATTERNS[pattern], float(scale), _DTYPES[q.dtype],
                       (FUSED if fused else 0) | (PAD if pad else 0), workspace, ws_bytes, _stream())
    return out


def skiparse_attn_fwd_sparse(q, k, v, T: int, H: int, W: int, s: int, pattern: str, out_layout: str = "other", scale: float = 0.0,
                             out: torch.Tensor | None = None):
    """Attention on tensors already in the sparse layout of `pattern` ([s*s*B][N/s^2][heads][D]); the output goes to the
    same layout ("same"), the other pattern's sparse layout ("other") or the original layout ("original")."""
    SB, Nsub, heads, D = q.shape
    B = SB // (s * s)
    if SB != B * s * s or Nsub * s * s != T * H * W:
        raise ValueError("sparse-layout shape does not match the grid")
    if out is None:
        shape = (B, T * H * W, heads, D) if out_layout == "original" else tuple(q.shape)
        out = torch.empty(shape, dtype=q.dtype, device=q.device)
    _skiparse_attn_fwd_sparse(q, k, v, out, B, heads, T, H, W, D, s, PATTERNS[pattern], OUT_LAYOUTS[out_layout], float(scale),
                              _DTYPES[q.dtype], _stream())
    return out


_INTS = (int,) * 9


@functools.lru_cache(maxsize=256)
def _bytes_of_ints(name: str, *sizes: int) -> int:
    return _size(name, *sizes)


def _bytes(name: str, *sizes) -> int:
    """A size that the library computes from (B, heads, T, H, W, D, s, pattern, flags).  Remembered for plain integers only: they are their
    own value, while a one-element tensor is looked up by identity and may change, and 8.0, which the call refuses, is found under 8."""
    if tuple(map(type, sizes)) == _INTS:
        return _bytes_of_ints(name, *sizes)
    return _size(name, *sizes)


def skiparse_lse_shape(B, heads, T, H, W, D, s, pattern: str, pad: bool = False):
    """Shape of the log-sum-exp tensor: [s*s*B][heads][positions per subsequence] (positions of the padded grid with pad=True)."""
    n = _bytes("skiparse_lse_bytes", B, heads, T, H, W, D, s, PATTERNS[pattern], PAD if pad else 0) // 4
    if n == 0:
        raise ValueError("grid does not fit the pattern (use pad=True for the any-resolution mode)")
    return (s * s * B, heads, n // (s * s * B * heads))


def skiparse_attn_fwd_lse(q, k, v, T: int, H: int, W: int, s: int, pattern: str, scale: float = 0.0,
                          out: torch.Tensor | None = None, lse: torch.Tensor | None = None, pad: bool = False):
    """Fused forward that also returns the log-sum-exp the backward pass needs: (out, lse), lse float32 in subsequence order."""
    B, heads, D = _dims(q, T, H, W)
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty(skiparse_lse_shape(B, heads, T, H, W, D, s, pattern, pad), dtype=torch.float32, device=q.device)
    _skiparse_attn_fwd_lse(q, k, v, out, lse, B, heads, T, H, W, D, s, PATTERNS[pattern], float(scale), _DTYPES[q.dtype], PAD if pad else 0,
                           _stream())
    return out, lse


def skiparse_bwd_workspace_bytes(B, heads, T, H, W, D, s, pattern: str, pad: bool = False) -> int:
    """Bytes that skiparse_attn_bwd cannot do without."""
    return _bytes("skiparse_bwd_workspace_bytes", B, heads, T, H, W, D, s, PATTERNS[pattern], PAD if pad else 0)


def skiparse_bwd_walk_workspace_bytes(B, heads, T, H, W, D, s, pattern: str, pad: bool = False) -> int:
    """Bytes with which skiparse_attn_bwd is fastest: more than the least for large problems at head_dim 128."""
    return _bytes("skiparse_bwd_walk_workspace_bytes", B, heads, T, H, W, D, s, PATTERNS[pattern], PAD if pad else 0)


def _bwd_workspace(device, *call) -> torch.Tensor:
    """For the fastest kernels (1.7 GB at 160 units of 20,160 positions), or where that is not to be had for the others (13 MB there)."""
    least, walk = skiparse_bwd_workspace_bytes(*call), skiparse_bwd_walk_workspace_bytes(*call)
    if walk > least:
        try:
            return torch.empty(walk, dtype=torch.uint8, device=device)
        except torch.cuda.OutOfMemoryError:
            pass
    return torch.empty(max(least, 1), dtype=torch.uint8, device=device)


def skiparse_attn_bwd(q, k, v, out, dout, lse, T: int, H: int, W: int, s: int, pattern: str, scale: float = 0.0,
                      dq=None, dk=None, dv=None, workspace: torch.Tensor | None = None, pad: bool = False):
    """Gradients (dq, dk, dv) of the Skiparse attention layer; out and lse come from skiparse_attn_fwd_lse (same pad flag).  A
    uint8 device workspace of skiparse_bwd_walk_workspace_bytes() bytes is allocated with torch if none is passed; a smaller one, down to
    skiparse_bwd_workspace_bytes(), selects kernels that need no more (slower on large problems at head_dim 128), as does a device that
    has no room for it.  The two round differently: pass a workspace where every call has to give the same bits."""
    B, heads, D = _dims(q, T, H, W)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    if workspace is None:
        workspace = _bwd_workspace(q.device, B, heads, T, H, W, D, s, pattern, pad)
    _skiparse_attn_bwd(q, k, v, out, dout, lse, dq, dk, dv, B, heads, T, H, W, D, s, PATTERNS[pattern], float(scale), _DTYPES[q.dtype],
                       PAD if pad else 0, workspace, workspace.numel() * workspace.element_size(), _stream())
    return dq, dk, dv


def skiparse_attn_bwd_static(q, k, v, out, dout, lse, dq, dk, dv, T: int, H: int, W: int, s: int, pattern: str, scale: float = 0.0,
                             pad: bool = False):
    """skiparse_attn_bwd for callers that cannot allocate: the delta workspace is the library's static device array, and this
    wrapper allocates nothing either (dq, dk, dv must be passed).  Results are those of skiparse_attn_bwd with a workspace of
    skiparse_bwd_workspace_bytes() bytes; problems that need more than the array's size raise (code -4)."""
    B, heads, D = _dims(q, T, H, W)
    _skiparse_attn_bwd_static(q, k, v, out, dout, lse, dq, dk, dv, B, heads, T, H, W, D, s, PATTERNS[pattern], float(scale),
                              _DTYPES[q.dtype], PAD if pad else 0, _stream())
    return dq, dk, dv


def skiparse_quantize_fp8(x: torch.Tensor, T: int, H: int, W: int, s: int, pattern: str, pad: bool = False):
    """bf16 [B][N][heads][D] (original layout) -> (uint8 E4M3 codes [s*s*B][positions][heads][D] in the sparse layout,
    float32 scales [s*s*B][heads][ceil(positions/128)]).  positions = N/s^2, or with pad=True (any-resolution mode) the positions
    of the grid padded to multiples of s*s, with zero codes at the padding."""
    B, heads, D = _dims(x, T, H, W)
    if x.dtype != torch.bfloat16:
        raise ValueError("skiparse_quantize_fp8 takes bf16 input")
    nsub = skiparse_lse_shape(B, heads, T, H, W, D, s, pattern, pad)[2]
    x8 = torch.empty((s * s * B, nsub, heads, D), dtype=torch.uint8, device=x.device)
    scales = torch.empty((s * s * B, heads, (nsub + 127) // 128), dtype=torch.float32, device=x.device)
    _skiparse_quantize_fp8_ex(x, x8, scales, B, heads, T, H, W, D, s, PATTERNS[pattern], PAD if pad else 0, _stream())
    return x8, scales


def skiparse_attn_fwd_fp8(q8, k8, v8, sq, sk, sv, T: int, H: int, W: int, s: int, pattern: str, scale: float = 0.0,
                          out: torch.Tensor | None = None, pad: bool = False):
    """Attention on quantised sparse-layout tensors (from skiparse_quantize_fp8, same pad flag); bf16 output [B][N][heads][D] in the
    original layout."""
    SB, nsub, heads, D = q8.shape
    B = SB // (s * s)
    if SB != B * s * s or (not pad and nsub * s * s != T * H * W):
        raise ValueError("sparse-layout shape does not match the grid")
    if out is None:
        out = torch.empty((B, T * H * W, heads, D), dtype=torch.bfloat16, device=q8.device)
    _skiparse_attn_fwd_fp8_ex(q8, k8, v8, sq, sk, sv, out, B, heads, T, H, W, D, s, PATTERNS[pattern], float(scale), PAD if pad else 0,
                              _stream())
    return out


def _here(*tensors) -> None:
    """Calls go to the current device's stream: a tensor of another device is refused.  (One on the CPU is refused where its address is asked for.)"""
    device = torch.cuda.current_device() if _get_device is None else _get_device()
    for t in tensors:
        if t is not None and (at := t.get_device()) != device and at != -1:
            raise ValueError(f"tensor on {t.device}, but the current device is {device}")


def _triple(x):
    return tuple(x) if isinstance(x, (tuple, list)) else (x, x, x)


class RopeTable(NamedTuple):
    """Cosines and sines of the places along the axes of a grid: `data` float32, for every axis [places][pairs][2], one after the other."""

    data: torch.Tensor
    lengths: tuple  # places of t, h, w
    axes: tuple     # turned channels of a head that belong to t, h, w


def skiparse_rope_table(lengths, axes, theta: float = 10000.0, scaling: str = "none", factor=1.0, trained=0, fast: float = 32.0, slow: float = 1.0,
                        attention: float = 1.0, device="cuda", out: torch.Tensor | None = None) -> RopeTable:
    """Table for skiparse_rope: `lengths` places along t, h, w, `axes` channels of a head that turn with each.  scaling "linear", "ntk" or "yarn" by `factor`
    (one number, or one an axis) for contexts longer than the `trained` places (yarn); `attention` multiplies cosines and sines."""
    (T, H, W), (rt, rh, rw) = lengths, axes
    if out is None:
        n = _table_bytes(T, H, W, rt, rh, rw) // 4
        out = torch.empty(n, dtype=torch.float32, device=device)
    elif out.dtype != torch.float32 or out.numel() * 4 != _table_bytes(T, H, W, rt, rh, rw):
        raise ValueError("out must be float32 and of the table's size")
    _here(out)
    ft, fh, fw = _triple(factor)
    nt, nh, nw = _triple(trained)
    _skiparse_rope_table_ex(out, T, H, W, rt, rh, rw, float(theta), ROPE_SCALINGS[scaling], float(ft), float(fh), float(fw), nt, nh, nw, float(fast),
                            float(slow), float(attention), _stream())
    return RopeTable(out, (T, H, W), (rt, rh, rw))


def _table_bytes(T, H, W, rt, rh, rw) -> int:
    n = _size("skiparse_rope_table_bytes", T, H, W, rt, rh, rw)
    if n == 0:
        raise ValueError("lengths are positive, channels even, and a table has less than 2^31 pairs")
    return n


def skiparse_rope(q: torch.Tensor, k: torch.Tensor | None, table: RopeTable, T: int, H: int, W: int, s: int = 1, pattern: str = "token", order: str = "same",
                  layout: str = "interleaved", inverse: bool = False, at=(0, 0, 0), q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
    """Turns the first channels of every head of q and k by their tokens' places: (q', k'), k' None without a k.  q, k: [B][T*H*W][heads][D], or
    [s*s*B][T*H*W/(s*s)][heads][D] for order "to_original" and "stay_sparse"; `at`: the table's place of the grid's first token along t, h, w.  inverse=True is the
    gradient.  Where rows keep their places, q_out=q and k_out=k turn in place."""
    B, n_in, heads, D = q.shape
    n, s2 = T * H * W, s * s
    sparse_in = order == "to_original" or order == "stay_sparse"
    rows = B * n_in
    if n < 1 or s < 1 or rows % n or (n_in * s2 if sparse_in else n_in) != n:
        raise ValueError("token axis does not match the grid")
    B = rows // n
    if k is not None and (k.shape != q.shape or k.dtype != q.dtype):
        raise ValueError("q and k differ in shape or type")
    data, (lt, lh, lw), (rt, rh, rw) = table
    t0, h0, w0 = at
    if data.dtype != torch.float32 or data.numel() != 2 * (lt * (rt // 2) + lh * (rh // 2) + lw * (rw // 2)):
        raise ValueError("the table is float32 and as long as its lengths and axes say")
    shape = (s2 * B, n // s2, heads, D) if order == "to_sparse" else (B, n, heads, D) if order == "to_original" else q.shape
    q_out = _into(q_out, shape, q)
    k_out = None if k is None else _into(k_out, shape, q)
    _here(q, k, q_out, k_out, data)
    _skiparse_rope(q, k, q_out, k_out, data, B, heads, T, H, W, D, rt, rh, rw, lt, lh, lw, t0, h0, w0, s, PATTERNS[pattern], ORDERS[order],
                   ROPE_LAYOUTS[layout], 1 if inverse else 0, _DTYPES[q.dtype], _stream())
    return q_out, k_out


def _into(out, shape, like, dtype=None):
    """`out`, or a new tensor of that shape; one that is passed has to have it.  (empty_like takes 1.2 us, new_empty 1.9, empty 2.4.  A `like` that is not contiguous is refused by the call.)"""
    if out is None:
        if dtype is not None and dtype != like.dtype:
            return like.new_empty(shape, dtype=dtype)
        return torch.empty_like(like) if shape == like.shape else like.new_empty(shape)
    dtype = dtype or like.dtype
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype:
        raise ValueError(f"an output of shape {tuple(shape)} and type {dtype} is needed")
    return out


class Checkpoint(NamedTuple):
    """An activation in 8 bits: E4M3 codes (uint8) of its shape, and one exponent byte for 32 channels of a row."""

    codes: torch.Tensor
    scales: torch.Tensor


def _checkpoint_of(shape, like) -> Checkpoint:
    return Checkpoint(like.new_empty(shape, dtype=torch.uint8), like.new_empty((*shape[:-1], (shape[-1] + 31) // 32), dtype=torch.uint8))


def _checked(c: Checkpoint, shape, what: str) -> Checkpoint:
    if c.codes.dtype != torch.uint8 or c.scales.dtype != torch.uint8 or tuple(c.codes.shape) != tuple(shape) or tuple(c.scales.shape) != (*shape[:-1], (shape[-1] + 31) // 32):
        raise ValueError(f"{what}: not a checkpoint of shape {tuple(shape)}")
    return c


def skiparse_checkpoint_save(x: torch.Tensor, out: Checkpoint | None = None) -> Checkpoint:
    """[..., channels] in bf16 or float32 -> its 8-bit checkpoint, in a little over half the bytes of bf16."""
    out = _checkpoint_of(x.shape, x) if out is None else _checked(out, x.shape, "out")
    _here(x, *out)
    cols = x.shape[-1]
    _skiparse_checkpoint_save(x, out.codes, out.scales, x.numel() // max(cols, 1), cols, _DTYPES[x.dtype], _stream())
    return out


def skiparse_checkpoint_load(c: Checkpoint, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that a checkpoint stands for."""
    _checked(c, c.codes.shape, "checkpoint")
    out = _into(out, c.codes.shape, c.codes, dtype)
    _here(out, *c)
    cols = out.shape[-1]
    _skiparse_checkpoint_load(c.codes, c.scales, out, out.numel() // max(cols, 1), cols, _DTYPES[out.dtype], _stream())
    return out


def _linear_rows(lead, order: str, T: int, H: int, W: int, s: int):
    """(B, T, H, W) of the rows, and the leading dimensions of the other side of `order`; `lead`: the leading dimensions of the side that rows come from."""
    rows = 1
    for d in lead:
        rows *= d
    if order == "same":
        return (1, 1, 1, rows), lead
    n, s2 = T * H * W, s * s
    if n < 1 or s < 1 or rows % n or n % s2 or len(lead) != 2 or lead[1] != (n if order == "to_sparse" else n // s2):
        raise ValueError("token axis does not match the grid")
    B = rows // n
    return (B, T, H, W), (s2 * B, n // s2) if order == "to_sparse" else (B, n)


_BACK = {"same": "same", "to_sparse": "to_original", "to_original": "to_sparse"}


def _bf16(what: str, *tensors) -> None:
    for t in tensors:
        if t is not None and t.dtype != torch.bfloat16:
            raise ValueError(f"{what} must be bfloat16")


def skiparse_linear_fwd(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, residual: torch.Tensor | None = None, act: str = "none",
                        order: str = "same", T: int = 0, H: int = 0, W: int = 0, s: int = 1, pattern: str = "token", keep: str | None = None,
                        out: torch.Tensor | None = None, pre=None, workspace: torch.Tensor | None = None):
    """act(x w^T + bias) + residual, bf16: x [..., in], w [out, in], bias [out], residual and result [..., out].  order "to_sparse" or "to_original" moves the rows
    of the grid T x H x W on the way: x then is [B][T*H*W][in] or [s*s*B][T*H*W/(s*s)][in], result and residual the other.  keep="bf16" or "checkpoint"
    returns (result, values in front of the activation) for the backward pass; `out`, `pre` (what keep returns) and `workspace` are buffers to use."""
    K, (N, Kw) = x.shape[-1], w.shape
    if K != Kw or (bias is not None and tuple(bias.shape) != (N,)):
        raise ValueError("x, w and bias do not fit each other")
    _bf16("x, w, bias and residual", x, w, bias, residual)
    grid, lead = _linear_rows(x.shape[:-1], order, T, H, W, s)
    shape = (*lead, N)
    out = _into(out, shape, x)
    if residual is not None and tuple(residual.shape) != shape:
        raise ValueError(f"residual must have the result's shape {shape}")
    if keep not in (None, "bf16", "checkpoint") or (keep is None and pre is not None):
        raise ValueError('keep is None, "bf16" or "checkpoint"')
    codes = scales = None
    if keep == "bf16":
        codes = pre = _into(pre, shape, x)
    elif keep == "checkpoint":
        codes, scales = pre = _checkpoint_of(shape, x) if pre is None else _checked(pre, shape, "pre")
    _here(x, w, bias, residual, out, codes, scales, workspace)
    M = grid[0] * grid[1] * grid[2] * grid[3]
    workspace, size = _space(workspace, x, "skiparse_linear_workspace_bytes", M, K, N)
    _skiparse_linear_fwd(x, w, bias, residual, out, codes, scales, *grid, K, N, s, PATTERNS[pattern], ORDERS[order], ACTS[act], BF16, workspace, size, _stream())
    return out if keep is None else (out, pre)


@functools.lru_cache(maxsize=256)
def _space_bytes(name: str, *sizes: int) -> int:
    return _size(name, *sizes)


def _space(workspace, like, name: str, *sizes):
    """The workspace of a call and its size: the one that is passed, a new one, or none where none is needed."""
    if workspace is not None:
        return workspace, workspace.numel() * workspace.element_size()
    n = _space_bytes(name, *sizes)
    return (like.new_empty(n, dtype=torch.uint8), n) if n else (None, 0)


def skiparse_linear_workspace_bytes(rows: int, in_features: int, out_features: int) -> int:
    return _size("skiparse_linear_workspace_bytes", rows, in_features, out_features)


def skiparse_linear_bwd_workspace_bytes(rows: int, in_features: int, out_features: int, order: str = "same", act: str = "none", x_checkpoint: bool = False) -> int:
    return _size("skiparse_linear_bwd_workspace_bytes", rows, in_features, out_features, ORDERS[order], ACTS[act], 1 if x_checkpoint else 0)


def skiparse_linear_bwd(dy: torch.Tensor, x, w: torch.Tensor | None, pre=None, act: str = "none", order: str = "same", T: int = 0, H: int = 0, W: int = 0, s: int = 1,
                        pattern: str = "token", need_dx: bool = True, need_dw: bool = True, need_db: bool = True, dx_add: torch.Tensor | None = None,
                        dx: torch.Tensor | None = None, dw: torch.Tensor | None = None, db: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """Gradients (dx, dw, db) of skiparse_linear_fwd for dL/dresult = dy; None for one that is not needed.  x: what the forward call had, or its Checkpoint; pre: what
    keep returned, bf16 or a Checkpoint (act "none" needs none).  dx = dz w + dx_add; dx_add may be dx.  The residual's gradient is dy.  x is read for dw, w for dx: None
    will do for one that is not."""
    if (need_dx and w is None) or (need_dw and x is None):
        raise ValueError("dx needs w, and dw x")
    N = dy.shape[-1]
    xc = x.codes if isinstance(x, Checkpoint) else x
    K = w.shape[-1] if w is not None else xc.shape[-1] if xc is not None else 8  # db alone has nothing to do with it
    if (xc is not None and xc.shape[-1] != K) or (w is not None and tuple(w.shape) != (N, K)):
        raise ValueError("dy, x and w do not fit each other")
    if isinstance(x, Checkpoint):
        _checked(x, xc.shape, "x")
    else:
        _bf16("x", x)
    _bf16("dy, w and dx_add", dy, w, dx_add)
    grid, back = _linear_rows(dy.shape[:-1], _BACK[order], T, H, W, s)
    shape = (*back, K)
    if (xc is not None and tuple(xc.shape) != shape) or (dx_add is not None and tuple(dx_add.shape) != shape):
        raise ValueError("dy, x or dx_add does not have its rows")
    codes = scales = None
    if act != "none":
        if pre is None:
            raise ValueError("an activation's gradient needs the values in front of it")
        if isinstance(pre, Checkpoint):
            codes, scales = _checked(pre, dy.shape, "pre")
        else:
            codes = _into(pre, dy.shape, dy)
    dx = _into(dx, shape, dy) if need_dx else None
    dw = _into(dw, (N, K), dy) if need_dw else None
    db = _into(db, (N,), dy) if need_db else None
    xs = x.scales if isinstance(x, Checkpoint) else None
    _here(dy, xc, xs, w, codes, scales, dx_add, dx, dw, db, workspace)
    M = grid[0] * grid[1] * grid[2] * grid[3]
    workspace, size = _space(workspace, dy, "skiparse_linear_bwd_workspace_bytes", M, K, N, ORDERS[order], ACTS[act], 0 if xs is None else 1)
    _skiparse_linear_bwd(dy, xc, xs, w, codes, scales, dx_add, dx, dw, db, *grid, K, N, s, PATTERNS[pattern], ORDERS[order], ACTS[act], BF16, workspace, size, _stream())
    return dx, dw, db


class Quantized(NamedTuple):
    """Rows in 8-bit integers: codes (int8) of the rows' shape, and one float32 scale a row: a value is code * scale."""

    codes: torch.Tensor
    scales: torch.Tensor


def _quantized_of(shape, like) -> Quantized:
    return Quantized(like.new_empty(shape, dtype=torch.int8), like.new_empty(shape[:-1], dtype=torch.float32))


def _is_quantized(q, what: str, shape=None) -> Quantized:
    if not isinstance(q, Quantized):
        raise ValueError(f"{what} must be Quantized")
    codes, scales = q
    at = codes.shape
    if codes.dtype != torch.int8 or scales.dtype != torch.float32 or scales.shape != at[:-1] or (shape is not None and at != shape):
        raise ValueError(f"{what}: not int8 codes{'' if shape is None else f' of shape {tuple(shape)}'} with a float32 scale a row")
    return q


def _from_16(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy where it does not begin at a multiple of 16 bytes, as the scales of a slice of rows.  (What lies in strides is refused as it stands.)"""
    return t if t.data_ptr() % 16 == 0 or not t.is_contiguous() else t.clone()


def _same_type(like, *tensors) -> None:
    dtype = like.dtype
    for t in tensors:
        if t is not None and t.dtype != dtype:
            raise ValueError(f"tensors of one type are needed, {like.dtype} here")


def _of_channels(weight, cols: int) -> None:
    if weight is not None and weight.shape != (cols,):
        raise ValueError(f"weight must have shape ({cols},)")


def skiparse_rmsnorm_fwd(x: torch.Tensor, weight: torch.Tensor | None = None, residual: torch.Tensor | None = None, eps: float = 1e-6, order: str = "same", T: int = 0,
                         H: int = 0, W: int = 0, s: int = 1, pattern: str = "token", quantize: bool = False, out=None, total: torch.Tensor | None = None):
    """h / sqrt(mean(h^2) + eps) * weight over the last dimension, h = x + residual: the result, or with a residual (result, h).  bf16 or float32, all of one type; h is rounded to it, the result made
    of what it is before that.  quantize=True: the result as Quantized, for skiparse_linear_fwd_int8.  order "to_sparse" or "to_original" moves the rows of the grid T x H x W on the way: x, residual and h
    are [B][T*H*W][channels] or [s*s*B][T*H*W/(s*s)][channels], the result the other; h stays where x is.  `out` and `total` (of h; may be residual or x) are buffers to use; out may be x where rows stay."""
    p = PATTERNS[pattern]
    if order == "same":
        place = None
    else:
        grid, lead = _linear_rows(x.shape[:-1], order, T, H, W, s)
        place = (*lead, *grid, s, p, ORDERS[order])
    if out is None and total is None:
        done = _plain_rmsnorm_fwd(x, weight, residual, eps, quantize, Quantized, place, _get_device, _raw_stream)
        if done is not NotImplemented:
            return done
    at = x.shape
    cols = at[-1]
    if place is None:
        grid, shape = (1, 1, 1, x.numel() // max(cols, 1)), at
    else:
        shape = (*lead, cols)
    _of_channels(weight, cols)
    _same_type(x, weight, residual)
    scales = None
    if quantize:
        codes, scales = out = _quantized_of(shape, x) if out is None else _is_quantized(out, "out", shape)
    else:
        codes = out = _into(out, shape, x)
    if residual is not None:
        if residual.shape != at:
            raise ValueError(f"residual must have the shape of x, {tuple(at)}")
        total = _into(total, at, x)
    elif total is not None:
        raise ValueError("without a residual the sum is x")
    _here(x, weight, residual, total, codes, scales)
    _skiparse_rmsnorm_fwd(x, residual, weight, total, codes, scales, *grid, cols, float(eps), s, p, ORDERS[order], _DTYPES[x.dtype], _stream())
    return out if residual is None else (out, total)


def skiparse_rmsnorm_bwd_workspace_bytes(rows: int, cols: int) -> int:
    return _size("skiparse_rmsnorm_bwd_workspace_bytes", rows, cols)


def skiparse_rmsnorm_bwd(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor | None = None, dx_add: torch.Tensor | None = None, eps: float = 1e-6, order: str = "same",
                         T: int = 0, H: int = 0, W: int = 0, s: int = 1, pattern: str = "token", need_dx: bool = True, need_dw: bool = True, dx: torch.Tensor | None = None,
                         dw: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """Gradients (dx, dweight) of skiparse_rmsnorm_fwd for dL/dresult = dy; None for one that is not needed.  h: what the forward call returned beside its result, or its x where it had no residual.
    dx is the gradient of x and of the residual, with dx_add, what comes along the residual stream, added to it; dx_add may be dx."""
    if not (need_dx or need_dw):
        return None, None
    p = PATTERNS[pattern]
    if order == "same" and dx is None and dw is None and workspace is None:
        done = _plain_rmsnorm_bwd(dy, h, weight, dx_add, eps, need_dx, need_dw, _get_device, _raw_stream)
        if done is not NotImplemented:
            return done
    cols = h.shape[-1]
    grid, back = _linear_rows(dy.shape[:-1], _BACK[order], T, H, W, s)
    if dy.shape[-1] != cols or tuple(h.shape) != (*back, cols) or (dx_add is not None and dx_add.shape != h.shape):
        raise ValueError("dy, h or dx_add does not have its shape")
    _of_channels(weight, cols)
    _same_type(h, dy, weight, dx_add)
    dx = _into(dx, h.shape, h) if need_dx else None
    dw = _into(dw, (cols,), h) if need_dw else None
    _here(dy, h, weight, dx_add, dx, dw, workspace)
    size = 0
    if need_dw:
        workspace, size = _space(workspace, h, "skiparse_rmsnorm_bwd_workspace_bytes", grid[0] * grid[1] * grid[2] * grid[3], cols)
    else:
        workspace = None
    _skiparse_rmsnorm_bwd(dy, h, weight, dx_add, dx, dw, *grid, cols, float(eps), s, p, ORDERS[order], _DTYPES[h.dtype], workspace, size, _stream())
    return dx, dw


def skiparse_quantize_int8(x: torch.Tensor, order: str = "same", T: int = 0, H: int = 0, W: int = 0, s: int = 1, pattern: str = "token", out: Quantized | None = None) -> Quantized:
    """[..., channels] in bf16 or float32 -> int8 codes and a float32 scale a row: activations in front of skiparse_linear_fwd_int8, or once its weights [out, in].  order moves rows on the way, as in
    skiparse_rmsnorm_fwd."""
    p = PATTERNS[pattern]
    if order == "same":
        place = None
    else:
        grid, lead = _linear_rows(x.shape[:-1], order, T, H, W, s)
        place = (*lead, *grid, s, p, ORDERS[order])
    if out is None:
        done = _plain_quantize_int8(x, Quantized, place, _get_device, _raw_stream)
        if done is not NotImplemented:
            return done
    shape = x.shape
    cols = shape[-1]
    if place is None:
        grid = (1, 1, 1, x.numel() // max(cols, 1))
    else:
        shape = (*lead, cols)
    codes, scales = out = _quantized_of(shape, x) if out is None else _is_quantized(out, "out", shape)
    _here(x, codes, scales)
    _skiparse_quantize_int8(x, codes, scales, *grid, cols, s, p, ORDERS[order], _DTYPES[x.dtype], _stream())
    return out


def skiparse_linear_fwd_int8_workspace_bytes(rows: int, in_features: int, out_features: int) -> int:
    return _size("skiparse_linear_fwd_int8_workspace_bytes", rows, in_features, out_features)


def skiparse_linear_fwd_int8(x: Quantized, w: Quantized, bias: torch.Tensor | None = None, residual: torch.Tensor | None = None, act: str = "none", order: str = "same", T: int = 0,
                             H: int = 0, W: int = 0, s: int = 1, pattern: str = "token", out: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """act(x w^T + bias) + residual in bf16 from 8-bit integers: x [..., in] and w [out, in] as skiparse_quantize_int8 or skiparse_rmsnorm_fwd leave them, bias [out], residual and result
    [..., out] bf16.  order as in skiparse_linear_fwd; the scales' rows move with the codes'.  A slice of either's rows will do, Quantized(q.codes[3:], q.scales[3:]); scales that begin off a multiple of 16
    bytes are copied first.  `out` (may be residual) and `workspace` are buffers to use."""
    p, a, place = PATTERNS[pattern], ACTS[act], None
    if out is None and workspace is None:
        if order != "same" and type(x) is Quantized:
            grid, lead = _linear_rows(x.codes.shape[:-1], order, T, H, W, s)
            place = (*lead, *grid, s, p, ORDERS[order])
        done = _plain_linear_fwd_int8(x, w, bias, residual, a, Quantized, place, _get_device, _raw_stream)
        if done is not NotImplemented:
            return done
    _is_quantized(x, "x")
    _is_quantized(w, "w")
    xc, xs = x
    wc, ws = w
    if wc.dim() != 2:
        raise ValueError("w is [out, in]")
    at, (N, K) = xc.shape, wc.shape
    if at[-1] != K or (bias is not None and bias.shape != (N,)):
        raise ValueError("x, w and bias do not fit each other")
    _bf16("bias and residual", bias, residual)
    grid, lead = _linear_rows(at[:-1], order, T, H, W, s)
    shape = (*lead, N)
    out = _into(out, shape, xc, torch.bfloat16)
    if residual is not None and residual.shape != shape:
        raise ValueError(f"residual must have the result's shape {shape}")
    _here(xc, xs, wc, ws, bias, residual, out, workspace)
    xs, ws = _from_16(xs), _from_16(ws)
    workspace, size = _space(workspace, xc, "skiparse_linear_fwd_int8_workspace_bytes", grid[0] * grid[1] * grid[2] * grid[3], K, N)
    _skiparse_linear_fwd_int8(xc, xs, wc, ws, bias, residual, out, *grid, K, N, s, p, ORDERS[order], a, workspace, size, _stream())
    return out
