"""ctypes binding of the C ABI in ``include/bcq.h``.

Argument marshalling only: every step of the product runs in the HIP kernels.
The product calls are marshalled by ``_bcq_host`` (``csrc/bcq_host.cpp``) where everything about a call is as it should
be; the Python code below is what makes the other calls, or says what is wrong with them.  It makes all of them, with a warning, where
``_bcq_host`` was not built for the Python and torch that run.
PyTorch supplies device memory and the current stream.  There is no CPU
fallback: if the shared library is missing the import of this module's
functions raises, and every call checks that its tensors live on the GPU.
"""
from __future__ import annotations

import ctypes
import os
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libbcq_hip.so")
_lib = None
_host = None

BCQ_MAX_PLANES = 8
KERNEL_AUTO, KERNEL_SIGN_SELECT, KERNEL_PLANE_MFMA, KERNEL_DEQUANT_MFMA = 0, 1, 2, 3
TYPES = {torch.float16: 0, torch.bfloat16: 1}           # bcq_type
ACTIVATIONS = {"silu": 0, "gelu": 1}                    # bcq_activation
KERNEL_IDS = {"auto": 0, "sign_select": 1, "plane_mfma": 2, "dequant_mfma": 3, "plane_f16": 4, "lut": 5}


class BcqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().bcq_strerror(status).decode()} (status {status})")


class _NoHost:
    """In the place of ``_bcq_host``: declines every call, so that the Python code makes it."""
    gemv = gemv_multi = gemm_mixed = int8_quantize = int8_gemm = int8_gated = staticmethod(lambda *args: None)
    int8_gemm_backward = int8_gated_backward = staticmethod(lambda *args: None)


def _load_host(functions, int8_functions):
    """``_bcq_host``, bound to the library's functions: it holds torch's inline code and so fits one Python and one torch only."""
    try:
        from . import _bcq_host as host
        if host.torch_version != torch.__version__:
            raise ImportError(f"built for torch {host.torch_version}, this is {torch.__version__}")
        if not hasattr(host, "bind_int8"):
            raise ImportError("built before the 8-bit operators")
    except ImportError as e:
        warnings.warn(f"_bcq_host does not load ({e}); calls from Python take about 5 us longer until the package is built again "
                      "(`python paper_2510_10467_amd/build.py`)", RuntimeWarning, stacklevel=3)
        return _NoHost
    host.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in functions), BcqError)
    host.bind_int8(*(ctypes.cast(f, ctypes.c_void_p).value for f in int8_functions))
    return host


def lib() -> ctypes.CDLL:
    """Load ``libbcq_hip.so`` (built in-tree by ``build.py``); fail loudly if absent."""
    global _lib, _host
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(
                f"{_LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
                "or `python paper_2510_10467_amd/build.py`")
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
        L.bcq_strerror.restype = ctypes.c_char_p
        L.bcq_strerror.argtypes = [i32]
        L.bcq_select_kernel.argtypes = [i32]
        L.bcq_select_dequant_shape.argtypes = [i32, i32]
        L.bcq_select_dequant_shape.restype = i32
        L.bcq_last_kernel.restype = ctypes.c_char_p
        L.bcq_dequant_shape_for.argtypes = [i32, i64, i64, i32, i32, i32, vp, vp]
        L.bcq_dequant_shape_for.restype = i32
        L.bcq_mixed_shape_for.argtypes = [i32, i64, i64, i32, i32, i32, vp, vp]
        L.bcq_mixed_shape_for.restype = i32
        L.bcq_level_layout.argtypes = [i32, i32, i64, i32, i32, vp]
        L.bcq_level_layout.restype = i32
        L.bcq_int8_layout.argtypes = [i32, i32, i64, i64, i64, vp]
        L.bcq_int8_layout.restype = i32
        L.bcq_pack.argtypes = [vp, vp, i32, i64, i64, vp]
        L.bcq_unpack.argtypes = [vp, vp, i32, i64, i64, vp]
        L.bcq_gemv.argtypes = [vp, vp, i32, vp, vp, i64, i64, i32, i32, vp]
        L.bcq_gemm_mixed.argtypes = [vp, vp, vp, i32, vp, vp, i64, i64, i32, i32, vp]
        L.bcq_gemv_multi.argtypes = [i32, vp, vp, vp, vp, i32, vp, i64, i32, i32, vp]
        L.bcq_gemv_multi.restype = i32
        L.bcq_gemv_offset.argtypes = [vp, vp, vp, i32, vp, vp, i64, i64, i32, i32, vp]
        L.bcq_gemm_mixed_offset.argtypes = [vp, vp, vp, vp, i32, vp, vp, i64, i64, i32, i32, vp]
        L.bcq_quantize.argtypes = [vp, i32, i32, i32, vp, vp, vp, i64, i64, i32, vp]
        L.bcq_quantize.restype = i32
        L.bcq_quantize_form.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, i64, i64, i32, vp]
        L.bcq_quantize_form.restype = i32
        L.bcq_bench_stream_read.argtypes = [vp, i64, vp, vp]
        L.bcq_bench_stream_read.restype = i32
        L.bcq_bench_fp16_gemv.argtypes = [vp, vp, vp, i64, i64, vp]
        L.bcq_bench_fp16_gemv.restype = i32
        L.bcq_bench_issue_probe.argtypes = [i32, i32, i32, i32, vp, vp, vp]
        L.bcq_bench_issue_probe.restype = i32
        for f in (L.bcq_select_kernel, L.bcq_pack, L.bcq_unpack, L.bcq_gemv, L.bcq_gemm_mixed, L.bcq_gemv_offset,
                  L.bcq_gemm_mixed_offset):
            f.restype = i32
        L.bcq_int8_quantize.argtypes = [vp, i32, vp, vp, i64, i64, vp]
        L.bcq_int8_gemm.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, vp]
        L.bcq_int8_gated.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, i32, i64, i64, i64, vp]
        L.bcq_int8_backward_workspace.argtypes = [i32, i64, i64, i64]
        L.bcq_int8_backward_workspace.restype = i64
        L.bcq_int8_gemm_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i64, i64, i64, vp, i64, vp]
        L.bcq_int8_gated_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, i64, i64, i64, vp, i64, vp]
        for f in (L.bcq_int8_quantize, L.bcq_int8_gemm, L.bcq_int8_gated, L.bcq_int8_gemm_backward, L.bcq_int8_gated_backward):
            f.restype = i32
        _host = _load_host((L.bcq_gemv_offset, L.bcq_gemv_multi, L.bcq_gemm_mixed, L.bcq_gemm_mixed_offset),
                           (L.bcq_int8_quantize, L.bcq_int8_gemm, L.bcq_int8_gated, L.bcq_int8_backward_workspace, L.bcq_int8_gemm_backward,
                            L.bcq_int8_gated_backward))
        _lib = L
    return _lib


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor (there is no CPU path)")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _check(status: int, where: str) -> None:
    if status != 0:
        raise BcqError(status, where)


def select_kernel(variant) -> None:
    """Force a kernel variant by name or id ('auto' restores the default choice)."""
    vid = KERNEL_IDS[variant] if isinstance(variant, str) else int(variant)
    _check(lib().bcq_select_kernel(vid), "bcq_select_kernel")


def select_dequant_shape(request_tiles: int = 0, row_blocks: int = 0) -> None:
    """Benchmarks and tests: force the workgroup shape of the large-batch kernel ((0, 0) = automatic)."""
    _check(lib().bcq_select_dequant_shape(int(request_tiles), int(row_blocks)), "bcq_select_dequant_shape")


def dequant_shape_for(p: int, m: int, n: int, batch: int, group: int = 128, with_offsets: bool = False) -> tuple:
    """Benchmarks and tests: the shape, as ``select_dequant_shape`` takes it, that the large-batch kernel runs such a product with."""
    pair = (ctypes.c_int * 2)()
    _check(lib().bcq_dequant_shape_for(p, m, n, batch, group, int(with_offsets), ctypes.byref(pair, 0), ctypes.byref(pair, 4)),
           "bcq_dequant_shape_for")
    return pair[0], pair[1]


def mixed_shape_for(precisions, m: int, n: int, batch: int, group: int = 128, with_offsets: bool = False) -> tuple:
    """Benchmarks and tests: the shape of the level form that the large-batch kernel runs a call with per-request precision on, the scale sets
    being those of ``precisions``; (0, 0) where its other kernels run it."""
    pair = (ctypes.c_int * 2)()
    _check(lib().bcq_mixed_shape_for(sum(1 << q for q in set(precisions)), m, n, batch, group, int(with_offsets), ctypes.byref(pair, 0),
                                     ctypes.byref(pair, 4)), "bcq_mixed_shape_for")
    return pair[0], pair[1]


def level_layout(p: int, row_blocks: int, n: int, group: int = 128, with_offsets: bool = False) -> dict:
    """Benchmarks and tests: what a workgroup of the level form keeps and asks for on shape ``(1, row_blocks)``."""
    got = (ctypes.c_int * 4)()
    _check(lib().bcq_level_layout(p, row_blocks, n, group, int(with_offsets), got), "bcq_level_layout")
    return dict(zip(("lds_bytes", "window_columns", "window_loads", "word_columns"), got))


def int8_layout(m: int, n: int, tokens: int, matrices: int = 1, backward: bool = False) -> dict:
    """Benchmarks and tests: what the 8-bit products of these sizes run on; ``kernel`` is "rows", "tiles" or "mixed" (tiles of two shapes)."""
    got = (ctypes.c_int * 15)()
    _check(lib().bcq_int8_layout(matrices, int(backward), m, n, tokens, got), "bcq_int8_layout")
    names = ("rows", "tokens", "step", "teams", "ring", "rounds", "lds_bytes")
    layout = dict(zip(names, got[1:8]), kernel=("rows", "tiles", "mixed")[got[0]])
    if backward:
        layout["second"] = dict(zip(("columns", "tokens", "teams", "ring", "rounds", "runs", "lds_bytes"), got[8:]))
    return layout


def last_kernel() -> str:
    return lib().bcq_last_kernel().decode()


def bcq_pack(codes: torch.Tensor, planes: torch.Tensor | None = None) -> torch.Tensor:
    """int8 codes [P][m][n] (>0 is +1) -> int32-typed planes [P][m][n/32] holding the uint32 words."""
    P, m, n = codes.shape
    if planes is None:
        planes = torch.empty((P, m, n // 32), dtype=torch.int32, device=codes.device)
    _check(lib().bcq_pack(_dev(codes, torch.int8, "codes"), _dev(planes, torch.int32, "planes"), P, m, n, _stream()),
           "bcq_pack")
    return planes


def bcq_unpack(planes: torch.Tensor, codes: torch.Tensor | None = None) -> torch.Tensor:
    """planes [P][m][n/32] -> int8 codes [P][m][n] in {-1,+1}."""
    P, m, words = planes.shape
    if codes is None:
        codes = torch.empty((P, m, words * 32), dtype=torch.int8, device=planes.device)
    _check(lib().bcq_unpack(_dev(planes, torch.int32, "planes"), _dev(codes, torch.int8, "codes"), P, m, words * 32,
                            _stream()), "bcq_unpack")
    return codes


def bcq_gemv(planes: torch.Tensor, scales_p: torch.Tensor, p: int, x: torch.Tensor,
             y: torch.Tensor | None = None, group: int = 128, offsets: torch.Tensor | None = None) -> torch.Tensor:
    """Uniform precision: y[b][r] = sum_{i<p} sum_j scales_p[i][r][j/group] * B_i[r][j] * x[b][j];
    with ``offsets`` (float16 [m][n/group], asymmetric scheme) plus sum_j offsets[r][j/group] * x[b][j]."""
    if _host is None:
        lib()
    done = _host.gemv(planes, scales_p, p, x, y, group, offsets)
    if done is not None:
        return done
    _, m, words = planes.shape
    n = words * 32
    batch = x.shape[0]
    if x.shape != (batch, n) or scales_p.shape != (p, m, n // group) or planes.shape[0] < p:
        raise ValueError("bcq_gemv: inconsistent shapes")
    if y is None:
        y = torch.empty((batch, m), dtype=torch.float16, device=x.device)
    elif y.shape != (batch, m):
        raise ValueError("bcq_gemv: y has the wrong shape")
    if offsets is not None:
        if offsets.shape != (m, n // group):
            raise ValueError("bcq_gemv: offsets have the wrong shape")
        _check(lib().bcq_gemv_offset(_dev(planes, torch.int32, "planes"), _dev(scales_p, torch.float16, "scales_p"),
                                     _dev(offsets, torch.float16, "offsets"), p, _dev(x, torch.float16, "x"),
                                     _dev(y, torch.float16, "y"), m, n, batch, group, _stream()), "bcq_gemv_offset")
        return y
    _check(lib().bcq_gemv(_dev(planes, torch.int32, "planes"), _dev(scales_p, torch.float16, "scales_p"), p,
                          _dev(x, torch.float16, "x"), _dev(y, torch.float16, "y"), m, n, batch, group, _stream()),
           "bcq_gemv")
    return y


def bcq_gemv_multi(planes: list, scales_p: list, p: int, x: torch.Tensor, ys: list | None = None, group: int = 128) -> list:
    """Several matrices (same n and precision) applied to the same activations in one call: the q/k/v or
    gate/up projections of a decoder layer.  Returns the list of outputs (those of bcq_gemv within the tolerance both are held
    to; bit for bit wherever the same kernel form serves both)."""
    if ys is None:
        if _host is None:
            lib()
        done = _host.gemv_multi(planes, scales_p, p, x, group)
        if done is not None:
            return done
    count = len(planes)
    batch, n = x.shape
    if len(scales_p) != count or (ys is not None and len(ys) != count):
        raise ValueError("bcq_gemv_multi: lists of different lengths")
    ms = []
    for k in range(count):
        _, m, words = planes[k].shape
        if words * 32 != n or scales_p[k].shape != (p, m, n // group) or planes[k].shape[0] < p:
            raise ValueError(f"bcq_gemv_multi: inconsistent shapes for matrix {k}")
        ms.append(m)
    if ys is None:
        ys = [torch.empty((batch, m), dtype=torch.float16, device=x.device) for m in ms]
    pp = (ctypes.c_void_p * count)(*[_dev(t, torch.int32, f"planes[{k}]") for k, t in enumerate(planes)])
    sp = (ctypes.c_void_p * count)(*[_dev(t, torch.float16, f"scales_p[{k}]") for k, t in enumerate(scales_p)])
    yp = (ctypes.c_void_p * count)(*[_dev(t, torch.float16, f"ys[{k}]") for k, t in enumerate(ys)])
    mp = (ctypes.c_int64 * count)(*ms)
    for k in range(count):
        if ys[k].shape != (batch, ms[k]):
            raise ValueError(f"bcq_gemv_multi: ys[{k}] has the wrong shape")
    _check(lib().bcq_gemv_multi(count, ctypes.cast(pp, ctypes.c_void_p), ctypes.cast(sp, ctypes.c_void_p),
                                ctypes.cast(mp, ctypes.c_void_p), ctypes.cast(yp, ctypes.c_void_p), p,
                                _dev(x, torch.float16, "x"), n, batch, group, _stream()), "bcq_gemv_multi")
    return ys


def bcq_gemm_mixed(planes: torch.Tensor, scales_by_p: dict, p_req: torch.Tensor, x: torch.Tensor,
                   y: torch.Tensor | None = None, group: int = 128, offsets_by_p: dict | None = None) -> torch.Tensor:
    """Per-request precision: request b uses planes 0..p_req[b]-1 and scale set scales_by_p[p_req[b]]
    (and the offset set offsets_by_p[p_req[b]] if there is one)."""
    if _host is None:
        lib()
    done = _host.gemm_mixed(planes, scales_by_p, p_req, x, y, group, offsets_by_p)
    if done is not None:
        return done
    p_max, m, words = planes.shape
    n = words * 32
    batch = x.shape[0]
    if x.shape != (batch, n) or p_req.shape != (batch,):
        raise ValueError("bcq_gemm_mixed: inconsistent shapes")
    ptrs = (ctypes.c_void_p * (p_max + 1))()
    for q, s in scales_by_p.items():
        if not 1 <= q <= p_max or s.shape != (q, m, n // group):
            raise ValueError(f"bcq_gemm_mixed: bad scale set for precision {q}")
        ptrs[q] = _dev(s, torch.float16, f"scales_by_p[{q}]")
    if y is None:
        y = torch.empty((batch, m), dtype=torch.float16, device=x.device)
    elif y.shape != (batch, m):
        raise ValueError("bcq_gemm_mixed: y has the wrong shape")
    if offsets_by_p:
        optrs = (ctypes.c_void_p * (p_max + 1))()
        for q, z in offsets_by_p.items():
            if not 1 <= q <= p_max or z.shape != (m, n // group):
                raise ValueError(f"bcq_gemm_mixed: bad offset set for precision {q}")
            optrs[q] = _dev(z, torch.float16, f"offsets_by_p[{q}]")
        _check(lib().bcq_gemm_mixed_offset(_dev(planes, torch.int32, "planes"), ctypes.cast(ptrs, ctypes.c_void_p),
                                           ctypes.cast(optrs, ctypes.c_void_p), _dev(p_req, torch.int32, "p_req"), p_max,
                                           _dev(x, torch.float16, "x"), _dev(y, torch.float16, "y"), m, n, batch, group,
                                           _stream()), "bcq_gemm_mixed_offset")
        return y
    _check(lib().bcq_gemm_mixed(_dev(planes, torch.int32, "planes"), ctypes.cast(ptrs, ctypes.c_void_p),
                                _dev(p_req, torch.int32, "p_req"), p_max, _dev(x, torch.float16, "x"),
                                _dev(y, torch.float16, "y"), m, n, batch, group, _stream()), "bcq_gemm_mixed")
    return y


def bcq_quantize(w: torch.Tensor, p_low: int, p_high: int, cycles: int, group: int = 128, with_offset: bool = False,
                 planes: torch.Tensor | None = None, scales_by_p: dict | None = None, offsets_by_p: dict | None = None,
                 listing_residual: bool = False):
    """Algorithm 1 on float16 weights [m][n]: returns ``(planes int32 [p_high][m][n/32], {p: scales float16
    [p][m][n/group]}, {p: offsets float16 [m][n/group]} or None)`` for p = p_low..p_high.  ``listing_residual``
    selects the expansion residual as the algorithm's listing prints it (``bcq_quantize_form``)."""
    m, n = w.shape
    if n % 32 or n % group:
        raise ValueError("bcq_quantize: n must be a multiple of 32 and of group")
    dev = w.device
    if planes is None:
        planes = torch.empty((p_high, m, n // 32), dtype=torch.int32, device=dev)
    elif planes.shape != (p_high, m, n // 32):
        raise ValueError("bcq_quantize: planes has the wrong shape")
    rng = range(max(p_low, 1), min(p_high, BCQ_MAX_PLANES) + 1)
    if scales_by_p is None:
        scales_by_p = {p: torch.empty((p, m, n // group), dtype=torch.float16, device=dev) for p in rng}
    if with_offset and offsets_by_p is None:
        offsets_by_p = {p: torch.empty((m, n // group), dtype=torch.float16, device=dev) for p in rng}
    size = max(p_high, 0) + 1
    sp = (ctypes.c_void_p * size)()
    op = (ctypes.c_void_p * size)()
    for p in rng:
        if scales_by_p[p].shape != (p, m, n // group):
            raise ValueError(f"bcq_quantize: bad scale set for precision {p}")
        sp[p] = _dev(scales_by_p[p], torch.float16, f"scales_by_p[{p}]")
        if offsets_by_p is not None:
            if offsets_by_p[p].shape != (m, n // group):
                raise ValueError(f"bcq_quantize: bad offset set for precision {p}")
            op[p] = _dev(offsets_by_p[p], torch.float16, f"offsets_by_p[{p}]")
    _check(lib().bcq_quantize_form(_dev(w, torch.float16, "w"), p_low, p_high, cycles, 1 if listing_residual else 0,
                                   _dev(planes, torch.int32, "planes"), ctypes.cast(sp, ctypes.c_void_p),
                                   ctypes.cast(op, ctypes.c_void_p) if offsets_by_p is not None else None,
                                   m, n, group, _stream()), "bcq_quantize")
    return planes, scales_by_p, offsets_by_p


def _type(dtype, where: str) -> int:
    if dtype not in TYPES:
        raise TypeError(f"{where}: 16-bit tensors are torch.float16 or torch.bfloat16, got {dtype}")
    return TYPES[dtype]


def _activation(name, where: str) -> int:
    if name not in ACTIVATIONS:
        raise ValueError(f"{where}: activation must be one of {sorted(ACTIVATIONS)}, got {name!r}")
    return ACTIVATIONS[name]


def _int8_shapes(where: str, q, token_scales, mats) -> tuple:
    """(tokens, m, n) of the codes of some tokens and of one or two matrices with their scales, all on one device."""
    for t in (q, token_scales, *(t for pair in mats for t in pair)):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError(f"{where}: codes and scales must be GPU tensors (there is no CPU path)")
        if t.device != q.device:
            raise ValueError(f"{where}: tensors on several devices")
    if q.dim() != 2 or token_scales.shape != q.shape[:1] or mats[0][0].dim() != 2:
        raise ValueError(f"{where}: inconsistent shapes")
    m, n = mats[0][0].shape[0], q.shape[1]
    for w, c in mats:
        if w.shape != (m, n) or c.shape != (m,):
            raise ValueError(f"{where}: inconsistent shapes")
    return q.shape[0], m, n


def _int8_result(where: str, t, shape: tuple, dtype, like) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    if not isinstance(t, torch.Tensor) or t.shape != shape or t.device != like.device:
        raise ValueError(f"{where}: the result's tensor has the wrong shape or device")
    return t


def bcq_int8_quantize(x: torch.Tensor, q: torch.Tensor | None = None, scales: torch.Tensor | None = None) -> tuple:
    """Rows of float16 or bfloat16 [rows][n] to ``(codes int8 [rows][n], scales float32 [rows])``: scale max |x| / 127, codes rounded to
    nearest, ties to even.  Tokens at run time, output channels of a weight matrix offline."""
    if _host is None:
        lib()
    done = _host.int8_quantize(x, q, scales)
    if done is not None:
        return done
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("x must be a GPU tensor (there is no CPU path)")
    if x.dim() != 2:
        raise ValueError("bcq_int8_quantize: x must be [rows][n]")
    rows, n = x.shape
    kind = _type(x.dtype, "bcq_int8_quantize")
    q = _int8_result("bcq_int8_quantize", q, (rows, n), torch.int8, x)
    scales = _int8_result("bcq_int8_quantize", scales, (rows,), torch.float32, x)
    with torch.cuda.device(x.device):
        _check(lib().bcq_int8_quantize(_dev(x, x.dtype, "x"), kind, _dev(q, torch.int8, "q"), _dev(scales, torch.float32, "scales"), rows, n,
                                       _stream()), "bcq_int8_quantize")
    return q, scales


def bcq_int8_gemm(q: torch.Tensor, token_scales: torch.Tensor, w: torch.Tensor, channel_scales: torch.Tensor,
                  dtype: torch.dtype = torch.float16, y: torch.Tensor | None = None) -> torch.Tensor:
    """y[t][r] = token_scales[t] * channel_scales[r] * sum_j q[t][j] w[r][j]: int8 codes q [tokens][n] and w [m][n], float32 scales,
    y [tokens][m] of ``dtype`` (float16 or bfloat16; a given ``y`` must have it)."""
    if _host is None:
        lib()
    done = _host.int8_gemm(q, token_scales, w, channel_scales, dtype, y)
    if done is not None:
        return done
    tokens, m, n = _int8_shapes("bcq_int8_gemm", q, token_scales, [(w, channel_scales)])
    kind = _type(dtype, "bcq_int8_gemm")
    y = _int8_result("bcq_int8_gemm", y, (tokens, m), dtype, q)
    with torch.cuda.device(q.device):
        _check(lib().bcq_int8_gemm(_dev(q, torch.int8, "q"), _dev(token_scales, torch.float32, "token_scales"), _dev(w, torch.int8, "w"),
                                   _dev(channel_scales, torch.float32, "channel_scales"), _dev(y, dtype, "y"), kind, m, n, tokens, _stream()),
               "bcq_int8_gemm")
    return y


def bcq_int8_gated(q: torch.Tensor, token_scales: torch.Tensor, w_gate: torch.Tensor, gate_scales: torch.Tensor, w_up: torch.Tensor,
                   up_scales: torch.Tensor, activation: str = "silu", dtype: torch.dtype = torch.float16,
                   h: torch.Tensor | None = None) -> torch.Tensor:
    """The gated feed-forward block up to its down projection in one kernel: h = act(g) * u with g and u the 8-bit products
    (``bcq_int8_gemm``, not rounded) of the gate and up matrices.  ``activation``: "silu" or "gelu" (tanh form)."""
    if _host is None:
        lib()
    done = _host.int8_gated(q, token_scales, w_gate, gate_scales, w_up, up_scales, activation, dtype, h)
    if done is not None:
        return done
    tokens, m, n = _int8_shapes("bcq_int8_gated", q, token_scales, [(w_gate, gate_scales), (w_up, up_scales)])
    kind, act = _type(dtype, "bcq_int8_gated"), _activation(activation, "bcq_int8_gated")
    h = _int8_result("bcq_int8_gated", h, (tokens, m), dtype, q)
    with torch.cuda.device(q.device):
        _check(lib().bcq_int8_gated(_dev(q, torch.int8, "q"), _dev(token_scales, torch.float32, "token_scales"),
                                    _dev(w_gate, torch.int8, "w_gate"), _dev(gate_scales, torch.float32, "gate_scales"),
                                    _dev(w_up, torch.int8, "w_up"), _dev(up_scales, torch.float32, "up_scales"), act, _dev(h, dtype, "h"),
                                    kind, m, n, tokens, _stream()), "bcq_int8_gated")
    return h


def _int8_backward_setup(where: str, dy, tokens: int, m: int, n: int, matrices: int, like) -> tuple:
    """The type, dx and the workspace of a backward call."""
    if not isinstance(dy, torch.Tensor) or not dy.is_cuda:
        raise TypeError(f"{where}: the gradient must be a GPU tensor (there is no CPU path)")
    if dy.shape != (tokens, m) or dy.device != like.device:
        raise ValueError(f"{where}: the gradient has the wrong shape or device")
    kind = _type(dy.dtype, where)
    size = lib().bcq_int8_backward_workspace(matrices, m, n, tokens)
    _check(min(size, 0), where)
    return (kind, torch.empty((tokens, n), dtype=dy.dtype, device=like.device), size,
            torch.empty((size,), dtype=torch.uint8, device=like.device))


def bcq_int8_gemm_backward(dy: torch.Tensor, q: torch.Tensor, token_scales: torch.Tensor, w: torch.Tensor,
                           channel_scales: torch.Tensor) -> tuple:
    """Gradients of ``bcq_int8_gemm`` with the codes fixed: ``(dx [tokens][n] of dy's type, dchannel_scales float32 [m])``, dx being the
    gradient of the activations that were quantised."""
    where = "bcq_int8_gemm_backward"
    if _host is None:
        lib()
    done = _host.int8_gemm_backward(dy, q, token_scales, w, channel_scales)
    if done is not None:
        return done
    tokens, m, n = _int8_shapes(where, q, token_scales, [(w, channel_scales)])
    with torch.cuda.device(q.device):
        kind, dx, size, workspace = _int8_backward_setup(where, dy, tokens, m, n, 1, q)
        dscales = torch.empty((m,), dtype=torch.float32, device=q.device)
        _check(lib().bcq_int8_gemm_backward(_dev(dy, dy.dtype, "dy"), _dev(q, torch.int8, "q"), _dev(token_scales, torch.float32, "token_scales"),
                                            _dev(w, torch.int8, "w"), _dev(channel_scales, torch.float32, "channel_scales"), dx.data_ptr(),
                                            dscales.data_ptr(), kind, m, n, tokens, workspace.data_ptr(), size, _stream()), where)
    return dx, dscales


def bcq_int8_gated_backward(dh: torch.Tensor, q: torch.Tensor, token_scales: torch.Tensor, w_gate: torch.Tensor, gate_scales: torch.Tensor,
                            w_up: torch.Tensor, up_scales: torch.Tensor, activation: str = "silu") -> tuple:
    """Gradients of ``bcq_int8_gated`` with the codes fixed: ``(dx [tokens][n] of dh's type, dgate_scales float32 [m], dup_scales float32
    [m])``; the projections are computed again."""
    where = "bcq_int8_gated_backward"
    if _host is None:
        lib()
    done = _host.int8_gated_backward(dh, q, token_scales, w_gate, gate_scales, w_up, up_scales, activation)
    if done is not None:
        return done
    tokens, m, n = _int8_shapes(where, q, token_scales, [(w_gate, gate_scales), (w_up, up_scales)])
    act = _activation(activation, where)
    with torch.cuda.device(q.device):
        kind, dx, size, workspace = _int8_backward_setup(where, dh, tokens, m, n, 2, q)
        dgate, dup = (torch.empty((m,), dtype=torch.float32, device=q.device) for _ in range(2))
        _check(lib().bcq_int8_gated_backward(_dev(dh, dh.dtype, "dh"), _dev(q, torch.int8, "q"),
                                             _dev(token_scales, torch.float32, "token_scales"), _dev(w_gate, torch.int8, "w_gate"),
                                             _dev(gate_scales, torch.float32, "gate_scales"), _dev(w_up, torch.int8, "w_up"),
                                             _dev(up_scales, torch.float32, "up_scales"), act, dx.data_ptr(), dgate.data_ptr(),
                                             dup.data_ptr(), kind, m, n, tokens, workspace.data_ptr(), size, _stream()), where)
    return dx, dgate, dup


def bench_stream_read(buf: torch.Tensor, sink: torch.Tensor) -> None:
    """Benchmark reference: stream ``buf`` (any dtype, a multiple of 16 bytes) through 128-bit loads."""
    if not buf.is_cuda or not buf.is_contiguous():
        raise TypeError("buf must be a contiguous GPU tensor")
    _check(lib().bcq_bench_stream_read(buf.data_ptr(), buf.numel() * buf.element_size(), _dev(sink, torch.int32, "sink"), _stream()),
           "bcq_bench_stream_read")


def bench_fp16_gemv(w: torch.Tensor, x: torch.Tensor, y: torch.Tensor) -> torch.Tensor:
    """Benchmark reference: y = w @ x in binary16 with fp32 accumulation, one wavefront per row."""
    m, n = w.shape
    if x.shape != (n,) or y.shape != (m,):
        raise ValueError("bench_fp16_gemv: inconsistent shapes")
    _check(lib().bcq_bench_fp16_gemv(_dev(w, torch.float16, "w"), _dev(x, torch.float16, "x"), _dev(y, torch.float16, "y"), m, n,
                                     _stream()), "bcq_bench_fp16_gemv")
    return y


def bench_issue_probe(kind: int, valu: int, waves: int, iters: int, ticks: torch.Tensor, sink: torch.Tensor) -> torch.Tensor:
    """Benchmark reference: one workgroup of ``waves`` wavefronts alternates matrix instructions of ``kind`` with ``valu``
    vector FMAs; ``ticks`` (int64[32]) receives per wavefront the shader-clock and the 100 MHz ticks of its loop."""
    if ticks.numel() < 32 or sink.numel() < 1024:
        raise ValueError("bench_issue_probe: ticks needs 32 values, sink 1024")
    _check(lib().bcq_bench_issue_probe(int(kind), int(valu), int(waves), int(iters), _dev(ticks, torch.int64, "ticks"),
                                       _dev(sink, torch.float32, "sink"), _stream()), "bcq_bench_issue_probe")
    return ticks
