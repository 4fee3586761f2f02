"""Python binding of the 8-bit integer operators of libcurvefp (argument marshalling only).

The functions carry the names of the C ABI in ``include/cfint8.h``: quantization with one fp32 scale
for each line, reconstruction, the product of such codes, and a mixture-of-experts layer for a few
tokens with such weights.  Tensors are checked like ``curvefp``'s: device, dtype, layout and size, a
failed check raising ValueError before anything reaches the library.

Matrices of codes are 2-D int8 tensors whose row stride is a multiple of 16 bytes; a matrix of odd
width is a view of a wider buffer (``codes_buffer``).

``stream``: the call runs there instead of on the current stream, as if it stood inside
``torch.cuda.stream(stream)``: outputs and workspaces that it allocates belong to that stream, and the
caller orders the operands' earlier and later use on others.
"""

import ctypes
from typing import Optional, Tuple

import torch

from . import curvefp as _cf
from .curvefp import DTYPES, CurveFPError, _check, _device, _on_gpu, _source_arg, _stream
from .curvefp import _matrix as _any_matrix

_FLOATS = tuple(DTYPES)
_fn = None


def lib() -> ctypes.CDLL:
    """libcurvefp.so with this header's signatures."""
    global _fn
    if _fn is None:
        L = _cf.lib()
        P, I, I64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
        L.cfint8_quantize_workspace_bytes.argtypes = [I64, I64, I]
        L.cfint8_quantize_workspace_bytes.restype = I64
        L.cfint8_quantize.argtypes = [P, I, I64, I64, I64, I, P, P, I64, P, P, I64, P]
        L.cfint8_quantize.restype = I
        L.cfint8_dequantize.argtypes = [P, I64, P, I64, I64, P, I, I64, P]
        L.cfint8_dequantize.restype = I
        L.cfint8_gemm_workspace_bytes.argtypes = [I64, I64, I64, I]
        L.cfint8_gemm_workspace_bytes.restype = I64
        L.cfint8_gemm.argtypes = [P, I64, P, P, I64, I, P, P, I64, I64, I64, P, I, I64, P, I64, P]
        L.cfint8_gemm.restype = I
        L.cfint8_moe_workspace_bytes.argtypes = [I64, I64, I64, I64, I64]
        L.cfint8_moe_workspace_bytes.restype = I64
        L.cfint8_moe.argtypes = [P, I, I64, I64, I64, P, I64, P, P, P, P, I64, I64, I, P, P, I64, P, P, P, I64, P]
        L.cfint8_moe.restype = I
        _fn = L
    return _fn


# ---------------------------------------------------------------- argument checks
# A call takes about as long on the host as a small kernel on the GPU, so each check asks a tensor once for its shape
# and strides and leaves the error's wording to the slow path.

def _place(what: str, stream, names, *tensors):
    """All tensors (None: absent) on the current GPU, and on the stream's when one is given."""
    if stream is None:
        dev = _device()
        try:
            for t in tensors:
                if t is not None and t.get_device() != dev:
                    break
            else:
                return
        except AttributeError:                       # no tensor: the slow path says so
            pass
    _on_gpu(what, [(name, t) for name, t in zip(names, tensors) if t is not None], stream)


_I8 = (torch.int8,)


def _matrix(what: str, name: str, t: torch.Tensor, rows: int, cols: int, dtypes) -> int:
    """A 2-D row-major matrix of at least rows x cols; its leading dimension (a single row of a matrix with 16-byte
    aligned rows has none of its own)."""
    st, sh = t.stride(), t.shape
    if len(st) != 2 or st[1] != 1 or sh[0] < rows or sh[1] < cols or (st[0] < cols and rows != 1) or t.dtype not in dtypes:
        _any_matrix(what, name, t, rows, cols, dtypes)
        st = t.stride()
    if rows > 1:
        return st[0]
    per = 16 // t.element_size()
    return -(-cols // per) * per


def _readable(what: str, name: str, t: torch.Tensor, rows: int, cols: int):
    """The last of the rows is readable up to the next multiple of 16 bytes (the others end in the next one)."""
    es = t.element_size()
    if (cols * es) % 16 == 0 or t.device.type == "meta":
        return
    end = (t.storage_offset() + (rows - 1) * t.stride(0)) * es + -(-cols * es // 16) * 16
    if t.untyped_storage().nbytes() < end:
        raise ValueError(f"{what}: {name}'s last row must be readable up to a multiple of 16 bytes "
                         f"(a view of a wider buffer)")


def _codes(what: str, name: str, t: torch.Tensor, rows: int, cols: int) -> int:
    """A matrix of codes that is read; its leading dimension."""
    ld = _matrix(what, name, t, rows, cols, _I8)
    if cols % 16:
        _readable(what, name, t, rows, cols)
    return ld


def _vector(what: str, name: str, t: torch.Tensor, n: int, dtype=torch.float32):
    """A contiguous vector (any shape) of at least n values."""
    if t.dtype is dtype and t.numel() >= n and t.is_contiguous():
        return
    if t.dtype != dtype:
        raise ValueError(f"{what}: {name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: {name} must be contiguous")
    if t.numel() < n:
        raise ValueError(f"{what}: {name} holds {t.numel()} values, the call needs {n}")


def _bytes(what: str, fn, *args) -> int:
    n = fn(*args)
    if n < 0:
        raise CurveFPError(int(n), what)
    return int(n)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """Memory that is first written on the call's stream comes from that stream's pool: a block of another one may
    still be in use there by what its last owner queued."""
    strides = (shape[1], 1) if len(shape) == 2 else (1,)
    if stream is not None and device.type == "cuda":
        with torch.cuda.stream(stream):
            return torch.empty_strided(shape, strides, dtype=dtype, device=device)
    return torch.empty_strided(shape, strides, dtype=dtype, device=device)      # 0.4 us less than torch.empty


def _scratch(what, workspace, need: int, device, stream):
    """(pointer, bytes, tensor) of the workspace, allocated here when not given."""
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = _empty((need,), torch.uint8, device, stream)
    have = workspace.numel() * workspace.element_size()
    if not workspace.is_contiguous() or have < need:
        raise ValueError(f"{what}: workspace must be contiguous and hold {need} bytes, it holds {have}")
    return workspace.data_ptr(), have, workspace


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def codes_buffer(rows: int, k: int, device, stream=None) -> torch.Tensor:
    """An uninitialised [rows, k] matrix of codes for use on a stream (None: the current one): contiguous where k is a
    multiple of 16, otherwise with rows of whole 16-byte pieces, or of whole 128-byte lines of memory where these add
    at most an eighth (a product reads rows by 128 codes: 333 x 6151 x 4099 20.8 us, 26.2 with rows of 4112 bytes)."""
    ld = -(-k // 16) * 16
    if ld != k and -(-k // 128) * 128 - k <= k // 8:
        ld = -(-k // 128) * 128
    t = _empty((rows, ld), torch.int8, torch.device(device), stream)
    return t if ld == k else t[:, :k]


# ---------------------------------------------------------------- entry points

def cfint8_quantize_workspace_bytes(rows: int, cols: int, block_axis: int = 1) -> int:
    return _bytes("cfint8_quantize_workspace_bytes", lib().cfint8_quantize_workspace_bytes, rows, cols, block_axis)


def cfint8_quantize(src: torch.Tensor, block_axis: int = 1, mul: Optional[torch.Tensor] = None,
                    codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Codes and scales of a 2-D fp32/bf16 tensor: block_axis=1, a scale for each row, codes
    [rows, cols]; block_axis=0, a scale for each column, codes [cols, rows].  mul: fp32 factors along
    the quantized axis, multiplied in first."""
    what = "cfint8_quantize"
    _place(what, stream, ("src", "mul", "codes", "scales", "workspace"), src, mul, codes, scales, workspace)
    sh = src.shape
    if len(sh) != 2:
        _source_arg(what, src)
    rows, cols = sh
    ld_src = _matrix(what, "src", src, rows, cols, _FLOATS)
    if block_axis == 1:
        outer, k = rows, cols
        if cols % 16:
            _readable(what, "src", src, rows, cols)
    else:
        outer, k = cols, rows
    if codes is None:
        codes = codes_buffer(outer, k, src.device, stream)
    ld_codes = _matrix(what, "codes", codes, outer, k, _I8)
    if scales is None:
        scales = _empty((outer,), torch.float32, src.device, stream)
    else:
        _vector(what, "scales", scales, outer)
    if mul is not None:
        _vector(what, "mul", mul, k)
    L = lib()
    wp, wb, held = None, 0, None
    if block_axis != 1 or workspace is not None:     # otherwise the library needs none
        wp, wb, held = _scratch(what, workspace,
                                _bytes(what, L.cfint8_quantize_workspace_bytes, rows, cols, block_axis), src.device,
                                stream)
    st = L.cfint8_quantize(src.data_ptr(), DTYPES[src.dtype], rows, cols, ld_src, block_axis, _ptr(mul),
                           codes.data_ptr(), ld_codes, scales.data_ptr(), wp, wb, _stream(stream))
    _check(st, what)
    return codes, scales


def cfint8_dequantize(codes: torch.Tensor, scales: torch.Tensor, outer: int, k: int, dtype=torch.float32,
                      dst: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """codes * scales, a scale for each row, as fp32 or bf16 (dst's dtype when it is given)."""
    what = "cfint8_dequantize"
    _place(what, stream, ("codes", "scales", "dst"), codes, scales, dst)
    ld_codes = _codes(what, "codes", codes, outer, k)
    _vector(what, "scales", scales, outer)
    if dst is None:
        if dtype not in DTYPES:
            raise ValueError(f"{what}: dtype must be one of {_FLOATS}, got {dtype}")
        per = 16 // dtype.itemsize
        dst = _empty((outer, -(-k // per) * per), dtype, codes.device, stream)[:, :k]
    ld_dst = _matrix(what, "dst", dst, outer, k, _FLOATS)
    st = lib().cfint8_dequantize(codes.data_ptr(), ld_codes, scales.data_ptr(), outer, k, dst.data_ptr(),
                                 DTYPES[dst.dtype], ld_dst, _stream(stream))
    _check(st, what)
    return dst


def cfint8_gemm_workspace_bytes(M: int, N: int, K: int, trans_b: int = 0) -> int:
    return _bytes("cfint8_gemm_workspace_bytes", lib().cfint8_gemm_workspace_bytes, M, N, K, trans_b)


def cfint8_gemm(a: torch.Tensor, a_scales: Optional[torch.Tensor], b: torch.Tensor,
                b_scales: Optional[torch.Tensor], M: int, N: int, K: int, trans_b: int = 0,
                bias: Optional[torch.Tensor] = None, dtype=torch.float32, c: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """C[M, N] = (a . b^T) a_scales[:, None] b_scales + bias in fp32 or bf16 (c's dtype when it is given).
    a: codes [M, K]; b: codes [N, K], or [K, N] with trans_b=1; scales of None are 1."""
    what = "cfint8_gemm"
    _place(what, stream, ("a", "b", "a_scales", "b_scales", "bias", "c", "workspace"), a, b, a_scales, b_scales, bias, c,
           workspace)
    lda = _codes(what, "a", a, M, K)
    ldb = _codes(what, "b", b, K, N) if trans_b else _codes(what, "b", b, N, K)
    if a_scales is not None:
        _vector(what, "a_scales", a_scales, M)
    if b_scales is not None:
        _vector(what, "b_scales", b_scales, N)
    if bias is not None:
        _vector(what, "bias", bias, N)
    if c is None:
        if dtype not in DTYPES:
            raise ValueError(f"{what}: dtype must be one of {_FLOATS}, got {dtype}")
        c = _empty((M, N), dtype, a.device, stream)
        ldc = N
    else:
        ldc = _matrix(what, "c", c, M, N, _FLOATS)
    L = lib()
    wp, wb, held = None, 0, None
    if trans_b or workspace is not None:             # otherwise the library needs none
        wp, wb, held = _scratch(what, workspace, _bytes(what, L.cfint8_gemm_workspace_bytes, M, N, K, trans_b), a.device,
                                stream)
    st = L.cfint8_gemm(a.data_ptr(), lda, _ptr(a_scales), b.data_ptr(), ldb, trans_b, _ptr(b_scales), _ptr(bias), M, N, K,
                       c.data_ptr(), DTYPES[c.dtype], ldc, wp, wb, _stream(stream))
    _check(st, what)
    return c


def cfint8_moe_workspace_bytes(T: int, E: int, topk: int, H: int, I: int) -> int:
    return _bytes("cfint8_moe_workspace_bytes", lib().cfint8_moe_workspace_bytes, T, E, topk, H, I)


def cfint8_moe(x: torch.Tensor, router: torch.Tensor, gate_up: torch.Tensor, gate_up_scales: torch.Tensor,
               down: torch.Tensor, down_scales: torch.Tensor, topk: int, renormalize: bool = True,
               active: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
               ids: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream=None):
    """A mixture-of-experts layer on x [T, H] (fp32 or bf16): router [E, H] of x's dtype, gate_up codes
    [E, 2 I, H] with scales [E, 2 I], down codes [E, H, I] with scales [E, H].  active: uint8 or bool
    [T], 0 for padded tokens (zero rows, ids -1).  Returns y [T, H], ids int32 and weights fp32 [T, topk]."""
    what = "cfint8_moe"
    _place(what, stream, ("x", "router", "gate_up", "gate_up_scales", "down", "down_scales", "active", "y", "ids",
                          "weights", "workspace"),
           x, router, gate_up, gate_up_scales, down, down_scales, active, y, ids, weights, workspace)
    sh = x.shape
    if len(sh) != 2:
        _source_arg(what, x)
    T, H = sh
    ld_x = _matrix(what, "x", x, T, H, _FLOATS)
    dtype, device = x.dtype, x.device
    rs, ds, gs = router.shape, down.shape, gate_up.shape
    if len(rs) != 2 or rs[1] != H or router.dtype != dtype or not router.is_contiguous():
        raise ValueError(f"{what}: router must be a contiguous [E, {H}] matrix of {dtype}, got "
                         f"{tuple(rs)} {router.dtype}")
    E = rs[0]
    if len(ds) != 3 or ds[0] != E or ds[1] != H:
        raise ValueError(f"{what}: down must be [{E}, {H}, I], got {tuple(ds)}")
    I = ds[2]
    if gs != (E, 2 * I, H):
        raise ValueError(f"{what}: gate_up must be {(E, 2 * I, H)}, got {tuple(gs)}")
    if gate_up.dtype != torch.int8 or down.dtype != torch.int8 or not (gate_up.is_contiguous() and down.is_contiguous()):
        name = "gate_up" if gate_up.dtype != torch.int8 or not gate_up.is_contiguous() else "down"
        raise ValueError(f"{what}: {name} must be contiguous torch.int8")
    _vector(what, "gate_up_scales", gate_up_scales, E * 2 * I)
    _vector(what, "down_scales", down_scales, E * H)
    if active is not None:
        _vector(what, "active", active, T, torch.bool if active.dtype == torch.bool else torch.uint8)
    L = lib()
    need = _bytes(what, L.cfint8_moe_workspace_bytes, T, E, topk, H, I)     # refuses sizes before anything is allocated
    if y is None:
        y = _empty((T, H), dtype, device, stream)
    ld_y = _matrix(what, "y", y, T, H, (dtype,))
    if ids is None:
        ids = _empty((T, topk), torch.int32, device, stream)
    else:
        _vector(what, "ids", ids, T * topk, torch.int32)
    if weights is None:
        weights = _empty((T, topk), torch.float32, device, stream)
    else:
        _vector(what, "weights", weights, T * topk)
    wp, wb, held = _scratch(what, workspace, need, device, stream)
    st = L.cfint8_moe(x.data_ptr(), DTYPES[dtype], T, H, ld_x, router.data_ptr(), E, gate_up.data_ptr(),
                      gate_up_scales.data_ptr(), down.data_ptr(), down_scales.data_ptr(), I, topk,
                      1 if renormalize else 0, _ptr(active), y.data_ptr(), ld_y, ids.data_ptr(),
                      weights.data_ptr(), wp, wb, _stream(stream))
    _check(st, what)
    return y, ids, weights
