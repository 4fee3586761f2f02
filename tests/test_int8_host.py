"""CPU-only checks of the 8-bit integer operators: the header's functions are exported and declared, sizes,
refusals of the C ABI (before any HIP call) and of the binding."""

import ctypes
import os
import re
import subprocess
import types

import numpy as np
import pytest
import torch

from paper_2608_10010_amd import build as B
from paper_2608_10010_amd import cfint8 as i8
from paper_2608_10010_amd import curvefp as cf
from tests import int8_ref as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "cfint8.h")
ENULL, ESHAPE, EFMT, EBLOCK, EALIGN = -1, -2, -3, -4, -5
STREAM = types.SimpleNamespace(cuda_stream=0)
P = 256                                              # a pointer that is never dereferenced here


@pytest.fixture(scope="module")
def L():
    return i8.lib()


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return {m.group(1): [p.strip() for p in m.group(2).split(",")]
            for m in re.finditer(r"\b(?:int|int64_t)\s+(cfint8_[a-z0-9_]+)\s*\(([^)]*)\)\s*;", text)}


def define(name):
    return int(re.search(r"#define\s+%s\s+\(\(int64_t\)(\d+)\)" % name, open(HEADER).read()).group(1))


def test_header_library_and_binding_agree(L):
    sigs = declared()
    out = subprocess.run(["nm", "-D", "--defined-only", B.LIB], capture_output=True, text=True, check=True).stdout
    assert set(re.findall(r"\bT (cfint8_[a-z0-9_]+)$", out, flags=re.M)) == set(sigs)
    width = {"int": ctypes.c_int, "int64_t": ctypes.c_int64}
    for name, params in sigs.items():
        assert hasattr(i8, name), name
        fn = getattr(L, name)
        assert len(fn.argtypes) == len(params), name
        for t, p in zip(fn.argtypes, params):
            assert t is (ctypes.c_void_p if "*" in p else width[p.split()[0]]), (name, p)
        assert fn.restype is (ctypes.c_int64 if name.endswith("_bytes") else ctypes.c_int), name


def test_reference_rounds_as_defined():
    """The tests' own quantizer: codes are nearest, ties to even, on values whose quotients are known."""
    x = np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 63.5, 126.49, 0.0]], np.float32)
    q, s = R.quantize(x)
    assert s[0] == 1.0 and q[0].tolist() == [127, 0, 2, 2, 0, -2, 64, 126, 0]
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 333)).astype(np.float32)
    q, s = R.quantize(x)
    d = np.abs(x.astype(np.float64) - q * s.astype(np.float64)[:, None])
    assert (d <= s[:, None].astype(np.float64) * (0.5 + 127 * 2.0 ** -24)).all() and (np.abs(q).max(axis=1) == 127).all()


def test_sizes(L):
    assert L.cfint8_quantize_workspace_bytes(100, 7, 1) == 0
    assert L.cfint8_quantize_workspace_bytes(1, 7, 0) == 4 * 7
    assert L.cfint8_quantize_workspace_bytes(0, 7, 0) == ESHAPE
    assert L.cfint8_quantize_workspace_bytes(1, 1 << 31, 1) == ESHAPE
    assert L.cfint8_quantize_workspace_bytes(1, 1, 2) == EBLOCK
    K = define("CFINT8_MAX_K")
    assert K * 128 * 128 < 2 ** 31
    assert L.cfint8_gemm_workspace_bytes(1, 1, K, 0) >= 0
    assert L.cfint8_gemm_workspace_bytes(1, 1, K + 1, 0) == ESHAPE
    assert L.cfint8_gemm_workspace_bytes(1, 0, 1, 0) == ESHAPE
    assert L.cfint8_gemm_workspace_bytes(1, 1, 1, 2) == EBLOCK
    T, E, k, W = (define("CFINT8_MOE_MAX_" + n) for n in ("TOKENS", "EXPERTS", "TOPK", "WIDTH"))
    assert L.cfint8_moe_workspace_bytes(T, E, k, W, W) > 0
    for bad in ((0, 8, 2, 64, 64), (T + 1, 8, 2, 64, 64), (4, E + 1, 2, 64, 64), (4, 8, 9, 64, 64), (4, 8, 0, 64, 64),
                (4, E, k + 1, 64, 64), (4, 8, 2, 72, 64), (4, 8, 2, 64, 8), (4, 8, 2, W + 16, 64), (4, 8, 2, 64, 0)):
        assert L.cfint8_moe_workspace_bytes(*bad) == ESHAPE, bad


def test_quantize_refusals(L):
    good = dict(src=P, dtype=1, rows=8, cols=40, ld=48, axis=1, mul=None, codes=P, ldq=48, scales=P, ws=None, wb=0)

    def st(**kw):
        a = {**good, **kw}
        return L.cfint8_quantize(a["src"], a["dtype"], a["rows"], a["cols"], a["ld"], a["axis"], a["mul"], a["codes"],
                                 a["ldq"], a["scales"], a["ws"], a["wb"], None)

    for k in ("src", "codes", "scales"):
        assert st(**{k: None}) == ENULL
    assert st(dtype=2) == EFMT
    assert st(axis=2) == EBLOCK
    for kw in (dict(rows=0), dict(cols=0), dict(rows=1 << 31), dict(ld=39), dict(ld=(1 << 30) + 8), dict(ldq=32),
               dict(ldq=define("CFINT8_MAX_LD") + 16), dict(axis=0, ws=P, wb=159)):
        assert st(**kw) == ESHAPE, kw
    assert st(axis=0, wb=160) == ENULL
    for kw in (dict(src=P + 8), dict(ld=44), dict(codes=P + 8), dict(ldq=56), dict(scales=P + 2), dict(mul=P + 4),
               dict(axis=0, ws=P + 8, wb=160), dict(axis=0, src=P + 1, ws=P, wb=160)):
        assert st(**kw) == EALIGN, kw


def test_dequantize_refusals(L):
    good = dict(codes=P, ldq=48, scales=P, outer=3, k=40, dst=P, dtype=0, ld=40)

    def st(**kw):
        a = {**good, **kw}
        return L.cfint8_dequantize(a["codes"], a["ldq"], a["scales"], a["outer"], a["k"], a["dst"], a["dtype"], a["ld"],
                                   None)

    for k in ("codes", "scales", "dst"):
        assert st(**{k: None}) == ENULL
    assert st(dtype=-1) == EFMT
    for kw in (dict(outer=0), dict(k=0), dict(ldq=32), dict(ld=39)):
        assert st(**kw) == ESHAPE, kw
    for kw in (dict(codes=P + 4), dict(ldq=56), dict(scales=P + 1), dict(dst=P + 8), dict(ld=42), dict(dtype=1, ld=44)):
        assert st(**kw) == EALIGN, kw


def test_gemm_refusals(L):
    good = dict(a=P, lda=48, sa=P, b=P, ldb=48, tr=0, sb=P, bias=P, M=3, N=40, K=33, c=P, ct=0, ldc=40, ws=P,
                wb=1 << 40)

    def st(**kw):
        g = {**good, **kw}
        return L.cfint8_gemm(g["a"], g["lda"], g["sa"], g["b"], g["ldb"], g["tr"], g["sb"], g["bias"], g["M"], g["N"],
                             g["K"], g["c"], g["ct"], g["ldc"], g["ws"], g["wb"], None)

    for k in ("a", "b", "c"):
        assert st(**{k: None}) == ENULL
    assert st(ct=2) == EFMT
    assert st(tr=2) == EBLOCK
    lim = define("CFINT8_MAX_LD")
    for kw in (dict(M=0), dict(N=0), dict(K=0), dict(M=1 << 31), dict(K=define("CFINT8_MAX_K") + 1, lda=lim, ldb=lim),
               dict(lda=32), dict(ldb=32), dict(tr=1, ldb=32), dict(lda=lim + 16), dict(ldc=39), dict(wb=-1)):
        assert st(**kw) == ESHAPE, kw
    for kw in (dict(a=P + 8), dict(lda=56), dict(b=P + 8), dict(ldb=56), dict(c=P + 8), dict(sa=P + 1), dict(sb=P + 2),
               dict(bias=P + 3)):
        assert st(**kw) == EALIGN, kw


def test_moe_refusals(L):
    good = dict(x=P, dtype=1, T=4, H=64, ldx=64, r=P, E=8, gu=P, gus=P, dn=P, dns=P, I=32, k=2, rn=1, act=None, y=P,
                ldy=64, ids=P, w=P, ws=P, wb=1 << 30)

    def st(**kw):
        a = {**good, **kw}
        return L.cfint8_moe(a["x"], a["dtype"], a["T"], a["H"], a["ldx"], a["r"], a["E"], a["gu"], a["gus"], a["dn"],
                            a["dns"], a["I"], a["k"], a["rn"], a["act"], a["y"], a["ldy"], a["ids"], a["w"], a["ws"],
                            a["wb"], None)

    for k in ("x", "r", "gu", "gus", "dn", "dns", "y", "ids", "w", "ws"):
        assert st(**{k: None}) == ENULL, k
    assert st(dtype=5) == EFMT
    for kw in (dict(T=0), dict(T=257), dict(E=0), dict(k=9), dict(k=0), dict(H=56), dict(I=40), dict(ldx=56),
               dict(ldy=56), dict(rn=2), dict(wb=L.cfint8_moe_workspace_bytes(4, 8, 2, 64, 32) - 1)):
        assert st(**kw) == ESHAPE, kw
    for kw in (dict(x=P + 8), dict(ldx=68), dict(r=P + 8), dict(gu=P + 8), dict(dn=P + 8), dict(gus=P + 2),
               dict(dns=P + 2), dict(y=P + 8), dict(ldy=68), dict(ids=P + 1), dict(w=P + 1), dict(ws=P + 128)):
        assert st(**kw) == EALIGN, kw


# ---------------------------------------------------------------- the binding ("meta" tensors stand for device ones)

@pytest.fixture
def meta(monkeypatch):
    monkeypatch.setattr(cf, "_GPU_DEVICE_TYPES", ("cuda", "meta"))
    return lambda shape, dtype=torch.int8: torch.empty(shape, dtype=dtype, device="meta")


def passes(fn):
    with pytest.raises(cf.CurveFPError) as e:        # a meta tensor's pointer is null
        fn()
    assert e.value.status == ENULL


def test_binding_refuses_host_tensors():
    x = torch.zeros((4, 32))
    with pytest.raises(ValueError, match="not on a GPU"):
        i8.cfint8_quantize(x, stream=STREAM)
    q = torch.zeros((4, 32), dtype=torch.int8)
    with pytest.raises(ValueError, match="not on a GPU"):
        i8.cfint8_gemm(q, None, q, None, 4, 4, 32, stream=STREAM)
    with pytest.raises(ValueError, match="not on a GPU"):
        i8.cfint8_dequantize(q, torch.zeros(4), 4, 32, stream=STREAM)


def test_binding_quantize(meta):
    f32 = torch.float32
    x = meta((8, 64), f32)
    passes(lambda: i8.cfint8_quantize(x, stream=STREAM))
    passes(lambda: i8.cfint8_quantize(x, block_axis=0, mul=meta(8, f32), stream=STREAM))
    for kw, match in ((dict(codes=meta((8, 48))), "needs at least"), (dict(codes=meta((8, 64), torch.uint8)), "one of"),
                      (dict(scales=meta(7, f32)), "holds 7"), (dict(scales=meta(8, torch.float64)), "must be"),
                      (dict(mul=meta(63, f32)), "holds 63"), (dict(mul=meta((64, 2), f32)[:, 0]), "contiguous"),
                      (dict(codes=meta((8, 64)).t()), "unit column stride")):
        with pytest.raises(ValueError, match=match):
            i8.cfint8_quantize(x, stream=STREAM, **kw)
    with pytest.raises(ValueError, match="one of"):
        i8.cfint8_quantize(meta((8, 64), torch.float16), stream=STREAM)
    with pytest.raises(ValueError, match="workspace"):
        i8.cfint8_quantize(x, block_axis=0, workspace=meta(16, torch.uint8), stream=STREAM)


def test_binding_readable_rows(monkeypatch):
    """A matrix of odd width whose storage ends with its last value is refused; a view of a wider one is not."""
    monkeypatch.setattr(cf, "_GPU_DEVICE_TYPES", ("cuda", "cpu"))
    tight = torch.zeros(3 * 48 - 10, dtype=torch.int8).as_strided((3, 38), (48, 1))
    with pytest.raises(ValueError, match="readable"):
        i8._codes("t", "a", tight, 3, 38)
    i8._codes("t", "a", torch.zeros((3, 48), dtype=torch.int8)[:, :38], 3, 38)
    i8._codes("t", "a", tight, 2, 38)


def test_binding_gemm(meta):
    f32 = torch.float32
    a, b, bt = meta((8, 64)), meta((40, 64)), meta((64, 48))[:, :40]
    sa, sb = meta(8, f32), meta(40, f32)
    passes(lambda: i8.cfint8_gemm(a, sa, b, sb, 8, 40, 64, stream=STREAM))
    passes(lambda: i8.cfint8_gemm(a, sa, bt, None, 8, 40, 64, trans_b=1, dtype=torch.bfloat16, stream=STREAM))
    for args, kw, match in (((a, sa, b, sb, 9, 40, 64), {}, "needs at least"), ((a, sa, b, sb, 8, 41, 64), {}, "at least"),
                            ((a, sa, bt, sb, 8, 40, 64), {}, "at least"), ((a, sb[:7], b, sb, 8, 40, 64), {}, "holds 7"),
                            ((a, sa, b, sa, 8, 40, 64), {}, "holds 8"),
                            ((a, sa, b, sb, 8, 40, 64), dict(bias=meta(39, f32)), "holds 39"),
                            ((a, sa, b, sb, 8, 40, 64), dict(c=meta((8, 39), f32)), "at least"),
                            ((a, sa, b, sb, 8, 40, 64), dict(dtype=torch.float16), "dtype"),
                            ((a, sa, meta((40, 64), torch.uint8), sb, 8, 40, 64), {}, "one of")):
        with pytest.raises(ValueError, match=match):
            i8.cfint8_gemm(*args, stream=STREAM, **kw)


def test_binding_moe(meta):
    f32 = torch.float32

    def call(x=(4, 64), r=(8, 64), gu=(8, 64, 64), gus=(8, 64), dn=(8, 64, 32), dns=(8, 64), topk=2, dt=f32, rdt=None,
             **kw):
        return i8.cfint8_moe(meta(x, dt), meta(r, rdt or dt), meta(gu), meta(gus, f32), meta(dn), meta(dns, f32), topk,
                             stream=STREAM, **kw)

    passes(call)
    passes(lambda: call(dt=torch.bfloat16, active=meta(4, torch.bool)))
    for kw, match in ((dict(r=(8, 32)), "router"), (dict(rdt=torch.bfloat16), "router"), (dict(dn=(7, 64, 32)), "down"),
                      (dict(gu=(8, 32, 64)), "gate_up"), (dict(gus=(8, 63)), "holds"), (dict(dns=(8, 63)), "holds"),
                      (dict(active=meta(3, torch.uint8)), "holds 3"), (dict(active=meta(4, f32)), "active"),
                      (dict(y=meta((4, 64), torch.bfloat16)), "one of"), (dict(ids=meta((4, 2), torch.int64)), "ids"),
                      (dict(weights=meta((4, 1), f32)), "holds 4")):
        with pytest.raises(ValueError, match=match):
            call(**kw)
    with pytest.raises(cf.CurveFPError):
        call(topk=9)
    with pytest.raises(cf.CurveFPError):
        call(x=(300, 64))


@pytest.mark.parametrize("topk", [-1, 0, 9, 33, 1 << 40])
def test_binding_moe_refuses_topk_before_it_allocates(meta, topk):
    """The library's error, whatever ids and weights of that size would have done."""
    f32 = torch.float32
    with pytest.raises(cf.CurveFPError) as e:
        i8.cfint8_moe(meta((4, 64), f32), meta((8, 64), f32), meta((8, 64, 64)), meta((8, 64), f32), meta((8, 64, 32)),
                      meta((8, 64), f32), topk, stream=STREAM)
    assert e.value.status == ESHAPE
