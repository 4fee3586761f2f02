"""Plain 64-bit references of the 8-bit integer operators (numpy, on the host)."""

import numpy as np
import torch

DEV = "cuda:0"
U32 = 2.0 ** -24          # half a step of fp32, relative
U_OUT = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}


def ceil16(n):
    return -(-n // 16) * 16


def quantize(v: np.ndarray):
    """(codes int8, scales fp32) of float32 lines [outer][k]: the scale rounded to fp32, the quotient in
    64 bits.  (A quotient that is no tie is at least 2^-32 away from one, relative: |v - (h + 1/2) s| is a
    multiple of half an ulp of s or of v.)"""
    v = v.astype(np.float32)
    amax = np.abs(v.astype(np.float64)).max(axis=1)
    bad = ~np.isfinite(amax)
    with np.errstate(invalid="ignore", divide="ignore"):
        s = (amax / 127.0).astype(np.float32)
        q = np.rint(v.astype(np.float64) / s.astype(np.float64)[:, None])
    q[(s == 0) | bad] = 0
    q = np.clip(np.where(np.isnan(q), 0, q), -127, 127).astype(np.int8)
    s[bad] = np.nan
    return q, s


def to_bf16(x: np.ndarray) -> torch.Tensor:
    return torch.from_numpy(x).to(torch.bfloat16)


def gemm(a, b, sa, sb, bias, dtype):
    """The product's own arithmetic: exact sum to fp32, significands multiplied, exponents in one step."""
    acc = (a.astype(np.float64) @ b.astype(np.float64).T)          # exact: below 2^53
    one = np.float32(1)
    sa = np.full(a.shape[0], one) if sa is None else sa.astype(np.float32)
    sb = np.full(b.shape[0], one) if sb is None else sb.astype(np.float32)
    ma, ea = np.frexp(sa)
    mb, eb = np.frexp(sb)
    m = acc.astype(np.float32) * (ma[:, None] * mb[None, :]).astype(np.float32)
    with np.errstate(over="ignore"):
        c = np.ldexp(m.astype(np.float64), (ea[:, None] + eb[None, :])).astype(np.float32)
    if bias is not None:
        c = c + bias.astype(np.float32)[None, :]
    t = torch.from_numpy(np.ascontiguousarray(c))
    return t if dtype == torch.float32 else t.to(torch.bfloat16)


def codes_tensor(q: np.ndarray, fill=77, ld=None):
    """int8 codes on the device in a wider buffer whose bytes behind each row hold `fill`."""
    ld = ceil16(q.shape[1]) if ld is None else ld
    t = torch.full((q.shape[0], ld), fill, dtype=torch.int8, device=DEV)
    t[:, :q.shape[1]] = torch.from_numpy(q).to(DEV)
    return t[:, :q.shape[1]]


def random_codes(rng, rows, k):
    return np.clip(np.rint(rng.standard_normal((rows, k)) * 40), -127, 127).astype(np.int8)


def same_bits(x: torch.Tensor, y: torch.Tensor, what: str):
    """Equal bit for bit; any NaN equals any NaN."""
    x, y = x.cpu(), y.cpu()
    assert x.dtype == y.dtype and x.shape == y.shape, what
    nx, ny = torch.isnan(x), torch.isnan(y)
    assert torch.equal(nx, ny), f"{what}: NaN in other places"
    same = (x == y) | nx
    assert bool(same.all()), f"{what}: {int((~same).sum())} of {same.numel()} differ, first at " \
                             f"{torch.nonzero(~same)[0].tolist()}"
