"""8-bit integer quantization with a scale for each line: codes and scales equal the 64-bit reference
exactly (the scale is one rounding, the quotient is rounded once), reconstruction is one product."""

import numpy as np
import pytest
import torch

from paper_2608_10010_amd import cfint8 as i8
from tests import int8_ref as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def source(rng, rows, cols, dtype, kind="normal"):
    x = rng.standard_normal((rows, cols)).astype(np.float32)
    if kind == "halves":           # many quotients next to 0.5, 1.5, ..., 63.5: x = max * odd / 254
        top = np.exp2(rng.integers(-3, 4, (rows, 1))).astype(np.float32) * \
            rng.uniform(1, 2, (rows, 1)).astype(np.float32)
        x = (top * (2 * rng.integers(-63, 64, (rows, cols)) + 1) / 254).astype(np.float32)
        x[:, :1] = top
        x[:, 1::3] = (top / 2).astype(np.float32)
    elif kind == "tiny":
        x = (x * np.exp2(rng.uniform(-149, -100, (rows, 1)))).astype(np.float32)
    elif kind == "huge":
        x = (x * np.float32(3e37)).astype(np.float32)
    elif kind == "zeros":
        x[:] = 0.0
        x[::2] = -0.0
    t = torch.from_numpy(x)
    return t.to(DT[dtype])


def placed(t, pad):
    """On the device with `pad` more columns behind each row, which hold infinities."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("inf"), dtype=t.dtype, device=R.DEV)
    wide[:, :t.shape[1]] = t.to(R.DEV)
    return wide[:, :t.shape[1]]


def check(t, dtype, axis, mul=None, pad=0, ldq=None):
    rows, cols = t.shape
    outer, k = (rows, cols) if axis == 1 else (cols, rows)
    x = placed(t, pad)
    ldq = R.ceil16(k) if ldq is None else ldq
    codes = torch.full((outer + 1, ldq), 99, dtype=torch.int8, device=R.DEV)
    scales = torch.full((outer + 1,), -5.0, device=R.DEV)
    m = None if mul is None else torch.from_numpy(mul).to(R.DEV)
    q, s = i8.cfint8_quantize(x, block_axis=axis, mul=m, codes=codes[:outer, :k], scales=scales)
    torch.cuda.synchronize()
    v = t.float().numpy() if axis == 1 else t.float().numpy().T
    with np.errstate(over="ignore"):
        v = v if mul is None else v * mul[None, :]
    wq, ws = R.quantize(v)
    got = codes.cpu().numpy()
    assert np.array_equal(scales[:outer].cpu().numpy(), ws, equal_nan=True), "scales"
    bad = np.argwhere(got[:outer, :k] != wq)
    assert bad.size == 0, f"codes: {len(bad)} differ, first at {bad[0]}"
    # nothing behind a row's codes, the last row or the last scale is written
    assert (got[:outer, k:] == 99).all() and (got[outer] == 99).all() and float(scales[outer]) == -5.0


# each side of every variant's widest row, and one past the register kernels' reach
WIDTHS = [1, 7, 8, 9, 500, 512, 513, 1024, 1031, 2048, 2049, 4096, 4099, 8192, 8195, 16384, 16391, 32768, 32775]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", WIDTHS)
def test_rows_of_every_width(cols, dtype):
    rng = np.random.default_rng(cols)
    pad = -cols % (8 if dtype == "bf16" else 4)
    for rows, mul in ((1, False), (5, True)):
        say(f"[int8 quantize] rows={rows} cols={cols} {dtype} mul={mul}")
        m = np.exp(rng.standard_normal(cols)).astype(np.float32) if mul else None
        check(source(rng, rows, cols, dtype), dtype, 1, m, pad=pad + 8, ldq=R.ceil16(cols) + 32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 300), (3, 129), (63, 128), (64, 5), (65, 250), (127, 131), (129, 8),
                                       (1000, 77), (2049, 260), (5000, 33)])
def test_columns(rows, cols, dtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    for pad, mul in ((0, True), (-cols % 8 + 8, False), (-cols % 8, True), (3, False)):
        say(f"[int8 quantize] columns rows={rows} cols={cols} {dtype} pad={pad} mul={mul}")
        m = np.exp(rng.standard_normal(rows)).astype(np.float32) if mul else None
        check(source(rng, rows, cols, dtype), dtype, 0, m, pad=pad, ldq=R.ceil16(rows) + 16)


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["halves", "tiny", "huge", "zeros"])
def test_values_next_to_a_border(kind, dtype, axis):
    rng = np.random.default_rng(5)
    for rows, cols in ((40, 344), (128, 1600)):
        say(f"[int8 quantize] {kind} {dtype} axis={axis} {rows}x{cols}")
        check(source(rng, rows, cols, dtype, kind), dtype, axis)


@pytest.mark.parametrize("axis", [0, 1])
def test_lines_that_are_not_finite(axis):
    rng = np.random.default_rng(6)
    t = source(rng, 48, 272, "f32")
    t[3, 5], t[17, 100], t[30, 271] = float("nan"), float("inf"), float("-inf")
    say(f"[int8 quantize] not finite, axis={axis}")
    check(t, "f32", axis)
    m = np.ones(272 if axis == 1 else 48, np.float32)
    m[2] = np.inf
    check(source(rng, 48, 272, "bf16"), "bf16", axis, m)       # every line holds x * inf
    m[2] = 1e38
    check(source(rng, 48, 272, "bf16") * 100, "bf16", axis, m)  # products past fp32's range are infinities


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("outer,k", [(1, 1), (3, 5), (200, 30), (7, 4096), (5, 4100), (2, 20001), (300, 1000)])
def test_reconstruction(outer, k, dtype):
    rng = np.random.default_rng(outer + k)
    q = R.random_codes(rng, outer, k)
    q[0, 0] = -128                                   # a code that no quantizer writes is read as it is
    s = np.exp(rng.standard_normal(outer) * 20).astype(np.float32)
    s[outer // 2] = np.nan if outer > 2 else s[outer // 2]
    per = 4 if dtype == "f32" else 8
    dst = torch.full((outer + 1, -(-k // per) * per + per), 3.0, dtype=DT[dtype], device=R.DEV)
    say(f"[int8 dequantize] {outer}x{k} {dtype}")
    i8.cfint8_dequantize(R.codes_tensor(q), torch.from_numpy(s).to(R.DEV), outer, k, dst=dst)
    torch.cuda.synchronize()
    want = torch.from_numpy(q.astype(np.float32) * s[:, None]).to(DT[dtype])   # one product, one rounding
    R.same_bits(dst[:outer, :k], want, "values")
    assert bool((dst[:outer, k:] == 3).all()) and bool((dst[outer] == 3).all())


def test_rows_past_32_bits_of_offset():
    """Rows whose elements lie past 2^31 from the first, codes past it as well."""
    rows, cols = 70000, 32768                        # 2.3e9 codes, 4.6e9 bytes of source
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device=R.DEV)
    rng = np.random.default_rng(9)
    pick = [0, 40000, 65536, 69999]
    t = source(rng, len(pick), cols, "bf16")
    x[pick] = t.to(R.DEV)
    say("[int8 quantize] 70000 x 32768")
    q, s = i8.cfint8_quantize(x)
    y = None
    torch.cuda.synchronize()
    wq, ws = R.quantize(t.float().numpy())
    assert np.array_equal(q[pick].cpu().numpy(), wq) and np.array_equal(s[pick].cpu().numpy(), ws)
    assert float(s[12345]) == 0.0
    del x
    y = i8.cfint8_dequantize(q, s, rows, cols, dtype=torch.bfloat16)
    torch.cuda.synchronize()
    R.same_bits(y[pick], torch.from_numpy(wq.astype(np.float32) * ws[:, None]).to(torch.bfloat16), "values")


@pytest.mark.parametrize("axis", [1, 0])
def test_more_lines_than_a_launch_takes(axis):
    lines, k = (1 << 21) + 37, 5
    say(f"[int8 quantize] {lines} lines, axis {axis}")
    rng = np.random.default_rng(3)
    v = rng.standard_normal((lines, k)).astype(np.float32)
    if axis == 1:
        x = torch.zeros((lines, 8), device=R.DEV)[:, :k]
        x.copy_(torch.from_numpy(v))
    else:
        x = torch.from_numpy(np.ascontiguousarray(v.T)).to(R.DEV)
    q, s = i8.cfint8_quantize(x, block_axis=axis)
    wq, ws = R.quantize(v)
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)
    y = i8.cfint8_dequantize(q, s, lines, k)
    R.same_bits(y, torch.from_numpy(wq.astype(np.float32) * ws[:, None]), "values")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(128, 7), (256, 8), (255, 9), (257, 1030), (200, 127), (129, 129), (300, 1), (400, 135)])
def test_columns_that_end_inside_pieces(rows, cols, dtype):
    """Rows whose pieces are aligned (a wider buffer) and not, in one launch and in two."""
    rng = np.random.default_rng(rows * cols)
    m = np.exp(rng.standard_normal(rows)).astype(np.float32)
    say(f"[int8 quantize] columns {rows} x {cols} {dtype}")
    for pad in (0, -cols % 8, 1):
        check(source(rng, rows, cols, dtype), dtype, 0, m if pad else None, pad=pad, ldq=R.ceil16(rows) + 16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [3000, 5900, 6143, 6144, 6145, 6151, 8193, 11007, 12287, 12288, 12289, 12295, 24001])
def test_rows_of_three_units_a_thread(cols, dtype):
    """Both ends of the row kernels with three units a thread (to 6144 and to 12288) and inside their third."""
    rng = np.random.default_rng(cols)
    for rows, mul in ((3, True), (2, False)):
        say(f"[int8 quantize] rows={rows} cols={cols} {dtype} mul={mul}")
        m = np.exp(rng.standard_normal(cols)).astype(np.float32) if mul else None
        check(source(rng, rows, cols, dtype), dtype, 1, m, pad=-cols % 8 + 8, ldq=R.ceil16(cols) + 32)


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(3, 5001), (2, 11111), (2, 20004), (2, 33001), (200, 136), (300, 136)])
def test_borders_in_every_kernel(rows, cols, dtype, axis):
    """Quotients next to ties, and lines whose scale is subnormal or rounds to 0, past the narrowest kernels."""
    rng = np.random.default_rng(cols)
    for kind in ("halves", "tiny", "huge"):
        say(f"[int8 quantize] {kind} {dtype} axis={axis} {rows}x{cols}")
        check(source(rng, rows, cols, dtype, kind), dtype, axis, pad=-cols % 8)
