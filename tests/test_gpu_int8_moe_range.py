"""The mixture-of-experts layer where its products leave fp32's range before their scales bring them back.

A power of two moved from one factor to another changes no rounding as long as every value stays normal, and neither
the router's logits, g, u nor y move: each result is compared bit for bit with that of the operands as they were.
"""

import numpy as np
import pytest
import torch

from paper_2608_10010_amd import cfint8 as i8
from tests.gpu_util import say
from tests.test_gpu_int8_moe import dev, make

pytestmark = pytest.mark.gpu

# one slot at a time (more columns than a workgroup takes), and each expert's codes for all its rows
SIZES = [(1, 4, 2, 512, 1040), (3, 8, 2, 256, 208), (64, 16, 8, 64, 128), (40, 300, 3, 1040, 592)]


def moved(v, k):
    """v times 2^k, still normal (or zero) in its type."""
    out = v * 2.0 ** k if isinstance(v, torch.Tensor) else np.ldexp(v, k)
    a = out.abs().double().numpy() if isinstance(v, torch.Tensor) else np.abs(out.astype(np.float64))
    assert a.max() < 2.0 ** 128 and a[a > 0].min() >= 2.0 ** -126
    return out


def same(got, want):
    torch.cuda.synchronize()
    for g, w, name in zip(got, want, ("y", "ids", "weights")):
        assert bool(torch.isfinite(w.double()).all())
        assert torch.equal(g.cpu(), w.cpu()), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,topk,H,I", SIZES)
@pytest.mark.parametrize("k", [114, -104])
def test_activations_far_from_one(T, E, topk, H, I, dtype, k):
    """x 2^k against router and gate/up scales 2^-k.  Two columns of x times codes add 2 * 100 * 127 to sums of about
    40 sqrt(H): 2^14 2^114 lies past fp32's range, g and u do not."""
    say(f"[int8 moe] x 2^{k} T={T} E={E} {dtype}")
    x, r, gu, gus, dn, dns = make(T, E, H, I, dtype, spread=0.3)
    x[:, H // 3] = x[:, H // 2] = 100
    gu[:, :, H // 3] = gu[:, :, H // 2] = 127
    for t in (x, r):
        t[t.abs() < 2.0 ** -10] = 0
    want = i8.cfint8_moe(*dev(x, r, gu, gus, dn, dns), topk)
    same(i8.cfint8_moe(*dev(moved(x, k), moved(r, -k), gu, moved(gus, -k), dn, dns), topk), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,topk,H,I", SIZES)
@pytest.mark.parametrize("k", [120, -90])
def test_inner_values_far_from_one(T, E, topk, H, I, dtype, k):
    """The up scales 2^k against the down scales 2^-k: h reaches 2^120 and its sums with codes of 127 pass 2^128."""
    say(f"[int8 moe] h 2^{k} T={T} E={E} {dtype}")
    x, r, gu, gus, dn, dns = make(T, E, H, I, dtype, spread=0.0)
    x.clamp_(-4, 4)
    dns = np.ldexp(dns, 30 if k > 0 else 0)           # so that dns 2^-k stays normal
    dn[:, ::2] = 127
    want = i8.cfint8_moe(*dev(x, r, gu, gus, dn, dns), topk)
    up = gus.copy()
    up[:, I:] = moved(gus[:, I:], k)
    same(i8.cfint8_moe(*dev(x, r, gu, up, dn, moved(dns, -k)), topk), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,topk,H,I", SIZES)
def test_subnormal_activations(T, E, topk, H, I, dtype):
    """x of whole numbers times 2^-133, every one of them subnormal, against the whole numbers themselves: the 2^133 lies
    in the router and the gate/up scales."""
    say(f"[int8 moe] subnormal x T={T} E={E} {dtype}")
    x, r, gu, gus, dn, dns = make(T, E, H, I, dtype)
    x = torch.from_numpy(np.random.default_rng(T).integers(-63, 64, (T, H)).astype(np.float32)).to(x.dtype)
    r[r.abs() < 2.0 ** -10] = 0
    low = dev(x, moved(r, -30), gu, moved(gus, -30), dn, dns)
    tiny = torch.from_numpy(np.ldexp(x.float().numpy(), -133)).to(x.dtype)
    assert float(tiny.abs().max()) < 2.0 ** -126 and torch.equal(tiny.double() * 2.0 ** 133, x.double())
    same(i8.cfint8_moe(*dev(tiny, moved(r, 103), gu, moved(gus, 103), dn, dns), topk), i8.cfint8_moe(*low, topk))
