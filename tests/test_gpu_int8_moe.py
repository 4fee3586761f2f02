"""The mixture-of-experts layer with 8-bit weights against its definition in 64 bits.

Bounds, element by element (u = 2^-24, half a step of fp32):
  x, h in fixed point   half a unit, 2^-23 (bf16) or 2^-31 (fp32) of the power of two above the row's largest
  sums                  exact for each digit of a row of x, and of 64 neighbours of h; digits, waves and groups of 64
                        meet in at most 16 + I / 64 fp32 operations on values of at most 3 times the sum of
                        magnitudes (signed digits), scales 3 more: 64 u of that sum, and 3 I / 64 u more of h's
  silu(g) u             |silu'| <= 1.1; exp, quotient and products: 16 u
  slot weights          exp of a difference rounded to u |l_j - l_0|, sum and quotient: 64 u + 2 u |l_j - l_0|; below
                        2^-126 fp32 steps by 2^-149 whatever the size: exp (2 steps), quotient by a sum >= 1 (its
                        numerator's error, and half a step): 2^-147 in all
  output                topk + 1 operations, and half a step of bf16
"""

import numpy as np
import pytest
import torch

from paper_2608_10010_amd import cfint8 as i8
from tests import int8_ref as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = R.U32


def make(T, E, H, I, dtype, seed=0, spread=1.0):
    rng = np.random.default_rng(seed + T + 7 * E + 11 * H + 13 * I)
    x = torch.from_numpy((rng.standard_normal((T, H)) * np.exp(rng.standard_normal((T, 1)) * spread))
                         .astype(np.float32)).to(DT[dtype])
    x[:, H // 3] *= 30
    r = torch.from_numpy((rng.standard_normal((E, H)) * 2 / np.sqrt(H)).astype(np.float32)).to(DT[dtype])
    gu, dn = R.random_codes(rng, E * 2 * I, H).reshape(E, 2 * I, H), R.random_codes(rng, E * H, I).reshape(E, H, I)
    gus = np.exp(rng.standard_normal((E, 2 * I)) * 0.2).astype(np.float32) / np.float32(40 * np.sqrt(H))
    dns = np.exp(rng.standard_normal((E, H)) * 0.2).astype(np.float32) / np.float32(40 * np.sqrt(I))
    return x, r, gu, gus, dn, dns


def unit(v, P):
    """Half a unit of each row's fixed point."""
    m = np.abs(v).max(axis=-1, keepdims=True)
    return np.where(m > 0, np.exp2(np.frexp(m)[1] - (30.0 if P == 4 else 22.0) - 1), 0.0)


def reference(x, r, gu, gus, dn, dns, topk, renorm, active, dtype):
    """(y, bound, ids, weights, weight bound)."""
    P = 3 if dtype == "bf16" else 4
    X, T = x.double().numpy(), x.shape[0]
    E, H, I = dn.shape
    held = (X @ r.double().numpy().T).astype(np.float32).astype(np.float64)
    order = np.argsort(-np.where(np.isnan(held), -np.inf, held), axis=1, kind="stable")[:, :topk]
    top = np.take_along_axis(held, order, 1)
    z = np.exp(top - top[:, :1])
    total = z.sum(1, keepdims=True) if renorm else np.exp(held - top[:, :1]).sum(1, keepdims=True)
    p = z / total
    far = np.abs(top - top[:, :1]) if renorm else np.abs(held - top[:, :1]).max(1, keepdims=True)
    dp = p * U * (64 + 2 * far.max(1, keepdims=True) + E) + 2.0 ** -147
    y, bound = np.zeros((T, H)), np.zeros((T, H))
    live = np.ones(T, bool) if active is None else active.astype(bool)
    silu = lambda g: g / (1 + np.exp(-g))  # noqa: E731
    for t in range(T):
        if not live[t]:
            continue
        for j in range(topk):
            e = order[t, j]
            W, S = gu[e].astype(np.float64), gus[e].astype(np.float64)
            dx = unit(X[t:t + 1], P)[0]
            v = (W @ X[t]) * S
            dv = S * (np.abs(W).sum(1) * dx + 64 * U * (np.abs(W) @ (np.abs(X[t]) + dx)))
            g, u, dg, du = v[:I], v[I:], dv[:I], dv[I:]
            h = silu(g) * u
            dh = 1.1 * dg * (np.abs(u) + du) + np.abs(silu(g)) * du + 16 * U * np.abs(h)
            hu = unit((np.abs(h) + dh)[None], P)[0]
            D, Sd = dn[e].astype(np.float64), dns[e].astype(np.float64)
            d = (D @ h) * Sd
            dd = Sd * (np.abs(D) @ (dh + hu) + (64 + 3 * I / 64) * U * (np.abs(D) @ (np.abs(h) + dh + hu)))
            y[t] += p[t, j] * d
            bound[t] += p[t, j] * dd + dp[t, j] * np.abs(d) + (topk + 1) * U * p[t, j] * np.abs(d)
    bound += R.U_OUT[DT[dtype]] * (np.abs(y) + bound) + 1e-40
    ids = order.astype(np.int32)
    ids[~live] = -1
    p[~live], dp[~live] = 0, 0                       # exactly zero there
    return y, bound, ids, p, dp


def dev(*vs):
    return [torch.from_numpy(v).to(R.DEV) if isinstance(v, np.ndarray) else v.to(R.DEV) for v in vs]


def run(T, E, topk, H, I, dtype, renorm=True, active=None, seed=0, ldx=0, change=None):
    say(f"[int8 moe] T={T} E={E} topk={topk} H={H} I={I} {dtype} renorm={renorm} active={active is not None}")
    x, r, gu, gus, dn, dns = make(T, E, H, I, dtype, seed)
    if change is not None:
        change(x, r)
    dx, dr, dgu, dgus, ddn, ddns = dev(x, r, gu, gus, dn, dns)
    wide = torch.full((T, H + ldx), float("nan"), dtype=x.dtype, device=R.DEV)
    wide[:, :H] = dx
    out = torch.full((T + 1, H + ldx), 5.0, dtype=x.dtype, device=R.DEV)
    act = None if active is None else torch.from_numpy(active).to(R.DEV)
    y, ids, w = i8.cfint8_moe(wide[:, :H], dr, dgu, dgus, ddn, ddns, topk, renormalize=renorm, active=act,
                              y=out[:T, :H])
    torch.cuda.synchronize()
    Y, bound, wi, wp, dp = reference(x, r, gu, gus, dn, dns, topk, renorm, active, dtype)
    assert np.array_equal(ids.cpu().numpy(), wi), "ids"
    assert (np.abs(w.cpu().double().numpy() - wp) <= dp).all(), "weights"
    err = np.abs(y.cpu().double().numpy() - Y)
    assert (err <= bound).all(), f"{(err > bound).sum()} beyond the bound, worst {np.max(err / bound):.3g} of it"
    assert bool((out[:T, H:] == 5).all()) and bool((out[T] == 5).all()), "written outside y"
    return y, ids, w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,topk,H,I", [
    (1, 1, 1, 16, 16), (1, 8, 2, 64, 48), (1, 64, 8, 512, 256), (2, 3, 3, 80, 112), (3, 130, 5, 144, 32),
    (7, 16, 2, 1024, 208), (16, 8, 4, 256, 528), (17, 2, 2, 272, 64), (40, 4, 1, 128, 96), (64, 128, 8, 256, 128),
    (5, 1024, 32, 64, 32), (256, 16, 4, 64, 32), (200, 1, 1, 96, 80), (4, 6, 6, 4096, 16), (2, 4, 2, 32, 2064)])
def test_sizes(T, E, topk, H, I, dtype):
    run(T, E, topk, H, I, dtype, renorm=True)
    run(T, E, topk, H, I, dtype, renorm=False, seed=1, ldx=16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_tokens(dtype):
    """Dead tokens, whatever they hold, get zero rows and take nothing."""
    T = 21
    active = np.ones(T, np.uint8)
    active[[0, 5, 6, 20]] = 0

    def poison(x, r):
        x[5] = float("nan")
        x[20, 3] = float("inf")

    y, ids, w = run(T, 9, 3, 128, 80, dtype, active=active, change=poison)
    assert bool((y[[0, 5, 6, 20]] == 0).all()) and bool((ids[[0, 5, 6, 20]] == -1).all())
    y, ids, w = run(T, 9, 3, 128, 80, dtype, active=np.zeros(T, np.uint8))
    assert bool((y == 0).all()) and bool((w == 0).all())


def test_ties_take_the_lowest_expert():
    def ties(x, r):
        r[:] = 0                                      # every logit 0
        r[5] = r[9]

    y, ids, w = run(6, 12, 4, 64, 32, "f32", change=ties)
    assert ids.cpu().tolist() == [[0, 1, 2, 3]] * 6 and bool((w == 0.25).all())

    def pairs(x, r):                                  # equal rows: the lower of each pair first
        r[8:] = r[:8]

    _, ids, _ = run(9, 16, 6, 64, 32, "bf16", change=pairs)
    ids = ids.cpu().numpy()
    assert (ids[:, 0::2] + 8 == ids[:, 1::2]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_not_finite_stay_alone(dtype):
    T, E, topk, H, I = 12, 6, 2, 160, 64
    x, r, gu, gus, dn, dns = make(T, E, H, I, dtype)
    say(f"[int8 moe] not finite {dtype}")
    clean, ids, _ = i8.cfint8_moe(*dev(x, r, gu, gus, dn, dns), topk)
    x[2, 7], x[9, 0] = float("nan"), float("inf")
    y, ids2, _ = i8.cfint8_moe(*dev(x, r, gu, gus, dn, dns), topk)
    torch.cuda.synchronize()
    assert bool(torch.isnan(y[[2, 9]]).all())
    keep = [t for t in range(T) if t not in (2, 9)]
    assert torch.equal(y[keep].cpu(), clean[keep].cpu()) and torch.equal(ids2[keep].cpu(), ids[keep].cpu())
    assert bool((ids2 >= 0).all()) and bool((ids2 < E).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zero_and_extreme_rows(dtype):
    def rows(x, r):
        x[0] = 0
        x[1] *= 1e-36                                # subnormal products
        x[2] *= 1e15
        x[3, 1:] = 0

    run(5, 5, 2, 96, 48, dtype, change=rows)


# many rows on each expert, or more experts than one workgroup ranks: each expert's codes read once for all its rows
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,topk,H,I", [
    (64, 16, 8, 64, 128), (256, 8, 4, 80, 48), (60, 12, 8, 272, 160), (256, 1, 1, 96, 528), (33, 260, 2, 64, 208),
    (1, 300, 5, 48, 80), (100, 300, 3, 144, 64)])
def test_expert_by_expert(T, E, topk, H, I, dtype):
    run(T, E, topk, H, I, dtype, renorm=True, ldx=8 if dtype == "bf16" else 4)
    active = np.ones(T, np.uint8)
    active[T // 2:T // 2 + 3] = 0

    def poison(x, r):
        x[T // 2] = float("nan")

    run(T, E, topk, H, I, dtype, renorm=False, seed=1, active=active, change=poison)


def test_the_way_to_the_sums_does_not_matter():
    """A token alone and in a batch large enough to go expert by expert: the same experts and weights, and outputs that
    differ by no more than both bounds."""
    T, E, topk, H, I = 80, 20, 4, 160, 288
    say("[int8 moe] alone and in a batch")
    x, r, gu, gus, dn, dns = make(T, E, H, I, "f32")
    d = dev(x, r, gu, gus, dn, dns)
    y, ids, w = i8.cfint8_moe(*d, topk)
    Y, bound = reference(x, r, gu, gus, dn, dns, topk, True, None, "f32")[:2]
    for t in (0, 41, 79):
        y1, ids1, w1 = i8.cfint8_moe(d[0][t:t + 1], *d[1:], topk)
        assert torch.equal(ids1[0], ids[t]) and torch.equal(w1[0], w[t])
        assert (np.abs(y1[0].cpu().double().numpy() - y[t].cpu().double().numpy()) <= 2 * bound[t]).all()
