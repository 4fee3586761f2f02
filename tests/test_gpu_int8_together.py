"""The 8-bit operators as they are used together: a linear layer with both gradients, a mixture-of-experts layer
on quantized weights, graphs, streams and workspaces.

A quantized line v has |v - q s| <= s / 2 (1 + 2^-23 for the quotient's tie at the rounded scale) per element, and s is
rounded, so that max |v| / s may pass 127 by 127 2^-24: inside the same half step.  A product with exact sums adds
three fp32 operations: 4 u relative to the result, u = 2^-24.
"""

import numpy as np
import pytest
import torch

from paper_2608_10010_amd import cfint8 as i8
from tests import int8_ref as R
from tests.gpu_util import say
from tests.test_gpu_int8_moe import make, reference

pytestmark = pytest.mark.gpu
U = R.U32
BF, F32 = torch.bfloat16, torch.float32


def normal(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape).astype(np.float32)


def to(v, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(v)).to(dtype).to(R.DEV)


def n64(t):
    return t.cpu().double().numpy()


def padded(rows, cols, dtype):
    """A matrix whose rows are whole 16-byte pieces."""
    per = 16 // dtype.itemsize
    return torch.zeros((rows, -(-cols // per) * per), dtype=dtype, device=R.DEV)[:, :cols]


def matrix(v, dtype):
    t = padded(*v.shape, dtype)
    t.copy_(torch.from_numpy(v))
    return t


# ---------------------------------------------------------------- a linear layer, forward and backward

def linear(x, w, g):
    """y = x w^T of quantized x [T, K], w [N, K], and both gradients for dy = g [T, N]."""
    T, K = x.shape
    N = w.shape[0]
    qx, sx = i8.cfint8_quantize(x)
    qw, sw = i8.cfint8_quantize(w)
    y = i8.cfint8_gemm(qx, sx, qw, sw, T, N, K)
    qr, sr = i8.cfint8_quantize(g, mul=sw)
    dx = i8.cfint8_gemm(qr, sr, qw, None, T, K, N, trans_b=1)
    qc, sc = i8.cfint8_quantize(g, block_axis=0, mul=sx)
    dw = i8.cfint8_gemm(qc, sc, qx, None, N, K, T, trans_b=1)
    return (qx, sx, qw, sw, sr, sc), y, dx, dw


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,N,K", [(1, 16, 16), (5, 33, 70), (64, 130, 200), (257, 96, 385), (300, 520, 1024)])
def test_linear_layer_and_its_gradients(T, N, K, dtype):
    """Against the formula in 64 bits on the reconstructed operands, and against differences of its output."""
    say(f"[int8 together] linear {T} {N} {K} {dtype}")
    dt = {"bf16": BF, "f32": F32}[dtype]
    x, w, g = (matrix(normal(i, *s), dt) for i, s in enumerate(((T, K), (N, K), (T, N))))
    (qx, sx, qw, sw, sr, sc), y, dx, dw = linear(x, w, g)
    torch.cuda.synchronize()
    QX, QW, SX, SW, G = n64(qx), n64(qw), n64(sx), n64(sw), n64(g)
    X, W = QX * SX[:, None], QW * SW[:, None]               # what the layer multiplies
    Y = X @ W.T
    # the reference itself: K + 2 roundings by 2^-53 of terms of |X| |W| at most (a sum of codes may be exactly 0)
    ref = (K + 2) * 2.0 ** -53 * (np.abs(X) @ np.abs(W).T)
    assert (np.abs(n64(y) - Y) <= 4 * U * (np.abs(Y) + ref) + ref).all(), "y"
    # dX: each element of g sw is off by half a step of its row and u (the product with sw in fp32)
    near = lambda err: err * (1 + 2.0 ** -20) + 1e-30       # noqa: E731
    ex = near((0.5 * n64(sr)[:, None] + U * np.abs(G * SW)) @ np.abs(QW) + 4 * U * np.abs(G * SW) @ np.abs(QW))
    ew = near((0.5 * n64(sc)[:, None] + U * np.abs(G * SX[:, None]).T) @ np.abs(QX)
              + 4 * U * np.abs(G * SX[:, None]).T @ np.abs(QX))
    DX, DW = n64(dx), n64(dw)
    assert (np.abs(DX - G @ W) <= ex).all(), "dX"
    assert (np.abs(DW - G.T @ X) <= ew).all(), "dW"
    # differences of L = sum(g y) along a direction, with the layer's own forward in 64 bits (L is linear in each)
    rng = np.random.default_rng(9)
    for D, E, shape, L in ((DX, ex, X.shape, lambda d: (G * ((X + d) @ W.T)).sum()),
                           (DW, ew, W.shape, lambda d: (G * (X @ (W + d).T)).sum())):
        d = rng.standard_normal(shape)
        diff = (L(d / 2) - L(-d / 2))
        assert abs(diff - (D * d).sum()) <= (E * np.abs(d)).sum() + 1e-9 * np.abs(G).sum() * T, "difference"


def test_moe_layer_on_quantized_weights():
    """Weights quantized along their rows, experts' matrices as one; the layer against its definition."""
    T, E, topk, H, I = 9, 12, 3, 160, 96
    say("[int8 together] moe on quantized weights")
    x, r = make(T, E, H, I, "bf16")[:2]
    gu, gus = i8.cfint8_quantize(to(normal(5, E * 2 * I, H) / np.sqrt(H)))
    dn, dns = i8.cfint8_quantize(to(normal(6, E * H, I) / np.sqrt(I), BF))
    y, ids, w = i8.cfint8_moe(x.to(R.DEV), r.to(R.DEV), gu.view(E, 2 * I, H), gus.view(E, 2 * I), dn.view(E, H, I),
                              dns.view(E, H), topk)
    Y, bound, wi, wp, dp = reference(x, r, gu.cpu().numpy().reshape(E, 2 * I, H), gus.cpu().numpy().reshape(E, 2 * I),
                                     dn.cpu().numpy().reshape(E, H, I), dns.cpu().numpy().reshape(E, H), topk, True,
                                     None, "bf16")
    assert np.array_equal(ids.cpu().numpy(), wi)
    assert (np.abs(n64(w) - wp) <= dp).all() and (np.abs(n64(y) - Y) <= bound).all()


# ---------------------------------------------------------------- graphs, streams, workspaces

SIZES = [(1, 4096, 520), (16, 256, 2048), (40, 96, 272), (200, 300, 400), (600, 1040, 256)]   # each kind of product
LAYERS = [(1, 8, 2, 256, 128, BF), (20, 16, 4, 96, 64, F32), (64, 128, 4, 64, 48, BF), (40, 24, 8, 64, 160, F32),
          (9, 260, 2, 80, 64, BF)]


class Work:
    """Every operator once for each kind of size, outputs and workspaces held."""

    def __init__(self, seed):
        self.lin = []
        for i, (T, N, K) in enumerate(SIZES):
            d = BF if i % 2 else F32
            self.lin.append(dict(
                x=matrix(normal(seed + i, T, K), d), g=matrix(normal(seed + 50 + i, T, N), d),
                w=i8.cfint8_quantize(matrix(normal(90 + i, N, K), F32)),
                qx=(i8.codes_buffer(T, K, R.DEV), torch.zeros(T, device=R.DEV)),
                qg=(i8.codes_buffer(T, N, R.DEV), torch.zeros(T, device=R.DEV)),
                qt=(i8.codes_buffer(N, T, R.DEV), torch.zeros(N, device=R.DEV)),
                y=torch.zeros((T, N), dtype=d, device=R.DEV), dx=torch.zeros((T, K), dtype=d, device=R.DEV),
                dw=torch.zeros((N, K), device=R.DEV), back=padded(T, K, d),
                wq=self.space(i8.cfint8_quantize_workspace_bytes(T, N, 0)),
                wx=self.space(i8.cfint8_gemm_workspace_bytes(T, K, N, 1)),
                ww=self.space(i8.cfint8_gemm_workspace_bytes(N, K, T, 1))))
        self.moe = []
        for i, (T, E, topk, H, I, d) in enumerate(LAYERS):
            x, r, gu, gus, dn, dns = make(T, E, H, I, "bf16" if d == BF else "f32", seed)
            ops = [x.to(R.DEV), r.to(R.DEV)] + [torch.from_numpy(v).to(R.DEV) for v in (gu, gus, dn, dns)]
            out = dict(y=torch.zeros_like(ops[0]), ids=torch.zeros((T, topk), dtype=torch.int32, device=R.DEV),
                       weights=torch.zeros((T, topk), device=R.DEV),
                       workspace=self.space(i8.cfint8_moe_workspace_bytes(T, E, topk, H, I)))
            self.moe.append((ops, topk, out))

    @staticmethod
    def space(n):
        return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=R.DEV)

    def run(self, stream=None, own=True):
        """own: with the held workspaces; otherwise each call allocates what it needs."""
        for (T, N, K), o in zip(SIZES, self.lin):
            i8.cfint8_quantize(o["x"], codes=o["qx"][0], scales=o["qx"][1], stream=stream)
            i8.cfint8_dequantize(*o["qx"], T, K, dst=o["back"], stream=stream)
            i8.cfint8_gemm(*o["qx"], *o["w"], T, N, K, c=o["y"], stream=stream)
            i8.cfint8_quantize(o["g"], mul=o["w"][1], codes=o["qg"][0], scales=o["qg"][1], stream=stream)
            i8.cfint8_gemm(*o["qg"], o["w"][0], None, T, K, N, trans_b=1, c=o["dx"],
                           workspace=o["wx"] if own else None, stream=stream)
            i8.cfint8_quantize(o["g"], block_axis=0, mul=o["qx"][1], codes=o["qt"][0], scales=o["qt"][1],
                               workspace=o["wq"] if own else None, stream=stream)
            i8.cfint8_gemm(*o["qt"], o["qx"][0], None, N, K, T, trans_b=1, c=o["dw"],
                           workspace=o["ww"] if own else None, stream=stream)
        for ops, topk, out in self.moe:
            i8.cfint8_moe(*ops, topk, stream=stream,
                          **(out if own else {k: v for k, v in out.items() if k != "workspace"}))

    def outputs(self):
        for o in self.lin:
            yield from (*o["qx"], *o["qg"], *o["qt"], o["back"], o["y"], o["dx"], o["dw"])
        for _, _, out in self.moe:
            yield from (out["y"], out["ids"], out["weights"])

    def workspaces(self):
        for o in self.lin:
            yield from (o["wq"], o["wx"], o["ww"])
        for _, _, out in self.moe:
            yield out["workspace"]

    def new_inputs(self, seed):
        for i, o in enumerate(self.lin):
            o["x"].copy_(torch.from_numpy(normal(seed + i, *o["x"].shape)))
            o["g"].copy_(torch.from_numpy(normal(seed + 20 + i, *o["g"].shape)))
        for i, (ops, _, _) in enumerate(self.moe):
            ops[0].copy_(torch.from_numpy(normal(seed + 40 + i, *ops[0].shape)))

    def clear(self):
        for t in self.outputs():
            t.fill_(3)

    def snapshot(self):
        torch.cuda.synchronize()
        return [t.cpu().clone() for t in self.outputs()]


def same(a, b, what):
    for i, (p, q) in enumerate(zip(a, b)):
        assert torch.equal(p, q), f"{what}: output {i}"


def test_graph_replays():
    """One graph of all operators, replayed with new inputs in place and eager work and waits in between."""
    say("[int8 together] graph")
    work, eager = Work(0), Work(0)
    work.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work.run()
    for rep in range(4):
        say(f"[int8 together] replay {rep}")
        for o in (work, eager):
            o.new_inputs(100 * rep)
            o.clear()
        graph.replay()
        eager.run()
        same(work.snapshot(), eager.snapshot(), f"replay {rep}")


def test_graph_with_memory_of_its_own():
    """Outputs and workspaces allocated inside the capture; two such graphs replayed in turn."""
    say("[int8 together] graphs with their own memory")
    works, graphs, outs = [Work(0), Work(7)], [], []
    for w in works:
        w.run(own=False)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = w.lin[3]
            T, N, K = SIZES[3]
            qx, sx = i8.cfint8_quantize(o["x"])
            qt, st = i8.cfint8_quantize(o["g"], block_axis=0, mul=sx)
            dw = i8.cfint8_gemm(qt, st, qx, None, N, K, T, trans_b=1)
            y, ids, _ = i8.cfint8_moe(*w.moe[0][0], w.moe[0][1])
        graphs.append(g)
        outs.append((qx, sx, dw, y, ids))
    for rep in range(3):
        for w, g, out in zip(works, graphs, outs):
            w.new_inputs(11 + rep)
            w.run()
            g.replay()
            torch.cuda.synchronize()
            o = w.lin[3]
            same([t.cpu() for t in out], [t.cpu() for t in (*o["qx"], o["dw"].float(), w.moe[0][2]["y"],
                                                             w.moe[0][2]["ids"])], f"replay {rep}")


def test_streams():
    """Two streams at once, each with its own operands, workspaces held or allocated by the calls."""
    say("[int8 together] streams")
    works = [Work(0), Work(30)]
    want = []
    for w in works:
        w.run()
        want.append(w.snapshot())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for own in (True, False):
        for w in works:
            w.clear()
        torch.cuda.synchronize()
        for s, w in zip(streams, works):
            w.run(stream=s, own=own)
        for i, (s, w) in enumerate(zip(streams, works)):
            s.synchronize()
            same(w.snapshot(), want[i], f"stream {i}, held workspaces {own}")


def test_memory_allocated_for_another_stream():
    """What a call on a given stream allocates comes from that stream's memory: a block that the current stream has
    just given back, with its last writes still queued, is not handed out."""
    say("[int8 together] allocation on a stream")
    s = torch.cuda.Stream()
    x = matrix(normal(1, 512, 1024), F32)
    want = i8.cfint8_quantize(x)
    torch.cuda.synchronize()
    for _ in range(5):
        big = torch.randn((4096, 4096), device=R.DEV)
        late = torch.empty((512, 1024), dtype=torch.int8, device=R.DEV)
        for _ in range(4):
            big = big @ big * 1e-4
        late.fill_(1)
        del late
        got = i8.cfint8_quantize(x, stream=s)
        torch.cuda.synchronize()
        same([t.cpu() for t in got], [t.cpu() for t in want], "codes")


@pytest.mark.parametrize("word", [0, 0x7F7F, -1, -0x8000])      # the last: an exponent that stands for NaN
def test_workspaces_need_no_contents(word):
    say(f"[int8 together] workspaces of {word}")
    work = Work(0)
    work.run()
    want = work.snapshot()
    for t in work.workspaces():
        t.view(torch.int16).fill_(word)
    work.clear()
    work.run()
    same(work.snapshot(), want, "again")
    work.run()                                        # and what a call leaves in them
    same(work.snapshot(), want, "third")


def test_operands_inside_wider_buffers():
    """Columns of a tensor at any element offset for the other axis; a slice of experts; scales inside a vector."""
    say("[int8 together] views")
    base = torch.zeros(70 * 91 + 3, dtype=BF, device=R.DEV)
    v = base[3:3 + 70 * 91].view(70, 91)
    v.copy_(torch.from_numpy(normal(3, 70, 91)))
    view = v[:, 1:86]
    q, s = i8.cfint8_quantize(view, block_axis=0)
    want = R.quantize(view.float().cpu().numpy().T)
    assert np.array_equal(q.cpu().numpy(), want[0]) and np.array_equal(s.cpu().numpy(), want[1])
    scales = torch.zeros(100, device=R.DEV)
    q2, _ = i8.cfint8_quantize(view, block_axis=0, scales=scales[5:90])
    assert torch.equal(q2, q) and torch.equal(scales[5:90], s) and not bool(scales[:5].any() or scales[90:].any())
    x, r, gu, gus, dn, dns = make(3, 8, 64, 32, "bf16")
    d = [torch.from_numpy(t).to(R.DEV) for t in (gu, gus, dn, dns)]
    part = i8.cfint8_moe(x.to(R.DEV), r.to(R.DEV)[2:6], *(t[2:6] for t in d), 2)
    alone = i8.cfint8_moe(x.to(R.DEV), r.to(R.DEV)[2:6].clone(), *(t[2:6].clone() for t in d), 2)
    same([t.cpu() for t in part], [t.cpu() for t in alone], "slice of experts")
