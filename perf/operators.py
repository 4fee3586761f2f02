"""Performance cases of the 8-bit integer operators: the quantizer and its reconstruction, the product
with scales for each token and channel, and the mixture-of-experts layer for a few tokens.

A case is a dict of plain values; its "kind" is

quantize    rows (axis 1: a scale for each token or output channel) or columns (axis 0) of a matrix
            quantized, with or without a multiplier along the quantized axis, and reconstructed
product     codes times codes with both scales, in fp32 or bf16, with or without a bias, the second
            operand as [N][K] or (trans) as the [K][N] codes of another product
backward    both gradients of a linear layer from its codes: dY quantized along its rows and its
            columns with the forward scales folded in, then two products
moe         a mixture-of-experts layer with 8-bit weights: router, gate and up, down, weighted sum

``run`` makes the calls of ``paper_2608_10010_amd.cfint8`` where ``own`` is true and computes the same
in elementary torch operations where it is not.  ``exact`` is the definition in 64 bits.
"""

import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # decode: the one new token's activations, where only latency counts
        dict(name="quantize_token", kind="quantize", dtype="bf16", rows=1, cols=4096, axis=1, mul=False),
        # prefill of 8192 tokens, the input of a down projection
        dict(name="quantize_prefill", kind="quantize", dtype="bf16", rows=8192, cols=14336, axis=1, mul=False),
        # fp32 rows of odd width out of a wider buffer
        dict(name="quantize_odd", kind="quantize", dtype="f32", rows=1511, cols=5155, axis=1, mul=False),
        # a training step's output gradient along its columns, the tokens' scales folded in
        dict(name="quantize_columns", kind="quantize", dtype="bf16", rows=4096, cols=11008, axis=0, mul=True),
        # decode of one token through a gate/up projection
        dict(name="product_token", kind="product", M=1, N=14336, K=4096, out="bf16", bias=False, trans=False),
        # decode of a batch of 32 through a square layer with a bias
        dict(name="product_batch", kind="product", M=32, N=4096, K=4096, out="bf16", bias=True, trans=False),
        # a short prompt, every size odd, fp32 results
        dict(name="product_ragged", kind="product", M=333, N=6151, K=4099, out="f32", bias=True, trans=False),
        # the largest: the gate/up projection on 8192 tokens
        dict(name="product_prefill", kind="product", M=8192, N=14336, K=4096, out="bf16", bias=False, trans=False),
        # backward pass of an up-projection on 4096 tokens
        dict(name="backward", kind="backward", dtype="bf16", tokens=4096, N=11008, K=4096),
        # one token through a layer of 64 experts, 8 of them taken
        dict(name="moe_token", kind="moe", dtype="bf16", T=1, E=64, topk=8, H=2048, I=1024, renorm=True, padded=0),
        # few large experts, fp32 activations, a batch padded with two dead tokens
        dict(name="moe_f32", kind="moe", dtype="f32", T=7, E=16, topk=2, H=4096, I=2048, renorm=False, padded=2),
        # a batch of 64 tokens over 128 experts: nearly all of them are read
        dict(name="moe_batch", kind="moe", dtype="bf16", T=64, E=128, topk=8, H=2048, I=1024, renorm=True, padded=0),
    ]


_MAX_OPS = 2.0 * 8192 * 14336 * 4096
_MAX_ELEMENTS = 8192 * 14336
_MAX_EXPERT_WEIGHTS = 128 * 3 * 1024 * 2048


def draw(rng):
    """One more case: kinds, types, flags and (log-uniform) sizes of the ranges above."""
    def size(lo, hi, step=1):
        v = math.exp(rng.uniform(math.log(lo), math.log(hi + step)))
        return int(min(hi, max(lo, int(v / step) * step)))

    kind = rng.choice(["quantize", "quantize", "product", "product", "product", "backward", "moe", "moe"])
    if kind == "quantize":
        c = dict(kind=kind, dtype=rng.choice(["bf16", "f32"]), rows=size(1, 16384), cols=size(16, 14336),
                 axis=rng.choice([1, 1, 0]), mul=rng.choice([False, True]))
        c["rows"] = min(c["rows"], _MAX_ELEMENTS * 2 // (c["cols"] * _SIZE[c["dtype"]]))
        return c
    if kind == "product":
        c = dict(kind=kind, M=size(1, 8192), N=size(16, 14336), K=size(32, 14336), out=rng.choice(["bf16", "f32"]),
                 bias=rng.choice([False, True]), trans=rng.choice([False, False, True]))
        c["M"] = max(1, min(c["M"], int(_MAX_OPS / (2.0 * c["N"] * c["K"]))))
        return c
    if kind == "backward":
        return dict(kind=kind, dtype=rng.choice(["bf16", "f32"]), tokens=size(64, 4096), N=size(256, 11008),
                    K=size(256, 4096))
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), T=size(1, 64), E=size(4, 128), H=size(256, 4096, 16),
             I=size(256, 2048, 16), renorm=rng.choice([True, False]))
    c["topk"] = rng.randint(1, min(8, c["E"]))
    c["padded"] = rng.choice([0, 0, c["T"] // 4])
    c["E"] = max(c["topk"], min(c["E"], _MAX_EXPERT_WEIGHTS // (3 * c["H"] * c["I"])))
    return c


# ---------------------------------------------------------------- inputs

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _gen(seed, salt):
    g = torch.Generator(device=_device())
    g.manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFF)
    return g


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=_device(), dtype=torch.float32)


def _activation(rows, cols, seed, dtype):
    """Activations: N(0, 1) with 0.1% of the channels 20 times larger."""
    g = _gen(seed, 1)
    x = _randn((rows, cols), g)
    ch = torch.randperm(cols, generator=g, device=_device())[:max(1, round(0.001 * cols))]
    x[:, ch] *= 20.0
    return x.to(_DT[dtype])


def _gradient(rows, cols, seed, dtype):
    """Gradients: N(0, 1) with a scale of its own, exp(N(0, 2)), for each row (token)."""
    g = _gen(seed, 2)
    return (_randn((rows, cols), g) * torch.exp(2.0 * _randn((rows, 1), g))).to(_DT[dtype])


def _ceil16(n):
    return -(-n // 16) * 16


def _aligned(x):
    """The same matrix with rows of whole 16-byte pieces (a view of a wider buffer where it is odd)."""
    per = 16 // x.element_size()
    ld = -(-x.shape[1] // per) * per
    if ld == x.shape[1]:
        return x
    wide = torch.zeros((x.shape[0], ld), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _codes_buffer(rows, k):
    return torch.zeros((rows, _ceil16(k)), dtype=torch.int8, device=_device())[:, :k]


def _kept_codes(rows, k, g, std):
    """Codes and row scales of a Gaussian matrix, as a program holds a quantized operand."""
    codes, scales = _codes_buffer(rows, k), torch.empty(rows, device=_device())
    step = max(1, (1 << 26) // k)
    for r in range(0, rows, step):
        w = _randn((min(step, rows - r), k), g).mul_(std)
        s = w.abs().amax(dim=1).double().div_(127.0).float()
        codes[r:r + step] = torch.round(w.div_(s[:, None])).to(torch.int8)
        scales[r:r + step] = s
    return codes, scales


def prepare(case, seed):
    c = dict(case)
    kind, dev = c["kind"], _device()
    s = dict(c=c)
    if kind == "quantize":
        x = _gradient(c["rows"], c["cols"], seed, c["dtype"]) if c["axis"] == 0 else \
            _activation(c["rows"], c["cols"], seed, c["dtype"])
        s["x"] = _aligned(x)
        outer, k = (c["rows"], c["cols"]) if c["axis"] == 1 else (c["cols"], c["rows"])
        s["mul"] = torch.exp(_randn((k,), _gen(seed, 3))) * 0.01 if c["mul"] else None
        s["codes"], s["scales"] = _codes_buffer(outer, k), torch.empty(outer, device=dev)
        s["values"] = _aligned(torch.empty((outer, k), device=dev))
    elif kind == "product":
        M, N, K = c["M"], c["N"], c["K"]
        g = _gen(seed, 4)
        s["a"], s["a_scales"] = _kept_codes(M, K, g, 1.0)
        if c["trans"]:                          # the [K][N] codes of another product, its scales folded in
            s["b"], s["b_scales"] = _kept_codes(K, N, g, 0.02)[0], None
        else:
            s["b"], s["b_scales"] = _kept_codes(N, K, g, 0.02)
        s["bias"] = _randn((N,), g) if c["bias"] else None
        s["out"] = torch.empty((M, N), dtype=_DT[c["out"]], device=dev)
    elif kind == "backward":
        T, N, K = c["tokens"], c["N"], c["K"]
        g = _gen(seed, 5)
        s["dy"] = _aligned(_gradient(T, N, seed, c["dtype"]))
        s["x"], s["x_scales"] = _kept_codes(T, K, g, 1.0)
        s["w"], s["w_scales"] = _kept_codes(N, K, g, 0.02)
        s["g_rows"], s["g_cols"] = _codes_buffer(T, N), _codes_buffer(N, T)
        s["dx"], s["dw"] = torch.empty((T, K), device=dev), torch.empty((N, K), device=dev)
    else:
        T, E, H, I = c["T"], c["E"], c["H"], c["I"]
        g = _gen(seed, 6)
        s["x"] = _activation(T, H, seed, c["dtype"])
        s["router"] = (_randn((E, H), g) * (1.5 / math.sqrt(H))).to(_DT[c["dtype"]])
        gu, gus = _kept_codes(E * 2 * I, H, g, 0.02)
        dn, dns = _kept_codes(E * H, I, g, 0.02)
        s["gate_up"], s["gate_up_scales"] = gu.view(E, 2 * I, H), gus.view(E, 2 * I)
        s["down"], s["down_scales"] = dn.view(E, H, I), dns.view(E, H)
        s["active"] = None
        if c["padded"]:
            s["active"] = (torch.arange(T, device=dev) < T - c["padded"]).to(torch.uint8)
        s["y"] = torch.empty((T, H), dtype=_DT[c["dtype"]], device=dev)
    return s


# ---------------------------------------------------------------- the framework's calls

def _own_quantize(s):
    from paper_2608_10010_amd import cfint8
    c = s["c"]
    codes, scales = cfint8.cfint8_quantize(s["x"], block_axis=c["axis"], mul=s["mul"], codes=s["codes"],
                                           scales=s["scales"])
    outer, k = codes.shape
    return dict(values=cfint8.cfint8_dequantize(codes, scales, outer, k, dst=s["values"]), scales=scales)


def _own_product(s):
    from paper_2608_10010_amd import cfint8
    c = s["c"]
    return cfint8.cfint8_gemm(s["a"], s["a_scales"], s["b"], s["b_scales"], c["M"], c["N"], c["K"],
                              trans_b=int(c["trans"]), bias=s["bias"], c=s["out"])


def _own_backward(s):
    from paper_2608_10010_amd import cfint8
    c = s["c"]
    T, N, K = c["tokens"], c["N"], c["K"]
    qr, sr = cfint8.cfint8_quantize(s["dy"], mul=s["w_scales"], codes=s["g_rows"])
    dx = cfint8.cfint8_gemm(qr, sr, s["w"], None, T, K, N, trans_b=1, c=s["dx"])
    qc, sc = cfint8.cfint8_quantize(s["dy"], block_axis=0, mul=s["x_scales"], codes=s["g_cols"])
    dw = cfint8.cfint8_gemm(qc, sc, s["x"], None, N, K, T, trans_b=1, c=s["dw"])
    return dict(dx=dx, dw=dw)


def _own_moe(s):
    from paper_2608_10010_amd import cfint8
    c = s["c"]
    y, ids, weights = cfint8.cfint8_moe(s["x"], s["router"], s["gate_up"], s["gate_up_scales"], s["down"],
                                        s["down_scales"], c["topk"], renormalize=c["renorm"], active=s["active"],
                                        y=s["y"])
    return dict(y=y, ids=ids, weights=weights)


# ---------------------------------------------------------------- the plain forms

def _plain_quantize(x, axis, mul):
    v = x.float() if axis == 1 else x.float().t()
    if mul is not None:
        v = v * mul                              # held in 32 bits
    s = (v.abs().amax(dim=1).double() / 127.0).float()
    # the quotient in 64 bits: it is often next to a border between two codes
    q = torch.where(s[:, None] > 0, torch.round(v.double() / s.double()[:, None]), 0.0).clamp(-127, 127)
    return q.to(torch.int8), s


def _plain_product(a, sa, b, sb, trans, bias, dtype):
    bf = b.float()
    c = torch.matmul(a.float(), bf if trans else bf.t())
    c = c * sa[:, None]
    if sb is not None:
        c = c * sb
    if bias is not None:
        c = c + bias
    return c.to(dtype)


def _plain_moe(s):
    c, x = s["c"], s["x"]
    T, E, H, I, k = c["T"], c["E"], c["H"], c["I"], c["topk"]
    logits = torch.matmul(x.double(), s["router"].double().t()).float()      # which experts: next to a border
    order = torch.sort(logits, dim=1, descending=True, stable=True)          # ties: the lowest index first
    ids, top = order.indices[:, :k], order.values[:, :k]
    lead = top[:, :1]
    total = torch.exp((top if c["renorm"] else logits) - lead).sum(dim=1, keepdim=True)
    p = torch.exp(top - lead) / total
    xf = x.float()
    gu = torch.matmul(xf, s["gate_up"].reshape(E * 2 * I, H).float().t()).view(T, E, 2 * I) * s["gate_up_scales"]
    gate, up = gu[:, :, :I], gu[:, :, I:]
    h = gate / (1.0 + torch.exp(-gate)) * up                                  # of every expert
    out = torch.matmul(h.transpose(0, 1).contiguous(), s["down"].float().transpose(1, 2).contiguous())
    out = out * s["down_scales"][:, None, :]                                  # [E][T][H]
    taken = torch.zeros((T, E), device=x.device).scatter_(1, ids, p)
    y = (out * taken.t()[:, :, None]).sum(dim=0)
    ids = ids.to(torch.int32)
    if s["active"] is not None:
        dead = (s["active"] == 0)[:, None]
        y, p, ids = y.masked_fill(dead, 0.0), p.masked_fill(dead, 0.0), ids.masked_fill(dead, -1)
    return dict(y=y.to(x.dtype), ids=ids, weights=p)


def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        return dict(quantize=_own_quantize, product=_own_product, backward=_own_backward, moe=_own_moe)[kind](s)
    if kind == "quantize":
        q, sc = _plain_quantize(s["x"], c["axis"], s["mul"])
        return dict(values=q.float() * sc[:, None], scales=sc)
    if kind == "product":
        return _plain_product(s["a"], s["a_scales"], s["b"], s["b_scales"], c["trans"], s["bias"], _DT[c["out"]])
    if kind == "backward":
        qr, sr = _plain_quantize(s["dy"], 1, s["w_scales"])
        dx = _plain_product(qr, sr, s["w"], None, True, None, torch.float32)
        qc, sc = _plain_quantize(s["dy"], 0, s["x_scales"])
        dw = _plain_product(qc, sc, s["x"], None, True, None, torch.float32)
        return dict(dx=dx, dw=dw)
    return _plain_moe(s)


# ---------------------------------------------------------------- work

def _experts_taken(c):
    """Expected number of distinct experts that the live tokens take."""
    return c["E"] * (1.0 - (1.0 - c["topk"] / c["E"]) ** (c["T"] - c["padded"]))


def work(case):
    """Bytes: inputs read once, results written once, the experts that some token takes read once."""
    c = case
    if c["kind"] == "quantize":
        n = c["rows"] * c["cols"]
        outer, k = (c["rows"], c["cols"]) if c["axis"] == 1 else (c["cols"], c["rows"])
        return {"bytes": n * (_SIZE[c["dtype"]] + 5.0) + 4.0 * outer + (4.0 * k if c["mul"] else 0.0), "flops": 0.0}
    if c["kind"] == "product":
        M, N, K = c["M"], c["N"], c["K"]
        b = M * K + N * K + 4.0 * M + (0.0 if c["trans"] else 4.0 * N) + (4.0 * N if c["bias"] else 0.0)
        return {"bytes": b + M * N * _SIZE[c["out"]], "flops": 2.0 * M * N * K}
    if c["kind"] == "backward":
        T, N, K = c["tokens"], c["N"], c["K"]
        return {"bytes": T * N * _SIZE[c["dtype"]] + T * K + N * K + 4.0 * (T + N) + 4.0 * (T * K + N * K),
                "flops": 4.0 * T * N * K}
    T, E, H, I, k = c["T"], c["E"], c["H"], c["I"], c["topk"]
    e, live = _SIZE[c["dtype"]], c["T"] - c["padded"]
    b = _experts_taken(c) * (3.0 * I * H + 4.0 * (2 * I + H)) + E * H * e + 2.0 * T * H * e + 8.0 * T * k
    return {"bytes": b, "flops": live * (2.0 * E * H + k * 6.0 * I * H)}


# ---------------------------------------------------------------- the definition in 64 bits

def _lines64(x, mul):
    """Values of lines quantized along the last axis: (codes as float64, scales as float32)."""
    v = x.to(torch.float32)
    if mul is not None:
        v = v * mul.reshape(1, -1)               # the operator's definition holds this product in 32 bits
    v = v.to(torch.float64)
    s = torch.div(torch.max(torch.abs(v), dim=1).values, 127).to(torch.float32)   # and the scale too
    d = s.to(torch.float64).reshape(-1, 1)
    q = torch.where(d == 0, torch.zeros_like(v), v / torch.where(d == 0, torch.ones_like(d), d))
    return torch.clip(torch.round(q), -127, 127), s


def exact(case, seed):
    c = case
    if _device() == "cpu" and work(case)["flops"] > 2e11:
        return None
    s = prepare(case, seed)
    f64 = torch.float64
    if c["kind"] == "quantize":
        q, sc = _lines64(s["x"] if c["axis"] == 1 else s["x"].t(), s["mul"])
        return dict(values=q * sc.to(f64).reshape(-1, 1), scales=sc.to(f64))
    if c["kind"] == "product":
        a = s["a"].to(f64) * s["a_scales"].to(f64).reshape(-1, 1)
        b = s["b"].to(f64).t() if c["trans"] else s["b"].to(f64) * s["b_scales"].to(f64).reshape(-1, 1)
        y = torch.mm(a, b.t())
        return y if s["bias"] is None else y + s["bias"].to(f64)
    if c["kind"] == "backward":
        qr, sr = _lines64(s["dy"], s["w_scales"])
        qc, sc = _lines64(s["dy"].t(), s["x_scales"])
        return dict(dx=torch.mm(qr * sr.to(f64).reshape(-1, 1), s["w"].to(f64)),
                    dw=torch.mm(qc * sc.to(f64).reshape(-1, 1), s["x"].to(f64)))
    T, E, H, I, k = c["T"], c["E"], c["H"], c["I"], c["topk"]
    x = s["x"].to(f64)
    held = torch.mm(x, s["router"].to(f64).t()).to(torch.float32).to(f64)    # logits are held in 32 bits
    y, weights = torch.zeros((T, H), dtype=f64, device=x.device), torch.zeros((T, k), dtype=f64, device=x.device)
    chosen = torch.argsort(held, dim=1, descending=True, stable=True)[:, :k]
    live = torch.ones(T, dtype=torch.bool, device=x.device) if s["active"] is None else s["active"].bool()
    weights = torch.softmax(torch.gather(held, 1, chosen), dim=1) if c["renorm"] else \
        torch.gather(torch.softmax(held, dim=1), 1, chosen)
    weights = weights * live.to(f64).reshape(-1, 1)
    for e in range(E):
        hit = (chosen == e) & live.reshape(-1, 1)
        rows = torch.nonzero(hit.any(dim=1)).reshape(-1)
        if rows.numel() == 0:
            continue
        w13 = s["gate_up"][e].to(f64) * s["gate_up_scales"][e].to(f64).reshape(-1, 1)
        w2 = s["down"][e].to(f64) * s["down_scales"][e].to(f64).reshape(-1, 1)
        gu = torch.mm(x[rows], w13.t())
        h = gu[:, :I] * torch.sigmoid(gu[:, :I]) * gu[:, I:]
        y[rows] += torch.mm(h, w2.t()) * (weights * hit.to(f64)).sum(dim=1)[rows].reshape(-1, 1)
    return dict(y=y, ids=None, weights=weights)
