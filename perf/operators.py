"""The operators on weight matrices, as cases that can be timed: each case is
one call that a program makes, with its plain form and its values in 64 bits.

A case is a dict of plain values.  Its ``kind`` names the operator:

  ns     newton_schulz: `batch` matrices of rows x cols brought near the nearest
         (semi-)orthogonal matrix by `steps` Newton-Schulz products
  muon   muon_update: momentum, the orthogonalised direction, the step, in place
  quant  quantize_rows: rows to 8-bit integers, each with its scale
  ip8    inner_product_int8: samples times a weight matrix of 8-bit rows

``own`` chooses between the plain form and the framework's entry points.  The
plain forms are elementary operations in 32 bits, in 64 where a value next to a
border decides (the rounding to 8 bits) or a long sum does (the norm).
"""
import math

import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)  # the quintic x -> a x + b x^3 + c x^5
EPS = 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01
ROW = 128  # 8-bit rows are padded with zeros to a multiple of this many bytes

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the second convolution of the LeNet example, 50 x (20 5 5): the
        # smallest call, where the latency of a launch is all there is
        dict(name="ns_lenet_conv2", kind="ns", dtype="f32", batch=1, rows=50, cols=500, steps=5),
        # a grouped convolution (conv4 of CaffeNet): each group's 192 x 1728 is
        # a matrix of its own, both in one call
        dict(name="ns_conv4_groups", kind="ns", dtype="f32", batch=2, rows=192, cols=1728, steps=5),
        # more rows than columns, no size round, bfloat16 in and out
        dict(name="ns_tall_odd_bf16", kind="ns", dtype="bf16", batch=1, rows=2305, cols=603,
             steps=5),
        # the first convolution of CaffeNet, 96 x (3 11 11)
        dict(name="muon_conv1", kind="muon", dtype="f32", batch=1, rows=96, cols=363, steps=5),
        # the last inner product of CaffeNet, an ordinary matrix
        dict(name="muon_fc8", kind="muon", dtype="f32", batch=1, rows=1000, cols=4096, steps=5),
        # the first inner product, the largest matrix of the network: 38 M
        # weights, all time goes to matrix products
        dict(name="muon_fc6", kind="muon", dtype="f32", batch=1, rows=4096, cols=9216, steps=5),
        # that matrix's weights made ready for the 8-bit product
        dict(name="quant_fc6_weight", kind="quant", dtype="f32", rows=4096, cols=9216),
        # a few samples' bfloat16 activations of odd length
        dict(name="quant_rows37_bf16", kind="quant", dtype="bf16", rows=37, cols=4095),
        # one sample through the first inner product: the stream of its weights
        dict(name="ip8_fc6_n1", kind="ip8", bottom="f32", top="f32", N=1, C=9216, K=4096,
             relu=True, bias=True),
        # the second inner product at the training batch, float in and out
        dict(name="ip8_fc7_n256", kind="ip8", bottom="f32", top="f32", N=256, C=4096, K=4096,
             relu=True, bias=True),
        # nothing round: samples, inputs and outputs, bfloat16 in and out
        dict(name="ip8_odd_bf16", kind="ip8", bottom="bf16", top="bf16", N=33, C=1003, K=507,
             relu=False, bias=True),
        # a scoring run over many samples already held in 8 bits
        dict(name="ip8_fc6_n8192", kind="ip8", bottom="int8", top="bf16", N=8192, C=9216, K=4096,
             relu=True, bias=False),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("ns", "ns", "muon", "muon", "quant", "ip8", "ip8", "ip8"))
    if kind in ("ns", "muon"):
        while True:
            batch = rng.choice((1, 1, 1, 2, 2, 4))
            a, b = _log(rng, 4, 4096), _log(rng, 16, 9216)
            if rng.random() < 0.3:
                a, b = b, a
            m, n = min(a, b), max(a, b)
            if m <= 4096 and batch * m * m * n <= 4096 * 4096 * 9216 and batch * a * b <= 4e7:
                return dict(kind=kind, dtype="f32" if kind == "muon" else
                            rng.choice(("f32", "f32", "bf16")), batch=batch, rows=a, cols=b,
                            steps=rng.choice((5, 5, 5, 3, 6)))
    if kind == "quant":
        while True:
            rows, cols = _log(rng, 1, 8192), _log(rng, 16, 16384)
            if rows * cols <= 4e7:
                return dict(kind=kind, dtype=rng.choice(("f32", "bf16")), rows=rows, cols=cols)
    while True:
        N, C, K = _log(rng, 1, 8192), _log(rng, 16, 9216), _log(rng, 10, 8192)
        if K * C <= 4e7 and N * max(C, K) <= 8e7:
            return dict(kind="ip8", bottom=rng.choice(("f32", "f32", "bf16", "int8")),
                        top=rng.choice(("f32", "bf16")), N=N, C=C, K=K, relu=rng.random() < 0.6,
                        bias=rng.random() < 0.8)


# ------------------------------------------------------------------- inputs
def _gradient(gen, batch, rows, cols):
    """A weight gradient: the sum over 64 samples of (output gradient) x
    (post-ReLU input), whose few directions carry most of it, and noise in the
    others, at the scale of a mean over a batch."""
    r = 64
    d = torch.randn((batch, rows, r), generator=gen, device="cuda")
    x = torch.randn((batch, r, cols), generator=gen, device="cuda").clamp_(min=0.0)
    e = torch.randn((batch, rows, cols), generator=gen, device="cuda")
    return torch.matmul(d, x).mul_(1.0 / r).add_(e, alpha=0.2).mul_(1e-3)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    if kind in ("ns", "muon"):
        shape = (case["batch"], case["rows"], case["cols"])
        g = _gradient(gen, *shape)
        if kind == "ns":
            return dict(case=case, g=g.to(_DT[case["dtype"]]))
        v = _gradient(gen, *shape).mul_(5.0)  # a history of several steps
        w = torch.randn(shape, generator=gen, device="cuda").mul_(0.005)
        return dict(case=case, g=g, v=v, w=w)
    if kind == "quant":
        x = torch.randn((case["rows"], case["cols"]), generator=gen, device="cuda").mul_(0.005)
        return dict(case=case, x=x.to(_DT[case["dtype"]]))
    N, C, K = case["N"], case["C"], case["K"]
    pitch = (C + ROW - 1) // ROW * ROW
    # weights as the quantiser leaves them: 8-bit rows with a scale each
    wq = torch.zeros((K, pitch), dtype=torch.int8, device="cuda")
    wq[:, :C] = torch.randn((K, C), generator=gen, device="cuda").mul_(30).round_().clamp_(-127, 127)
    ws = torch.rand(K, generator=gen, device="cuda").mul_(1e-4).add_(5e-5)
    b = torch.randn(K, generator=gen, device="cuda").mul_(0.1) if case["bias"] else None
    st = dict(case=case, wq=wq, ws=ws, b=b)
    # post-ReLU activations, about half of them zero
    x = torch.randn((N, C), generator=gen, device="cuda").clamp_(min=0.0)
    if case["bottom"] == "int8":
        st["xq"] = torch.zeros((N, pitch), dtype=torch.int8, device="cuda")
        st["xq"][:, :C] = x.mul_(40).round_().clamp_(max=127)
        st["xs"] = torch.rand(N, generator=gen, device="cuda").mul_(0.01).add_(0.02)
    else:
        st["x"] = x.to(_DT[case["bottom"]])
    return st


# ------------------------------------------------------------- plain forms
def _ns_plain(g, steps):
    a, b, c = COEF
    tall = g.shape[1] > g.shape[2]
    x = g.float()
    if tall:
        x = x.transpose(1, 2).contiguous()
    norm = (x * x).sum(dim=(1, 2), dtype=torch.float64).sqrt()
    x = x * (1.0 / (norm + EPS)).float()[:, None, None]
    for _ in range(steps):
        A = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * A + c * torch.matmul(A, A), x)
    return x.transpose(1, 2).contiguous() if tall else x


def _quant_plain(x):
    amax = x.float().abs().amax(1)
    scale = (amax.double() / 127.0).float()
    q = torch.round(x.double() / scale.double()[:, None])
    q = torch.where(scale[:, None] > 0, q, torch.zeros_like(q)).clamp(-127, 127)
    return q, scale


def _muon_scale(case):
    return math.sqrt(max(1.0, case["rows"] / case["cols"]))


def _run_plain(st):
    case = st["case"]
    if case["kind"] == "ns":
        return _ns_plain(st["g"], case["steps"]).to(_DT[case["dtype"]])
    if case["kind"] == "muon":
        w, g, v = st["w"], st["g"], st["v"]
        v.mul_(MOMENTUM).add_(g)
        o = _ns_plain(g + MOMENTUM * v, case["steps"])
        w.sub_(LR * (_muon_scale(case) * o + DECAY * w))
        return {"w": w, "v": v}
    if case["kind"] == "quant":
        q, scale = _quant_plain(st["x"])
        return {"q": q.to(torch.int8), "scale": scale}
    C = case["C"]
    if case["bottom"] == "int8":
        q, s = st["xq"][:, :C].float(), st["xs"]
    else:
        q, s = _quant_plain(st["x"])
        q = q.float()
    y = torch.matmul(q, st["wq"][:, :C].float().t()) * s[:, None] * st["ws"][None, :]
    if st["b"] is not None:
        y = y + st["b"]
    if case["relu"]:
        y = y.clamp(min=0.0)
    return y.to(_DT[case["top"]])


def _run_own(st):
    import paper_1408_5093_amd as lib

    case = st["case"]
    ws = st.setdefault("workspace", lib.Workspace())  # kept, as a program keeps it
    if case["kind"] == "ns":
        return lib.newton_schulz(st["g"], steps=case["steps"], coef=COEF, eps=EPS, ws=ws)
    if case["kind"] == "muon":
        lib.muon_update(st["w"], st["g"], st["v"], LR, momentum=MOMENTUM, weight_decay=DECAY,
                        nesterov=True, steps=case["steps"], coef=COEF, eps=EPS, ws=ws)
        return {"w": st["w"], "v": st["v"]}
    if case["kind"] == "quant":
        q, scale = lib.quantize_rows(st["x"])
        return {"q": q[:, :case["cols"]], "scale": scale}
    x, xs = (st["xq"], st["xs"]) if case["bottom"] == "int8" else (st["x"], None)
    return lib.inner_product_int8(x, st["wq"], st["ws"], st["b"], C=case["C"], x_scale=xs,
                                  relu=case["relu"], top_dtype=_DT[case["top"]], ws=ws)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The definitions in double precision: the iteration in the form
    X <- X (a I + (b I + c M) M) with M = X^T X of the narrower side, the
    8-bit rows from the quotients themselves."""
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("ns", "muon"):
        g = st["g"].double()
        if kind == "muon":
            v = MOMENTUM * st["v"].double() + g
            g = MOMENTUM * v + g
        a, b, c = COEF
        outs = []
        for x in g.unbind(0):
            wide = x.shape[1] > x.shape[0]
            x = (x.t() if wide else x) / (torch.linalg.vector_norm(x) + EPS)
            eye = torch.eye(x.shape[1], dtype=torch.float64, device=x.device)
            for _ in range(case["steps"]):
                M = x.t() @ x
                x = x @ (a * eye + (b * eye + c * M) @ M)
            outs.append(x.t() if wide else x)
        o = torch.stack(outs)
        if kind == "ns":
            return o
        w = st["w"].double()
        return {"w": w * (1 - LR * DECAY) - LR * _muon_scale(case) * o, "v": v}
    if kind == "quant":
        q, scale = _rows_exact(st["x"])
        return {"q": q.to(torch.int8), "scale": scale}
    if case["bottom"] == "int8":
        q, s = st["xq"][:, :case["C"]].double(), st["xs"].double()
    else:
        q, s = _rows_exact(st["x"])
    y = torch.addmm(torch.zeros(1, dtype=torch.float64, device=q.device), q * s[:, None],
                    (st["wq"][:, :case["C"]].double() * st["ws"].double()[:, None]).t())
    y = y if st["b"] is None else y + st["b"].double()
    return torch.where(y > 0, y, torch.zeros_like(y)) if case["relu"] else y


def _rows_exact(x):
    """Scales as they are stored, one float each, and the whole numbers next to
    the quotients, halves to the even one."""
    x = x.double()
    scale = (torch.maximum(x.max(1).values, -x.min(1).values) / 127.0).float().double()
    t = x / torch.where(scale == 0, torch.ones_like(scale), scale)[:, None]
    low = t.floor()
    d = t - low
    up = (d > 0.5) | ((d == 0.5) & (torch.remainder(low, 2) == 1))
    return (low + up) * (scale > 0)[:, None], scale


# --------------------------------------------------------------------- work
def work(case):
    kind = case["kind"]
    if kind in ("ns", "muon"):
        count = case["batch"] * case["rows"] * case["cols"]
        m, n = sorted((case["rows"], case["cols"]))
        s = case["steps"]
        # symmetric products by their half; either each step's three products,
        # or the iteration on the m x m matrix of X X^T and one product at the end
        each = s * (m * m * n + m * m * m + 2 * m * m * n)
        gram = m * m * n + (4 * s - 3) * m * m * m + 2 * m * m * n
        size = 20 if kind == "muon" else 2 * _DT[case["dtype"]].itemsize
        return {"bytes": count * size, "flops": case["batch"] * min(each, gram)}
    if kind == "quant":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": rows * cols * (_DT[case["dtype"]].itemsize + 1) + 4 * rows,
                "flops": 2 * rows * cols}
    N, C, K = case["N"], case["C"], case["K"]
    size = 1 if case["bottom"] == "int8" else _DT[case["bottom"]].itemsize
    return {"bytes": K * C + 4 * K + N * C * size + N * K * _DT[case["top"]].itemsize +
            (4 * K if case["bias"] else 0) + (4 * N if size == 1 else 0), "flops": 2 * N * C * K}
