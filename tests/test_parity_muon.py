"""Newton-Schulz orthogonalisation and the update along it, against the
definitions in 64 bits (step by step, on the CPU).

Tolerance, in the 2-norm relative to the result's.  The operands hold 22 bits
(two half terms), a rounding error of at most 2^-23 of an element, and float
sums add 2^-24 of a partial sum at a time; in one product of unit operands
these make an error of at most about 2^-20 in the largest singular direction.
A segment lets errors of the Gram matrix grow at most 2^8 against a value that
stays below 1, so the worst direction of the worst matrix ends near
2^-20 * 2^8 = 2.4e-4 (HARD: matrices with singular values near zero in few
dimensions).  Where m directions share the rounding errors, they are
independent and each takes 1/sqrt(m) of them or less: 2^-16 (TOL, 1.5e-5) for
gradient-like matrices.  A bfloat16 result adds its own rounding, 2^-8 at the
most (TOL_BF16 = 2^-8 + TOL).
"""
import numpy as np
import pytest
import torch

import paper_1408_5093_amd as cc

pytestmark = pytest.mark.gpu
DEV = "cuda"
TOL, HARD = 2.0 ** -16, 2.0 ** -12
TOL_BF16 = 2.0 ** -8 + TOL
CUBIC = (1.5, -0.5, 0.0)


def ns_ref(g, steps, coef=cc.NS_COEF, eps=1e-7):
    a, b, c = (float(np.float32(v)) for v in coef)
    out = []
    for x in np.asarray(g, dtype=np.float64):
        tall = x.shape[0] > x.shape[1]
        x = x.T if tall else x
        n = np.sqrt((x * x).sum())
        x = x / (n + float(np.float32(eps))) if n else x
        for _ in range(steps):
            A = x @ x.T
            x = a * x + (b * A + c * (A @ A)) @ x
        out.append(x.T if tall else x)
    return np.stack(out)


def gradient(rng, batch, rows, cols, rank=8, noise=0.2):
    d = rng.standard_normal((batch, rows, rank))
    x = np.maximum(rng.standard_normal((batch, rank, cols)), 0)
    return ((d @ x / rank + noise * rng.standard_normal((batch, rows, cols))) * 1e-3).astype(
        np.float32)


def rel(got, ref):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape
    assert np.isfinite(got).all()
    return float(np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-300))


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


SIZES = [(1, 1, 1), (1, 1, 7), (1, 5000, 1), (2, 3, 5), (1, 20, 25), (3, 31, 33), (1, 50, 500),
         (3, 64, 64), (1, 65, 63), (1, 127, 513), (1, 1000, 33), (1, 128, 128), (1, 129, 65),
         (2, 129, 1000), (2, 192, 1728), (1, 130, 4100), (1, 257, 300), (4, 200, 210),
         (1, 500, 800), (1, 900, 640), (1, 16, 40000)]


@pytest.mark.parametrize("batch,rows,cols", SIZES)
def test_newton_schulz_float(batch, rows, cols):
    print(f"newton_schulz {batch}x{rows}x{cols}", flush=True)
    g = gradient(np.random.default_rng([1, batch, rows, cols]), batch, rows, cols)
    ref = ns_ref(g, 5)
    x = dev(g)
    assert rel(cc.newton_schulz(x), ref) <= TOL
    assert np.array_equal(x.cpu().numpy(), g)  # the input is left as it was


@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 9), (2, 50, 500), (1, 605, 603), (1, 1111, 300),
                                             (3, 100, 77), (1, 33, 130)])
def test_newton_schulz_bf16(batch, rows, cols):
    print(f"newton_schulz bf16 {batch}x{rows}x{cols}", flush=True)
    x = dev(gradient(np.random.default_rng([2, batch, rows, cols]), batch, rows, cols),
            torch.bfloat16)
    out = cc.newton_schulz(x)
    assert out.dtype == torch.bfloat16
    assert rel(out, ns_ref(x.double().cpu().numpy(), 5)) <= TOL_BF16


@pytest.mark.parametrize("coef,steps", [(cc.NS_COEF, 1), (cc.NS_COEF, 2), (cc.NS_COEF, 3),
                                        (cc.NS_COEF, 4), (cc.NS_COEF, 6), (cc.NS_COEF, 10),
                                        (CUBIC, 1), (CUBIC, 7), (CUBIC, 16),
                                        ((15 / 8, -10 / 8, 3 / 8), 9)])
@pytest.mark.parametrize("shape", [(2, 40, 90), (1, 150, 200)])
def test_newton_schulz_steps_and_coefficients(coef, steps, shape):
    print(f"newton_schulz {shape} {coef} x {steps}", flush=True)
    g = gradient(np.random.default_rng([3, steps]), *shape)
    assert rel(cc.newton_schulz(dev(g), steps, coef), ns_ref(g, steps, coef)) <= TOL


@pytest.mark.parametrize("n", [3, 40, 100, 160, 300])
def test_newton_schulz_hard_matrices(n):
    """Singular values that vanish or span nine decades, equal rows, an
    orthogonal matrix, a lower-triangular one."""
    rng = np.random.default_rng([4, n])
    q, _ = np.linalg.qr(rng.standard_normal((n, n)))
    u, _ = np.linalg.qr(rng.standard_normal((n, n)))
    mats = {"rank one": np.outer(rng.standard_normal(n), rng.standard_normal(n)),
            "orthogonal": q, "decades": (q * np.logspace(0, -9, n)) @ u,
            "equal rows": np.tile(rng.standard_normal(n), (n, 1)),
            "triangular": np.tril(rng.standard_normal((n, n)))}
    for name, g in mats.items():
        print(f"hard {n}: {name}", flush=True)
        g = g.astype(np.float32)[None]
        assert rel(cc.newton_schulz(dev(g)), ns_ref(g, 5)) <= HARD, name


def test_newton_schulz_scale_of_the_input():
    """The norm is taken in double: no scale of the floats over- or underflows
    it, and eps counts as it is defined (a norm far below eps leaves nothing:
    the operands' absolute accuracy is 2^-39)."""
    g = gradient(np.random.default_rng(5), 1, 60, 90)
    for s in (1e-30, 1e-8, 1.0, 1e20, 1e38):
        x = (g / np.abs(g).max() * np.float32(s)).astype(np.float32)
        if s > 1e-10:
            assert rel(cc.newton_schulz(dev(x)), ns_ref(x, 5)) <= TOL, s
        # at eps = 0 the direction alone counts
        assert rel(cc.newton_schulz(dev(x), eps=0.0), ns_ref(x, 5, eps=0.0)) <= TOL, s


@pytest.mark.parametrize("rows,cols", [(40, 70), (200, 260)])
def test_newton_schulz_zero_and_not_finite(rows, cols):
    """A zero matrix gives zeros, one with a NaN or infinity NaN everywhere; the
    others of the batch are as without them."""
    g = gradient(np.random.default_rng(6), 5, rows, cols)
    alone = cc.newton_schulz(dev(g))
    g[1] = 0
    g[2, 3, 4] = np.nan
    g[3, rows - 1, cols - 1] = np.inf
    for eps in (1e-7, 0.0):
        out = cc.newton_schulz(dev(g), eps=eps)
        assert (out[1] == 0).all()
        assert torch.isnan(out[2]).all() and torch.isnan(out[3]).all()
        if eps:
            assert torch.equal(out[0], alone[0]) and torch.equal(out[4], alone[4])


@pytest.mark.parametrize("rows,cols", [(60, 90), (300, 170)])
def test_newton_schulz_in_place_any_workspace_any_stream(rows, cols):
    """The same bits in place, on a workspace full of NaN, and on another
    stream."""
    g = gradient(np.random.default_rng(7), 2, rows, cols)
    first = cc.newton_schulz(dev(g))
    ws = cc.Workspace()
    ws.get(cc.newton_schulz_workspace_size(cc.ns_desc(g.shape))).fill_(255)
    x = dev(g)
    assert torch.equal(cc.newton_schulz(x, out=x, ws=ws), first)
    x = dev(g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(x)
    with torch.cuda.stream(s):
        cc.newton_schulz(x, out=out)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, first)
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    cc.newton_schulz(x, out=out, stream=s, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(out, first)


def ns_ref_gpu(g, steps):
    """ns_ref of one matrix with the device's double-precision products."""
    a, b, c = (float(np.float32(v)) for v in cc.NS_COEF)
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    x = x / (torch.linalg.vector_norm(x) + float(np.float32(1e-7)))
    for _ in range(steps):
        A = x @ x.t().contiguous()
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.t() if tall else x


# sizes from which the products take tiles of 128, 192 and 256 x 192, round and
# odd, tall and wide
LARGE = [(2600, 2601), (3400, 3300), (1500, 7001), (4090, 4100), (4097, 3900), (4080, 9101),
         (9100, 4080)]


@pytest.mark.parametrize("rows,cols", LARGE)
def test_newton_schulz_large(rows, cols):
    print(f"newton_schulz {rows}x{cols}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(rows + cols)
    d = torch.randn((rows, 64), generator=gen, device=DEV)
    x = torch.randn((64, cols), generator=gen, device=DEV)
    g = (d @ x / 64 + 0.2 * torch.randn((rows, cols), generator=gen, device=DEV)) * 1e-3
    o = cc.newton_schulz(g)
    ref = ns_ref_gpu(g, 5)
    norm = torch.linalg.vector_norm(ref)
    assert float(torch.linalg.vector_norm(o.double() - ref) / norm) <= TOL
    # the update along it, from a zero history: u = (1 + momentum) g
    w = torch.randn((rows, cols), generator=gen, device=DEV) * 0.01
    w0, v = w.double(), torch.zeros_like(g)
    cc.muon_update(w, g, v, 0.5, weight_decay=0.1, scale=0.3)
    assert torch.equal(v, g)
    want = w0 - 0.5 * (float(np.float32(0.3)) * ref + float(np.float32(0.1)) * w0)
    err = float(torch.linalg.vector_norm(w.double() - want))
    # eps counts against 1.95 times the norm here: 1e-7 / ||g|| more, ||g|| > 0.1
    step = 0.15 * float(norm)
    assert err <= (TOL + 1e-6) * step + 2.0 ** -22 * (float(torch.linalg.vector_norm(w0)) + step)
    ob = cc.newton_schulz(g.bfloat16())
    rb = ns_ref_gpu(g.bfloat16(), 5)
    assert float(torch.linalg.vector_norm(ob.double() - rb) / norm) <= TOL_BF16


@pytest.mark.parametrize("batch,rows,cols", [(3000, 4, 4), (300, 33, 20), (200, 20, 700),
                                             (40, 129, 130)])
def test_newton_schulz_many_matrices(batch, rows, cols):
    print(f"newton_schulz {batch} x {rows}x{cols}", flush=True)
    g = gradient(np.random.default_rng([11, rows]), batch, rows, cols)
    out = cc.newton_schulz(dev(g))
    pick = [0, 1, batch // 2, batch - 1]
    ref = ns_ref(g[pick], 5)
    # (four by four: singular values may vanish in few dimensions)
    assert rel(out[pick], ref) <= (HARD if rows == 4 else TOL)
    assert torch.isfinite(out).all()
    # alone it may take other tiles, whose sums run in another order
    one = cc.newton_schulz(dev(g[batch - 1]))
    assert rel(one, ref[3]) <= (HARD if rows == 4 else TOL)


def muon_ref(w, g, v, lr, mu, wd, nesterov, scale, steps=5):
    f = lambda t: float(np.float32(t))  # noqa: E731
    w, g, v = (np.asarray(t, dtype=np.float64) for t in (w, g, v))
    v = f(mu) * v + g
    o = ns_ref(g + f(mu) * v if nesterov else v, steps)
    return w - f(lr) * (f(scale) * o + f(wd) * w), v, o


@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 3), (1, 50, 500), (2, 75, 31), (1, 300, 140),
                                             (2, 130, 333)])
@pytest.mark.parametrize("nesterov,wd", [(True, 0.01), (False, 0.0)])
def test_muon_update(batch, rows, cols, nesterov, wd):
    print(f"muon {batch}x{rows}x{cols}", flush=True)
    rng = np.random.default_rng([8, batch, rows, cols])
    g, v = gradient(rng, batch, rows, cols), 3 * gradient(rng, batch, rows, cols)
    w = (rng.standard_normal(g.shape) * 0.05).astype(np.float32)
    wt, gt, vt = dev(w), dev(g), dev(v)
    cc.muon_update(wt, gt, vt, 0.02, 0.95, wd, nesterov)
    scale = max(1.0, rows / cols) ** 0.5
    w_ref, v_ref, o = muon_ref(w, g, v, 0.02, 0.95, wd, nesterov, scale)
    # v: a product and a sum, two roundings of 2^-24 of |mu v| + |g|
    assert (np.abs(vt.cpu().numpy() - v_ref) <= 2.0 ** -23 * (0.95 * np.abs(v) + np.abs(g))).all()
    # w: the step's error, and three roundings of 2^-24 of |w| + the step
    err = np.linalg.norm(wt.double().cpu().numpy() - w_ref)
    step = 0.02 * scale * np.linalg.norm(o)
    assert err <= TOL * step + 2.0 ** -22 * (np.linalg.norm(w) + step)
    assert np.array_equal(gt.cpu().numpy(), g)


def test_muon_update_of_a_grouped_convolution():
    """A (K, C/group, kh, kw) blob: each group's filters are one matrix."""
    rng = np.random.default_rng(9)
    shape = (24, 6, 3, 3)
    g = gradient(rng, 2, 12, 54).reshape(shape)
    w = rng.standard_normal(shape).astype(np.float32)
    wt, vt = dev(w), torch.zeros(shape, device=DEV)
    cc.muon_update(wt, dev(g), vt, 0.1, 0.9, scale=0.5, group=2)
    w_ref, _, _ = muon_ref(w.reshape(2, 12, 54), g.reshape(2, 12, 54), np.zeros((2, 12, 54)), 0.1,
                           0.9, 0.0, True, 0.5)
    assert rel(wt, w_ref.reshape(shape)) <= TOL


@pytest.mark.parametrize("rows,cols", [(50, 500), (260, 150)])
def test_muon_update_captured(rows, cols):
    """A captured update follows the rate in device memory, replay after
    replay, with eager work between, bit for bit the eager update."""
    rng = np.random.default_rng(10)
    g, w = gradient(rng, 1, rows, cols), rng.standard_normal((1, rows, cols)).astype(np.float32)
    we, ve, wg, vg = dev(w), torch.zeros(w.shape, device=DEV), dev(w), torch.zeros(w.shape,
                                                                                    device=DEV)
    gt, lr = dev(g), torch.empty(1, device=DEV)
    ws = cc.Workspace()
    ws.get(cc.newton_schulz_workspace_size(cc.ns_desc(w.shape)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cc.muon_update(wg, gt, vg, lr, weight_decay=0.01, ws=ws)
    for it in range(4):
        rate = 0.1 / (it + 1)
        cc.muon_update(we, gt, ve, rate, weight_decay=0.01)
        lr.fill_(rate)
        graph.replay()
        torch.cuda.synchronize()
        _ = torch.randn(1000, device=DEV).sum().item()
        assert torch.equal(we, wg) and torch.equal(ve, vg), it


def test_two_streams_at_once():
    """Calls on two streams with a workspace each, small and tiled matrices, are
    the calls one after the other."""
    rng = np.random.default_rng(12)
    gs = [dev(gradient(rng, 2, r, c)) for r, c in ((40, 700), (300, 400), (30, 50), (700, 640))]
    want = [cc.newton_schulz(g) for g in gs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [cc.Workspace() for _ in range(2)]
    size = max(cc.newton_schulz_workspace_size(cc.ns_desc(g.shape)) for g in gs)
    for w in spaces:
        w.get(size)
    outs = [[torch.empty_like(g) for g in gs] for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for k, g in enumerate(gs):
            for s, w, o in zip(streams, spaces, outs):
                cc.newton_schulz(g, out=o[k], ws=w, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        for a, b in zip(o, want):
            assert torch.equal(a, b)


def test_graphs_that_share_a_workspace():
    """Two captured updates on one workspace, replayed in turn, are the eager
    ones in turn (nothing is kept in a workspace between calls)."""
    rng = np.random.default_rng(13)
    shapes = [(1, 60, 300), (1, 260, 200)]
    ws = cc.Workspace()
    ws.get(max(cc.newton_schulz_workspace_size(cc.ns_desc(s)) for s in shapes))
    g = [dev(gradient(rng, *s)) for s in shapes]
    eager = [[dev(rng.standard_normal(s)), torch.zeros(s, device=DEV)] for s in shapes]
    mine = [[w.clone(), v.clone()] for w, v in eager]
    torch.cuda.synchronize()
    graphs = []
    for k in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            cc.muon_update(mine[k][0], g[k], mine[k][1], 0.1, ws=ws)
    for it in range(4):
        for k in (it % 2, 1 - it % 2):
            graphs[k].replay()
            cc.muon_update(eager[k][0], g[k], eager[k][1], 0.1)
        torch.cuda.synchronize()
        for k in range(2):
            assert torch.equal(mine[k][0], eager[k][0]) and torch.equal(mine[k][1], eager[k][1])


def test_muon_update_refuses():
    x = torch.zeros(4, 8, device=DEV)
    with pytest.raises(ValueError, match="contiguous"):
        cc.newton_schulz(torch.zeros(8, 4, device=DEV).t())
    with pytest.raises(ValueError, match="same shape"):
        cc.muon_update(x, x.clone(), torch.zeros(8, 4, device=DEV), 0.1)
    with pytest.raises(ValueError, match="one element"):
        cc.muon_update(x, x.clone(), x.clone(), torch.zeros(2, device=DEV))
    with pytest.raises(ValueError, match="float32"):
        cc.muon_update(x, x.bfloat16(), x.clone(), 0.1)
    with pytest.raises(cc.CaffeError, match="ALIGN"):
        cc.newton_schulz(torch.zeros(33, device=DEV)[1:].view(4, 8))


def test_memory_of_a_call_belongs_to_its_stream(monkeypatch):
    """With stream=, the workspace that a call drops again and its outputs are
    that stream's memory: the current stream is not given them while the call
    may still run."""
    taken = []
    get = cc.Workspace.get

    def noted(self, nbytes):
        buf = get(self, nbytes)
        taken.append((buf.data_ptr(), buf.numel()))
        return buf

    monkeypatch.setattr(cc.Workspace, "get", noted)
    rng = np.random.default_rng(14)
    g = dev(gradient(rng, 2, 300, 400))
    x = dev(rng.standard_normal((40, 900)))
    w, v = g.clone(), torch.zeros_like(g)
    q, t = cc.quantize_rows(x)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [cc.newton_schulz(g, stream=s), cc.inner_product_int8(x, q, t, stream=s),
            *cc.quantize_rows(x, stream=s)]
    cc.muon_update(w, g, v, 0.1, stream=s)
    assert len(taken) == 3
    mine = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2) for _, n in taken]
    for a, n in taken:
        for b in mine:
            assert b.data_ptr() + b.numel() <= a or a + n <= b.data_ptr()
    torch.cuda.synchronize()
    w2, v2 = g.clone(), torch.zeros_like(g)
    cc.muon_update(w2, g, v2, 0.1)
    for a, b in zip(outs + [w, v], [cc.newton_schulz(g), cc.inner_product_int8(x, q, t), q, t,
                                    w2, v2]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("shape", [(2, 20, 30), (1, 132, 200)])
def test_blobs_next_to_each_other(shape):
    """Blobs without a gap between them do not overlap."""
    rng = np.random.default_rng(15)
    g = gradient(rng, *shape)
    near = torch.zeros(4, *shape, device=DEV)
    near[0], near[2] = 1.0, dev(g)
    w, v = torch.ones(shape, device=DEV), torch.zeros(shape, device=DEV)
    cc.muon_update(w, dev(g), v, 0.1)
    cc.muon_update(near[0], near[2], near[1], 0.1)
    cc.newton_schulz(near[2], out=near[3])
    assert torch.equal(near[0], w) and torch.equal(near[1], v)
    assert torch.equal(near[2], dev(g)) and torch.equal(near[3], cc.newton_schulz(dev(g)))


SMALL_SEGMENTS_TILES = [(1, 20, 30), (2, 50, 500), (1, 192, 300)]  # one launch, slabs, tiles


@pytest.mark.parametrize("shape", SMALL_SEGMENTS_TILES)
@pytest.mark.parametrize("coef,steps", [((1.0, 1e-9, 0.0), 5), ((1.0, 1e-9, 0.0), 64),
                                        ((1.0, 1e-30, 1e-30), 7), ((1.0, 2e-9, 0.0), 5)])
def test_coefficients_next_to_the_identity(shape, coef, steps):
    """|q| just above 1, where steps of any number make one segment."""
    print(f"next to the identity {shape} {coef} x {steps}", flush=True)
    g = gradient(np.random.default_rng([16, steps]), *shape)
    x = dev(g)
    out = cc.newton_schulz(x, steps, coef, out=torch.full_like(x, float("nan")))
    assert rel(out, ns_ref(g, steps, coef)) <= TOL
    w, v = torch.zeros_like(x), torch.zeros_like(x)
    cc.muon_update(w, x, v, 1.0, 0.0, nesterov=False, scale=1.0, steps=steps, coef=coef)
    assert rel(-w, ns_ref(g, steps, coef)) <= TOL and torch.equal(v, x)


@pytest.mark.parametrize("shape", SMALL_SEGMENTS_TILES)
@pytest.mark.parametrize("c", [1e-17, -1e-25])
def test_range_of_coefficients_with_a_vanishing_third(shape, c):
    """t (2.9 - 2.9 t)^2 is largest inside [0, 1] (1.25) and vanishes at both ends."""
    print(f"vanishing third {shape} {c}", flush=True)
    g = gradient(np.random.default_rng(17), *shape, rank=1, noise=0.5)
    coef = (2.9, -2.9, c)
    assert rel(cc.newton_schulz(dev(g), 2, coef), ns_ref(g, 2, coef)) <= TOL


@pytest.mark.parametrize("shape", SMALL_SEGMENTS_TILES)
@pytest.mark.parametrize("coef,steps", [((0.1, 0.02, 0.0), 20), ((0.25, 0.0, 0.0), 40),
                                        ((0.01, 0.0, 0.0), 12)])
def test_coefficients_that_shrink(shape, coef, steps):
    """Products of q down to 2^-96 keep the operands' bits."""
    print(f"shrinking {shape} {coef} x {steps}", flush=True)
    g = gradient(np.random.default_rng([18, steps]), *shape)
    assert rel(cc.newton_schulz(dev(g), steps, coef), ns_ref(g, steps, coef)) <= TOL


def test_workspace_grown_on_another_stream():
    """A kept workspace that a call on another stream replaces by a larger one: the
    first stream is not given its memory while that stream still works."""
    rng = np.random.default_rng(19)
    small, large = dev(gradient(rng, 1, 40, 700)), torch.randn((2048, 2048), device=DEV)
    want = cc.newton_schulz(small), cc.newton_schulz(large)
    ws, s = cc.Workspace(), torch.cuda.Stream()
    cc.newton_schulz(small, ws=ws)
    torch.cuda.synchronize()
    at, n = ws.buf.data_ptr(), ws.buf.numel()
    outs = [torch.empty_like(large) for _ in range(10)]
    out = torch.empty_like(small)
    torch.cuda.synchronize()
    busy = cc.Workspace()
    for o in outs:
        cc.newton_schulz(large, out=o, ws=busy, stream=s)
    cc.newton_schulz(small, out=out, ws=ws, stream=s)
    cc.newton_schulz(large, out=outs[0], ws=ws, stream=s)  # grows
    mine = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(4)]
    still = not s.query()  # (a host held up for tens of ms proves nothing)
    torch.cuda.synchronize()
    assert ws.buf.numel() > n
    for t in mine if still else ():
        assert t.data_ptr() + n <= at or at + n <= t.data_ptr()
    assert torch.equal(out, want[0])
    for o in outs:
        assert torch.equal(o, want[1])


def test_workspace_grown_after_a_capture():
    """A larger call after a capture on the same workspace: replays write neither
    what was allocated since nor read it."""
    rng = np.random.default_rng(20)
    small, large = dev(gradient(rng, 1, 40, 700)), dev(gradient(rng, 1, 700, 900))
    x, out, ws = small.clone(), torch.empty_like(small), cc.Workspace()
    cc.newton_schulz(x, out=out, ws=ws)
    torch.cuda.synchronize()
    n = ws.buf.numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cc.newton_schulz(x, out=out, ws=ws)
    cc.newton_schulz(large, ws=ws)
    assert ws.buf.numel() > n
    mine = [torch.full((n,), 255, dtype=torch.uint8, device=DEV) for _ in range(8)]
    for it in range(3):
        x.copy_(small * (it + 1))
        out.zero_()
        graph.replay()
        eager = cc.newton_schulz(x)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), it
        assert all(int((t != 255).sum()) == 0 for t in mine), it
