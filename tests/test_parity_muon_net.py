"""The orthogonalised update and the 8-bit inner products where a network uses
them: training iterations of LeNet and of a net with a grouped convolution,
checked step by step on the tensors that the GPU consumed, the captured
iteration against the eager one, and scoring with 8-bit weights afterwards.
Tolerances: those of the operators' own tests."""
import numpy as np
import pytest
import torch

import oracle
import paper_1408_5093_amd as cc
from paper_1408_5093_amd import workloads as wl
from paper_1408_5093_amd.net import ConvStack, MuonTrainer
from helpers import TOL_F32, assert_close
from test_parity_int8 import check_top, ip_ref, rows_ref
from test_parity_muon import TOL, muon_ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
GROUPED = (wl.ConvLayer("conv", 8, 9, 9, 24, 3, 1, 1, 2, True),
           wl.ConvLayer("ip", 24 * 81, 1, 1, 10, 1, 1, 0, 1, False))


def _np(t):
    torch.cuda.synchronize()
    return t.detach().cpu().numpy().astype(np.float64)


def _lenet(N):
    inp = wl.lenet_train(N, 2)
    net = ConvStack(wl.LENET_NET, N, inp["W"], inp["b"], glue=wl.LENET_NET_GLUE)
    return inp["x"], inp["labels"], net


def _grouped(N):
    rng = np.random.default_rng(30)
    W = [(rng.standard_normal((L.K, L.C // L.g, L.k, L.k)) * 0.1).astype(np.float32)
         for L in GROUPED]
    b = [np.zeros(L.K, np.float32) for L in GROUPED]
    x = [rng.standard_normal((N, 8, 9, 9)).astype(np.float32) for _ in range(2)]
    y = [rng.integers(0, 10, N).astype(np.int32) for _ in range(2)]
    return x, y, ConvStack(GROUPED, N, W, b)


NETS = {"lenet": _lenet, "grouped": _grouped}


def _trainer(net):
    return MuonTrainer(net, weight_lr=0.02, weight_decay_w=0.01, policy="inv", base_lr=0.01)


@pytest.mark.parametrize("name", NETS)
def test_training_iterations(name):
    xs, ys, net = NETS[name](16)
    tr = _trainer(net)
    for it in range(2):
        print(f"{name} iteration {it}", flush=True)
        tr.forward_backward(torch.from_numpy(xs[it]).to(DEV), torch.from_numpy(ys[it]).to(DEV))
        W0, b0 = [_np(w) for w in net.W], [_np(b) for b in net.b]
        vW0, vb0 = [_np(v) for v in tr.vW], [_np(v) for v in tr.vb]
        dW, db = [_np(w) for w in net.dW], [_np(b) for b in net.db]
        lr = tr.update()
        for l, L in enumerate(net.layers):
            mats = (L.g, L.K // L.g, W0[l].size // L.K)
            scale = max(1.0, mats[1] / mats[2]) ** 0.5
            w_ref, v_ref, o = muon_ref(W0[l].reshape(mats), dW[l].reshape(mats),
                                       vW0[l].reshape(mats), 2 * lr, 0.95, 0.01, True, scale)
            err = np.linalg.norm(_np(net.W[l]).reshape(mats) - w_ref)
            step = 2 * lr * scale * np.linalg.norm(o)
            # (2 lr is formed in double here and rounded to float: 2^-24 of the step)
            assert err <= (TOL + 2.0 ** -23) * step + 2.0 ** -22 * (np.linalg.norm(W0[l]) + step)
            assert_close(_np(tr.vW[l]).reshape(mats), v_ref, TOL_F32, f"vW{l}")
            b_ref, vb_ref = oracle.sgd_step(b0[l], db[l], vb0[l], lr, 0.9, 5e-4)
            assert_close(_np(net.b[l]), b_ref, TOL_F32, f"b{l}")


@pytest.mark.parametrize("name", NETS)
def test_captured_iterations_are_the_eager_ones(name):
    xs, ys, net_e = NETS[name](16)
    _, _, net_g = NETS[name](16)
    tr_e, tr_g = _trainer(net_e), _trainer(net_g)
    xs = [torch.from_numpy(a).to(DEV) for a in xs]
    ys = [torch.from_numpy(a).to(DEV) for a in ys]
    xg, yg = xs[0].clone(), ys[0].clone()
    tr_g.capture(xg, yg)
    for it in range(4):
        print(f"{name} replay {it}", flush=True)
        tr_e.step(xs[it % 2], ys[it % 2])
        xg.copy_(xs[it % 2])
        yg.copy_(ys[it % 2])
        tr_g.replay()
        torch.cuda.synchronize()
        _ = torch.randn(1000, device=DEV).sum().item()
        for a, b in zip(net_e.W + net_e.b + tr_e.vW + tr_e.vb,
                        net_g.W + net_g.b + tr_g.vW + tr_g.vb):
            assert torch.equal(a, b)


@pytest.mark.parametrize("name", NETS)
@pytest.mark.parametrize("N", [1, 16, 70])
def test_scoring_in_8_bits_after_training(name, N):
    """Trained a little, then scored with 8-bit inner products: every layer on
    the input that it consumed; rows made again after a further step."""
    xs, ys, net = NETS[name](N)
    tr = _trainer(net)
    x, y = torch.from_numpy(xs[0]).to(DEV), torch.from_numpy(ys[0]).to(DEV)
    tr.step(x, y)
    plain = net.forward(x).clone()
    ips = [l for l, L in enumerate(net.layers) if L.H == 1]
    for again in range(2):
        assert net.quantize_inner_products() == ips
        net.forward(x)
        for l in ips:
            L = net.layers[l]
            q, s = rows_ref(_np(net.bottom[l]).reshape(N, L.C).astype(np.float32))
            p, t = rows_ref(_np(net.W[l]).reshape(L.K, L.C).astype(np.float32))
            check_top(net.top[l].view(N, L.K), *ip_ref(q, s, p, t, _np(net.b[l]), L.relu))
        if again == 0:
            # a row's rounding is off by half a scale at most: each product of a
            # sample's C terms by |x| t / 2 + |w| s / 2 + s t / 4
            L, l = net.layers[ips[-1]], ips[-1]
            if len(ips) == 1:
                xl, w = np.abs(_np(net.bottom[l]).reshape(N, L.C)), np.abs(_np(net.W[l]).reshape(L.K, L.C))
                s, t = xl.max(1) / 127, w.max(1) / 127
                bound = (xl.sum(1)[:, None] * t / 2 + w.sum(1) * s[:, None] / 2 +
                         L.C * s[:, None] * t / 4)
                diff = np.abs(_np(net.top[l]).reshape(N, L.K) - _np(plain).reshape(N, L.K))
                assert (diff <= 1.001 * bound + 1e-5).all()
            with pytest.raises(ValueError, match="8 bits"):
                tr.forward_backward(x, y)
            with torch.no_grad():
                for l in ips:
                    net.W[l].mul_(-0.5)


def test_bf16_network_scores_in_8_bits():
    """CaffeNet's last layers, bf16: the weights' rows from their bf16 values."""
    layers = (wl.ConvLayer("fc7", 512, 1, 1, 256, 1, 1, 0, 1, True),
              wl.ConvLayer("fc8", 256, 1, 1, 100, 1, 1, 0, 1, False))
    rng = np.random.default_rng(31)
    W = [(rng.standard_normal((L.K, L.C, 1, 1)) * 0.05).astype(np.float32) for L in layers]
    b = [rng.standard_normal(L.K).astype(np.float32) for L in layers]
    net = ConvStack(layers, 8, W, b, bf16=True)
    assert net.quantize_inner_products() == [0, 1]
    net.forward(torch.from_numpy(rng.standard_normal((8, 512, 1, 1)).astype(np.float32)).to(DEV))
    for l, L in enumerate(layers):
        q, s = rows_ref(_np(net.bottom[l]).reshape(8, L.C).astype(np.float32))
        p, t = rows_ref(_np(net.W[l].float()).reshape(L.K, L.C).astype(np.float32))
        check_top(net.top[l].view(8, L.K), *ip_ref(q, s, p, t, _np(net.b[l]), L.relu))


def test_rows_made_again_under_a_captured_forward():
    """The rows made again after a forward pass was captured: replays use the new
    ones, in the memory that the capture saw."""
    xs, _, net = NETS["lenet"](16)
    x = torch.from_numpy(xs[0]).to(DEV)
    ips = net.quantize_inner_products()
    net.forward(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        top = net.forward(x)
    held = [net.ws_int8.buf.data_ptr()] + [t.data_ptr() for l in ips for t in net.int8[l]]
    for it in range(3):
        for l in ips:
            net.W[l].mul_(-0.5)
        net.quantize_inner_products()
        assert held == [net.ws_int8.buf.data_ptr()] + [t.data_ptr() for l in ips
                                                       for t in net.int8[l]]
        want = net.forward(x).clone()
        top.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(top, want), it


@pytest.mark.parametrize("name", NETS)
def test_rows_made_on_the_stream_of_the_update(name):
    """Update, rows and scoring on one stream that is busy, nothing waited for, are
    the same calls on the current stream."""
    xs, ys, net = NETS[name](16)
    _, _, one = NETS[name](16)
    x, y = torch.from_numpy(xs[0]).to(DEV), torch.from_numpy(ys[0]).to(DEV)
    tr, tr1 = _trainer(net), _trainer(one)
    s = torch.cuda.Stream()
    busy = torch.randn((2048, 2048), device=DEV)
    ips = [l for l, L in enumerate(net.layers) if L.H == 1]
    tr1.step(x, y)
    want = []
    for it in range(2):  # (the second time over the first rows)
        assert one.quantize_inner_products() == ips
        want.append(one.forward(x).clone())
        for w in one.W:
            w.mul_(-0.5)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        cc.newton_schulz(busy)
    tr.step(x, y, stream=s)
    for it in range(2):
        assert net.quantize_inner_products(stream=s) == ips
        top = net.forward(x, stream=s)
        with torch.cuda.stream(s):
            got = top.clone()
            for w in net.W:
                w.mul_(-0.5)
            cc.newton_schulz(busy)
        s.synchronize()
        assert torch.equal(got, want[it]), it


def test_a_layer_that_has_no_8_bit_rows_changes_nothing():
    """The second layer's samples are longer than a row may be: refused, and the
    network is as it was."""
    C = (1 << 17) + 128
    layers = (wl.ConvLayer("one", 32, 1, 1, C, 1, 1, 0, 1, True),
              wl.ConvLayer("two", C, 1, 1, 3, 1, 1, 0, 1, False))
    rng = np.random.default_rng(32)
    W = [(rng.standard_normal((L.K, L.C, 1, 1)) * 0.05).astype(np.float32) for L in layers]
    net = ConvStack(layers, 4, W, [np.zeros(L.K, np.float32) for L in layers])
    x = torch.from_numpy(rng.standard_normal((4, 32, 1, 1)).astype(np.float32)).to(DEV)
    want = net.forward(x).clone()
    with pytest.raises(cc.CaffeError, match="C must be"):
        net.quantize_inner_products()
    assert net.int8 == [None, None]
    assert torch.equal(net.forward(x), want)


def _bf16_pair(N):
    """A fused max-pool and LRN that stage for the next convolution, and an inner product."""
    layers = (wl.ConvLayer("conv", 3, 17, 17, 16, 3, 1, 1, 1, True),
              wl.ConvLayer("conv2", 16, 8, 8, 32, 3, 1, 1, 1, True),
              wl.ConvLayer("ip", 32 * 64, 1, 1, 10, 1, 1, 0, 1, False))
    glue = {0: [("pool", dict(kernel=3, stride=2)),
                ("lrn", dict(size=5, alpha=1e-4, beta=0.75, k=1.0))]}
    rng = np.random.default_rng(33)
    W = [(rng.standard_normal((L.K, L.C // L.g, L.k, L.k)) * 0.1).astype(np.float32)
         for L in layers]
    b = [np.zeros(L.K, np.float32) for L in layers]
    x = rng.standard_normal((N, 3, 17, 17)).astype(np.float32)
    return torch.from_numpy(x).to(DEV), ConvStack(layers, N, W, b, glue=glue, bf16=True)


@pytest.mark.parametrize("name", [*NETS, "bf16"])
def test_back_to_the_float_weights(name):
    """Scored in 8 bits and taken back, a network gives and trains the bits of one
    that never was; the backward pass needs a float forward pass first."""
    if name == "bf16":
        (x, net), (_, never) = _bf16_pair(16), _bf16_pair(16)
    else:
        xs, _, net = NETS[name](16)
        never, x = NETS[name](16)[2], torch.from_numpy(xs[0]).to(DEV)
    want = never.forward(x).clone()
    g = torch.randn(want.shape, device=DEV)
    never.backward(g)
    ips = net.quantize_inner_products()
    scores = net.forward(x).clone()
    assert net.float_inner_products() == ips and net.float_inner_products() == []
    with pytest.raises(ValueError, match="8 bits"):
        net.backward(g)
    assert net.bottom_staged == never.bottom_staged
    assert net.lrn_stage_only == never.lrn_stage_only
    assert torch.equal(net.forward(x), want)
    net.backward(g)
    torch.cuda.synchronize()
    for a, b in zip(net.dW + net.db, never.dW + never.db):
        assert torch.equal(a, b)
    # and again in 8 bits, in the same rows
    assert net.quantize_inner_products() == ips
    assert torch.equal(net.forward(x), scores)
