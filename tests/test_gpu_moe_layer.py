"""The example's mixture-of-experts layer on the GPU: its wiring against a plain layer in 64 bits, training that gets better, serving,
and a whole training step captured into a graph."""
import importlib.util
import os

import pytest
import torch

import paper_2507_16099_amd as fp8

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def moe():
    spec = importlib.util.spec_from_file_location("moe_layer_example", os.path.join(ROOT, "examples", "moe_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _x(T, dim, seed):
    return torch.randn((T, dim), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _off(got, want):
    return ((got.cpu().double() - want).norm() / want.norm()).item()


def _plain(layer, x, dout):
    """The layer and its gradients by autograd in float64, on the CPU."""
    wr, w1, w2, xd = (t.detach().cpu().double().requires_grad_() for t in (*layer.params, x))
    logits = xd @ wr.T
    top = layer.kept[2][1].cpu().long()      # the experts that were chosen (in float32; close logits may order otherwise in 64 bits)
    gates = torch.gather(torch.softmax(logits, 1), 1, top)
    gates = gates / gates.sum(1, keepdim=True)
    out = torch.zeros_like(xd)
    for e in range(w1.shape[0]):
        y = torch.nn.functional.silu(xd @ w1[e].T) @ w2[e].T
        out = out + y * (gates * (top == e)).sum(1, keepdim=True)
    out.backward(dout.cpu().double())
    return out.detach(), [t.grad for t in (wr, w1, w2, xd)]


@pytest.mark.parametrize("T,dim,hidden,E,k", [(300, 128, 256, 8, 2), (1, 64, 96, 4, 1), (77, 256, 144, 24, 5)])
def test_layer_and_gradients(moe, T, dim, hidden, E, k):
    layer = moe.MoeLayer(dim, hidden, E, k, seed=T)
    x, dout = _x(T, dim, 5), _x(T, dim, 6)
    out = layer.forward(x.cuda())
    dx = layer.backward(dout.cuda())
    want, grads = _plain(layer, x, dout)
    # a code is off by at most half a step: 2^-4 of its value in e4m3, 2^-3 in e5m2; bf16 roundings, 2^-8 each, are a tenth of that.
    # Forward products take two e4m3 operands, backward ones an e5m2 and an e4m3; what a tensor has come through adds up
    # (silu keeps a relative error to within 1.1): out two forward products, dW2 one and its own, dW1, dX and the router's one or two of
    # each kind.
    fwd, bwd = 2 * 2 ** -4, 2 ** -3 + 2 ** -4
    assert _off(out, want) < 1.1 * fwd + fwd
    assert _off(layer.grads[2], grads[2]) < 1.1 * fwd + bwd
    for got, ref in ((layer.grads[1], grads[1]), (dx, grads[3])):
        assert _off(got, ref) < 1.1 * fwd + 2 * bwd
    if k > 1:      # (the gates of one expert, normalised, have no gradient)
        # dgates = <dout, y>, whose y is off by 2 forward products; the renormalised softmax takes differences of them
        assert _off(layer.grads[0], grads[0]) < 2 * (1.1 * fwd + fwd)
    else:
        assert layer.grads[0].abs().max() < 1e-6


def test_training_lowers_the_loss_and_serving_agrees(moe):
    layer = moe.MoeLayer(128, 256, 8, 2, seed=3)
    x = _x(512, 128, 1).cuda()
    losses = moe.train(layer, x, torch.tanh(x.float().roll(1, 1)), 40, 3e-3)
    assert losses[-1] < 0.6 * losses[0] and all(l == l for l in losses)
    layer.freeze()
    for n in (1, 3, 64, 512):
        served, want = layer.serve(x[:n]).double(), layer.forward(x[:n]).double()
        # the same codes; sums in another order, whose bf16 rounding can move a code of the second product
        assert ((served - want).norm() / want.norm()).item() < 2 ** -6


def test_a_captured_training_step(moe):
    """Forward, backward and the optimizer's launch recorded once: every replay equals the same step run eagerly."""
    make = lambda: moe.MoeLayer(128, 256, 8, 2, seed=9)
    x, dout = _x(200, 128, 2).cuda(), _x(200, 128, 4).cuda()
    layer, eager = make(), make()
    layer.optimizer(), eager.optimizer()

    def step(l):
        out = l.forward(x)
        dx = l.backward(dout)
        fp8.fp8_adamw_step(l.adamw, 1e-3, 1)
        return out, dx

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(layer), step(eager)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, dx = step(layer)
    for _ in range(4):
        graph.replay()
        want = step(eager)
        torch.cuda.synchronize()
        for a, b in ((out, want[0]), (dx, want[1]), *zip(layer.params, eager.params), *zip(layer.grads, eager.grads)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
