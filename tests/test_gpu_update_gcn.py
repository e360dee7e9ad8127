"""The update phase's operators together, as a node classifier uses them."""
import numpy as np
import pytest
import torch

import paper_2210_10737_amd as rsc
import synth
from paper_2210_10737_amd.gcn import GCNClassifier, RscConfig

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu(gpu):
    yield


def setup(cfg, feats=30, hidden=64, classes=41, layers=2):
    A = synth.make_graph("tiny", 0)
    X = torch.from_numpy(synth.dense_normal(A.n, feats, seed=1)).cuda()
    t = torch.from_numpy(np.random.default_rng(3).integers(0, classes, A.n)).cuda()
    t[::3] = -100
    model = GCNClassifier(rsc.DeviceCsr.from_host(A.rowptr, A.col, A.val, A.n), feats, hidden, classes, cfg, layers)
    return A, X, t, model


def test_gradients_of_the_exact_step():
    """Against autograd in 64 bits on the dense operand. The ReLUs' masks come
    from the fp32 activations (a sum next to zero may change sides). Errors:
    three products and two aggregations deep, fewer than 2,000 roundings of
    2^-24 in all, so 1.2e-4 of the gradient's largest value bounds them."""
    A, X, t, model = setup(RscConfig(enabled=False))
    loss = model.train_step(X, t, None, 0)
    dense = torch.zeros((A.n, A.n), dtype=torch.float64, device="cuda")
    row = torch.from_numpy(np.repeat(np.arange(A.n), np.diff(A.rowptr))).cuda()
    dense[row, torch.from_numpy(A.col).long().cuda()] = torch.from_numpy(A.val).double().cuda()
    with torch.no_grad():
        H = [rsc.linear(X, model.weights[0], model.biases[0], act="relu")]
        for agg, W, b in zip(model.aggregations, model.weights[1:], model.biases[1:]):
            H.append(rsc.linear(agg.plan.run(H[-1]), W, b, residual=H[-1], act="relu"))
    ws = [w.detach().double().requires_grad_() for w in model.weights]
    bs = [b.detach().double().requires_grad_() for b in model.biases]
    h = (X.double() @ ws[0] + bs[0]) * (H[0] > 0)
    for i in (1, 2):
        h = ((dense @ h) @ ws[i] + bs[i] + h) * (H[i] > 0)
    z = h @ ws[3] + bs[3]
    keep = t != -100
    want = (torch.logsumexp(z, 1) - z.gather(1, t.clamp_min(0)[:, None])[:, 0])[keep].mean()
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= 1e-5 * float(want.detach())
    for got, ref in list(zip(model.weights, ws)) + list(zip(model.biases, bs)):
        assert float((got.grad.double() - ref.grad).abs().max()) <= 1.2e-4 * float(ref.grad.abs().max())
    logits = model(X).detach().double()
    assert float((logits - z.detach()).abs().max()) <= 1.2e-4 * float(z.detach().abs().max())
    model.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_training_runs_through_every_mode(bits):
    """Score, sampled and exact steps with the optimizer: the weights move, stay
    finite, and two runs agree bit for bit."""
    def run():
        _, X, t, model = setup(RscConfig(budget=(1, 2), refresh_interval=3, total_steps=8))
        opt = rsc.AdamW(model.parameters(), lr=1e-2, state_bits=bits)
        losses = [model.train_step(X, t, opt, i).detach() for i in range(8)]
        modes = [r.mode for r in model.controller.history]
        weights = [p.detach().clone() for p in model.parameters()]
        model.close()
        return torch.stack(losses), modes, weights

    losses, modes, weights = run()
    assert modes == ["score", "sampled", "sampled"] * 2 + ["score", "exact"]
    assert bool(losses.isfinite().all()) and all(bool(w.isfinite().all()) for w in weights)
    again, _, weights2 = run()
    assert torch.equal(losses, again) and all(torch.equal(a, b) for a, b in zip(weights, weights2))
    first = setup(RscConfig())[3]
    assert all(not torch.equal(a, b) for a, b in zip(weights, first.parameters()))
    first.close()


def test_more_classes_than_hidden_units():
    _, X, t, model = setup(RscConfig(enabled=False), classes=3000, layers=1)
    t[1] = 2999
    loss = model.train_step(X, t, None, 0)
    assert bool(loss.isfinite()) and all(bool(p.grad.isfinite().all()) for p in model.parameters())
    model.close()


def test_refusals():
    for bad in (dict(hidden=30), dict(layers=0)):
        with pytest.raises(ValueError):
            setup(RscConfig(), **bad)


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 32), (torch.bfloat16, 8)])
def test_a_whole_step_captured_is_the_eager_one(dtype, bits):
    """Layer, loss, gradients and optimizer in one graph, replayed between eager
    steps of a twin."""
    def build():
        g = torch.Generator(device="cuda").manual_seed(8)
        ps = [torch.nn.Parameter((torch.randn(s, generator=g, device="cuda") / 8).to(dtype))
              for s in ((50, 70), (70,), (70, 41), (41,))]
        return ps, rsc.AdamW(ps, lr=1e-2, state_bits=bits)

    g = torch.Generator(device="cuda").manual_seed(9)
    x, r = (torch.randn((200, c), generator=g, device="cuda").to(dtype) for c in (50, 70))
    t = torch.randint(0, 41, (200,), generator=g, device="cuda")
    t[::7] = -100

    def step(ps, opt):
        loss = rsc.linear_cross_entropy(rsc.linear(x, ps[0], ps[1], residual=r, act="relu"), ps[2], t, ps[3])
        for p, d in zip(ps, torch.autograd.grad(loss, ps)):
            p.grad = d
        opt.step()
        return loss.detach()

    (ps, opt), (qs, twin) = build(), build()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(ps, opt)
    torch.cuda.current_stream().wait_stream(stream)
    step(qs, twin)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = step(ps, opt)
    for i in range(4):
        with torch.no_grad():
            x.mul_(0.9)
            t[i] = i
        graph.replay()
        torch.cuda.synchronize()
        want = step(qs, twin)
        assert torch.equal(loss, want) and all(torch.equal(p, q) for p, q in zip(ps, qs)), i
    assert int(opt.param_groups[0]["step"]) == int(twin.param_groups[0]["step"]) == 5
