"""Host threads, each with its own stream, train small models on the update
phase's operators at the same time: every result equals, bit for bit, the one
of the same steps run alone."""
import threading

import pytest
import torch

import paper_2210_10737_amd as rsc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu(gpu):
    yield


def _train(i, out):
    """Six steps of two layers, a loss and the optimizer; odd sizes, a type and a
    direction of the weights a thread."""
    dtype = [torch.float32, torch.bfloat16, torch.float16, torch.float32][i % 4]
    n, k, m, v = 300 + 61 * i, 40 + 3 * i, 90 + 7 * i, 30 + 40 * i
    g = torch.Generator(device="cuda").manual_seed(70 + i)
    x = torch.randn((n, k), generator=g, device="cuda").to(dtype)
    r = torch.randn((n, m), generator=g, device="cuda").to(dtype)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    t[::5] = -100
    shapes = [(m, k) if i % 2 else (k, m), (m,), (m, v), (v,)]
    ps = [torch.nn.Parameter((torch.randn(s, generator=g, device="cuda") / 8).to(dtype)) for s in shapes]
    opt = rsc.AdamW(ps, lr=1e-2, state_bits=8 if i % 2 else 32, seed=i)
    got = []
    for _ in range(6):
        w = ps[0].t() if i % 2 else ps[0]
        h = rsc.linear(x, w, ps[1], residual=r, act=["relu", "gelu", "silu", "relu"][i % 4])
        loss = rsc.linear_cross_entropy(h, ps[2], t, ps[3])
        grads = torch.autograd.grad(loss, ps)
        for p, d in zip(ps, grads):
            p.grad = d
        opt.step()
        got += [loss.detach(), *[p.detach().clone() for p in ps]]
    torch.cuda.current_stream().synchronize()
    out.extend(a.cpu() for a in got)


def test_concurrent_training_matches_training_alone():
    count = 4
    alone, together, errors = [[] for _ in range(count)], [[] for _ in range(count)], []
    for i in range(count):
        _train(i, alone[i])
    ready = torch.cuda.Event()
    ready.record()

    def work(i):
        try:
            stream = torch.cuda.Stream()
            stream.wait_event(ready)
            with torch.cuda.stream(stream):
                for _ in range(3):
                    together[i].clear()
                    _train(i, together[i])
        except Exception as e:  # noqa: BLE001
            errors.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(count)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for i in range(count):
        assert all(torch.equal(a, b) for a, b in zip(alone[i], together[i])) and len(alone[i]) == len(together[i]), i
