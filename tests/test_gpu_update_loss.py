"""The class loss and its gradients against the formula in 64 bits.

Tolerances: a logit is off by at most 2 (k + 8) 2^-24 of its sum of magnitudes
(as in the layer's tests), `z` at most over a row; log sum exp by z and by the
relative error of a sum of positive terms: at most 600 additions in a chain
(16 within a lane's tile columns, 4 waves, the tiles) and an exponential
within 2^-20 of its value (|arguments| up to 16 log2 e, rounded to 24 bits), so 2^-14 in
all with room; the gradient of a logit is off by its share of both and, held
in the operands' type, by half a step."""
import math

import pytest
import torch

import paper_2210_10737_amd as rsc

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
# the last two: several pieces of the vocabulary in the backward pass
SIZES = [(1, 1, 1), (1, 8, 2), (3, 5, 7), (17, 64, 33), (33, 100, 257), (130, 33, 64), (300, 257, 70), (64, 1000, 41),
         (257, 64, 1500), (1, 512, 5000), (4000, 24, 300), (2, 64, 70001)]


@pytest.fixture(scope="module", autouse=True)
def _gpu(gpu):
    yield


def half(dtype):
    return torch.finfo(dtype).eps / 2


def sums(k):
    return 2 * (k + 8) * 2.0 ** -24


def rand(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def close(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, what
    bad = (got - want).abs() - bound
    assert bool((bad <= 0).all()), (what, float(bad.max()), float(want.abs().max()))


def inputs(n, k, v, dtype, out_major, valid, seed, ignore=-100, i32=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = rand((n, k), dtype, g)
    w = rand((v, k), dtype, g, 2 / math.sqrt(k)).t() if out_major else rand((k, v), dtype, g, 2 / math.sqrt(k))
    b = rand((v,), dtype, g)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    t[torch.rand(n, generator=g, device="cuda") >= valid] = ignore
    return x, w, b, t.int() if i32 else t


def reference(x, w, b, t, ignore, reduction, up):
    """(rows' losses, their bound, gradients with their bounds) in 64 bits."""
    x, w = x.detach().double(), w.detach().double()
    dtype_half = 0
    k = x.shape[1]
    z, mag = x @ w, x.abs() @ w.abs()
    if b is not None:
        z, mag = z + b.detach().double(), mag + b.detach().double().abs()
    keep = t != ignore
    t = torch.where(keep, t.long(), torch.zeros_like(t.long()))
    lse = torch.logsumexp(z, 1)
    z_off = sums(k) * mag
    row_off = z_off.amax(1)
    rows = torch.where(keep, lse - z.gather(1, t[:, None])[:, 0], torch.zeros_like(lse))
    rows_bound = 2 * row_off + 2.0 ** -14 + 2.0 ** -22 * (lse.abs() + z.abs().amax(1))
    count = max(1, int(keep.sum()))
    weight = keep.double() * (up.double() if reduction == "none" else float(up) / (count if reduction == "mean" else 1))
    p = torch.exp(z - lse[:, None])
    off = p * (2 * row_off + 2.0 ** -14)[:, None]
    p.scatter_add_(1, t[:, None], -torch.ones_like(t[:, None], dtype=torch.float64))
    return rows, rows_bound, weight[:, None] * p, weight.abs()[:, None] * off, weight.abs()[:, None] * p.abs(), count


def check(n, k, v, dtype, out_major, bias, valid, reduction="mean", ignore=-100, i32=False, seed=5, up_scale=1.0,
          bias_f32=False):
    x, w, b, t = inputs(n, k, v, dtype, out_major, valid, seed + n + 7 * k + 31 * v, ignore, i32)
    b = (b.float() if bias_f32 else b) if bias else None
    leaves = [a for a in (x, w, b) if a is not None]
    for a in leaves:
        a.requires_grad_()
    g = torch.Generator(device="cuda").manual_seed(seed)
    up = torch.randn(n, generator=g, device="cuda") * up_scale if reduction == "none" else \
        torch.full((), 1.5 * up_scale, device="cuda")
    loss = rsc.linear_cross_entropy(x, w, t, b, ignore_index=ignore, reduction=reduction)
    assert loss.dtype == torch.float32 and tuple(loss.shape) == ((n,) if reduction == "none" else ())
    rows, rows_bound, grad, grad_off, grad_mag, count = reference(x, w, b, t, ignore, reduction, up)
    keep = (t != ignore).double()
    if reduction == "none":
        close(loss.detach(), rows, rows_bound, ("loss", n, k, v))
        assert bool((loss.detach()[t == ignore] == 0).all())
    else:
        by = count if reduction == "mean" else 1
        close(loss.detach(), rows.sum() / by, (rows_bound * keep).sum() / by + 2.0 ** -23 * rows.sum() / by + 1e-7,
              ("loss", n, k, v))
    with torch.no_grad():
        assert torch.equal(rsc.linear_cross_entropy(x, w, t, b, ignore_index=ignore, reduction=reduction), loss)
    got = torch.autograd.grad(loss, leaves, up)
    # the rounding of G to its type (fp16: half of its smallest step, 2^-25 over 2^10, for small ones)
    tiny = up.abs().max().double() * 2.0 ** -34 if dtype == torch.float16 else 0.0
    grad_off = grad_off + (half(dtype) * grad_mag + tiny * (grad_mag > 0)) * (1 if dtype != torch.float32 else 0.5) \
        + 2.0 ** -22 * grad_mag
    x6, w6 = x.detach().double(), w.detach().double()
    small = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps   # a result's own smallest step
    pieces = 4
    want, mag = grad @ w6.t(), (grad_mag + grad_off) @ w6.abs().t()
    off = grad_off @ w6.abs().t() + (sums(v) + pieces * 2.0 ** -23) * mag
    close(got[0], want, off + half(dtype) * (want.abs() + off) + small, ("dx", n, k, v))
    assert not got[0][t == ignore].any()
    want, mag = x6.t() @ grad, x6.abs().t() @ (grad_mag + grad_off)
    off = x6.abs().t() @ grad_off + (sums(n) + 2.0 ** -23) * mag
    close(got[1], want, off + half(dtype) * (want.abs() + off) + small, ("dw", n, k, v))
    if bias:
        want, off = grad.sum(0), grad_off.sum(0)
        assert got[2].dtype == b.dtype
        close(got[2], want, off + half(b.dtype) * (want.abs() + off) + small, ("db", n, k, v))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out_major", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_loss_and_gradients(size, out_major, dtype):
    check(*size, dtype, out_major, bias=True, valid=0.8)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("valid", [1.0, 0.05, 0.0])
def test_reductions_and_masks(valid, reduction, dtype):
    check(70, 48, 300, dtype, True, bias=False, valid=valid, reduction=reduction, i32=True)
    check(41, 48, 90, dtype, False, bias=True, valid=valid, reduction=reduction, ignore=3)
    check(150, 48, 41, dtype, False, bias=True, valid=valid, reduction=reduction, ignore=3, bias_f32=True)
    check(150, 40, 64, dtype, True, bias=False, valid=valid, reduction=reduction)
    check(150, 40, 65, dtype, True, bias=True, valid=valid, reduction=reduction, bias_f32=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_small_upstream_gradients(dtype):
    check(64, 32, 1000, dtype, True, bias=True, valid=0.9, reduction="none", up_scale=2.0 ** -10)
    check(64, 32, 1000, dtype, True, bias=True, valid=0.9, reduction="none", up_scale=64.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_pieces_of_the_vocabulary(dtype):
    """More than one piece in the backward pass: 60,000 rows, pieces of 2,048
    classes or the next multiple of 256."""
    check(66000, 16, 4500, dtype, True, bias=True, valid=0.9)
    check(66000, 16, 2300, dtype, False, bias=True, valid=0.9)


def test_large_logits_and_masked_classes():
    """A bias of -inf takes a class out, one of the lowest value nearly so;
    logits far apart neither overflow nor vanish."""
    n, k, v = 40, 16, 700
    x, w, b, t = inputs(n, k, v, torch.float32, True, 1.0, 11)
    b[100:400] = -float("inf")
    b[400:410] = torch.finfo(torch.float32).min
    b[3] = 300.0
    t.fill_(3)
    t[0] = 5
    x.requires_grad_()
    loss = rsc.linear_cross_entropy(x, w, t, b, reduction="none")
    z = x.detach().double() @ w.double() + b.double()
    want = torch.logsumexp(z, 1) - z.gather(1, t[:, None])[:, 0]
    close(loss.detach(), want, 2.0 ** -14 + 2.0 ** -20 * want.abs(), "loss")
    gx, = torch.autograd.grad(loss.sum(), x)
    p = torch.softmax(z, 1)
    p[torch.arange(n, device="cuda"), t] -= 1
    close(gx, p @ w.double().t(), torch.full_like(gx, 1e-3, dtype=torch.float64), "dx")
    t[1] = 200   # the class of a row itself taken out: an infinite loss
    assert float(rsc.linear_cross_entropy(x.detach(), w, t, b, reduction="none")[1]) == float("inf")


@pytest.mark.parametrize("v", [30, 300])
def test_targets_out_of_range_show(v):
    x, w, b, t = inputs(20, 16, v, torch.float32, True, 1.0, 2)
    for bad in (v, -1, 1 << 40):
        t2 = t.clone()
        t2[4] = bad
        xg = x.clone().requires_grad_()
        g, = torch.autograd.grad(rsc.linear_cross_entropy(xg, w, t2, b), xg)
        assert bool(g[4].isnan().all()) and not g[:4].isnan().any() and not g[5:].isnan().any()
        rows = rsc.linear_cross_entropy(x, w, t2, b, reduction="none")
        assert bool(rows.isnan().nonzero()[:, 0].eq(4).all()) and int(rows.isnan().sum()) == 1
        assert bool(rsc.linear_cross_entropy(x, w, t2, b).isnan())


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows(dtype):
    x = torch.empty((0, 12), dtype=dtype, device="cuda", requires_grad=True)
    w = torch.ones((12, 5), dtype=dtype, device="cuda", requires_grad=True)
    b = torch.ones(5, dtype=dtype, device="cuda", requires_grad=True)
    t = torch.empty(0, dtype=torch.int64, device="cuda")
    loss = rsc.linear_cross_entropy(x, w, t, b)
    assert float(loss.detach()) == 0.0
    gx, gw, gb = torch.autograd.grad(loss, [x, w, b])
    assert tuple(gx.shape) == (0, 12) and not gw.any() and not gb.any()
    assert tuple(rsc.linear_cross_entropy(x, w, t, b, reduction="none").shape) == (0,)


def test_gradients_against_differences():
    x, w, b, t = inputs(12, 20, 50, torch.float32, False, 0.8, 3)
    leaves = [a.requires_grad_() for a in (x, w, b)]
    grads = torch.autograd.grad(rsc.linear_cross_entropy(x, w, t, b), leaves)
    g = torch.Generator(device="cuda").manual_seed(1)
    h = 2.0 ** -6
    for i, gr in enumerate(grads):
        d = rand(tuple(gr.shape), torch.float32, g)
        d = d / d.norm()

        def at(s):
            xs, ws, bs = (a.detach() + s * h * d if j == i else a.detach() for j, a in enumerate(leaves))
            return float(rsc.linear_cross_entropy(xs, ws, t, bs))

        slope, want = (at(1) - at(-1)) / (2 * h), float((gr * d).sum())
        # third derivatives of a softmax are below 1 in these units, two losses of 5 are rounded at 2^-22
        assert abs(slope - want) <= h * h + 2 * 2.0 ** -21 / h, (i, slope, want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured(dtype):
    x, w, b, t = inputs(150, 64, 500, dtype, True, 0.8, 3)
    leaves = [a.requires_grad_() for a in (x, w, b)]

    def work():
        loss = rsc.linear_cross_entropy(x, w, t, b)
        return [loss.detach(), *torch.autograd.grad(loss, leaves)]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        work()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for i in range(3):
        with torch.no_grad():
            x.mul_(0.9)
            t[i] = -100
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(held, work()):
            assert torch.equal(got, want), i


def test_refusals():
    x, w, b, t = inputs(6, 16, 30, torch.float32, True, 1.0, 2)
    for bad in (dict(targets=t.float()), dict(targets=t[:5]), dict(targets=t.cpu()), dict(reduction="max"),
                dict(ignore_index=1 << 63), dict(bias=b[:3]), dict(weight=w.half()), dict(x=x.half()), dict(x=x.cpu()),
                dict(x=x[:, :8])):
        args = {**dict(x=x, weight=w, targets=t, bias=b), **bad}
        with pytest.raises(ValueError):
            rsc.linear_cross_entropy(**args)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lowest", [torch.float32, None])      # of an fp32 bias, or of the operands' type
@pytest.mark.parametrize("v,masked", [(1500, (300, 1100)), (1500, (0, 1400)), (50, (2, 50)), (50, (0, 40)), (700, (256, 700))])
def test_long_ranges_of_classes_at_the_lowest_value(v, masked, lowest, dtype):
    """A bias of the type's lowest value takes a range of classes out that is
    wider than a tile: loss and gradients are those without these classes."""
    n, k = 70, 48
    x, w, b, t = inputs(n, k, v, dtype, True, 0.8, 13)
    b = b.float() if lowest else b
    b[masked[0]:masked[1]] = torch.finfo(b.dtype).min
    rest = torch.cat([torch.arange(masked[0]), torch.arange(masked[1], v)]).cuda()
    t = torch.where(t >= 0, rest[t.clamp_min(0) % rest.numel()], t)
    among = torch.where(t >= 0, torch.searchsorted(rest, t.clamp_min(0)), t)
    up = torch.full((), 1.5, device="cuda")
    for a in (x, w, b):
        a.requires_grad_()
    loss = rsc.linear_cross_entropy(x, w, t, b)
    rows, rows_bound, grad, grad_off, grad_mag, count = reference(x, w[:, rest], b[rest], among, -100, "mean", up)
    keep = (t >= 0).double()
    close(loss.detach(), rows.sum() / count, (rows_bound * keep).sum() / count + 2.0 ** -23 * rows.sum() / count + 1e-7, v)
    got = torch.autograd.grad(loss, [x, w, b], up)
    tiny = 1.5 * 2.0 ** -34 if dtype == torch.float16 else 0.0
    grad_off = grad_off + half(dtype) * grad_mag + tiny * (grad_mag > 0) + 2.0 ** -22 * grad_mag
    small = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    x6, w6 = x.detach().double(), w.detach()[:, rest].double()
    want, off = grad @ w6.t(), grad_off @ w6.abs().t() + sums(v) * ((grad_mag + grad_off) @ w6.abs().t())
    close(got[0], want, off + half(dtype) * (want.abs() + off) + small, "dx")
    want, off = x6.t() @ grad, x6.abs().t() @ grad_off + sums(n) * (x6.abs().t() @ (grad_mag + grad_off))
    close(got[1][:, rest], want, off + half(dtype) * (want.abs() + off) + small, "dw")
    want, off = grad.sum(0), grad_off.sum(0)
    close(got[2][rest], want, off + half(b.dtype) * (want.abs() + off) + small, "db")
    assert not got[1][:, masked[0]:masked[1]].any() and not got[2][masked[0]:masked[1]].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("reduction", ["mean", "none"])
@pytest.mark.parametrize("size", [(70, 48, 300), (150, 48, 41), (257, 64, 1500), (4000, 24, 300), (66000, 16, 2300), (1, 8, 2)])
def test_an_fp32_bias_gets_its_gradient_from_unrounded_values(size, reduction, dtype):
    """The logits' gradient is held in the operands' type for the products; the
    bias's sums are formed before that rounding. A probability is off by its
    logit and its row's lse (`row_off` each) and by two exponentials and a sum of at
    most 130 positive terms, arguments up to 32: (64 + 130 + 8) 2^-24 < 2^-16; the
    sum over rows by fewer than 32 roundings of 2^-24, the result by one."""
    n, k, v = size
    x, w, b, t = inputs(n, k, v, dtype, True, 0.8, 31)
    b = b.float().requires_grad_()
    g = torch.Generator(device="cuda").manual_seed(1)
    up = torch.randn(n, generator=g, device="cuda") if reduction == "none" else torch.full((), 1.5, device="cuda")
    for leaves in ((b,), (b, x, w)):
        for a in (x, w):
            a.requires_grad_(len(leaves) > 1)
        got = torch.autograd.grad(rsc.linear_cross_entropy(x, w, t, b, reduction=reduction), leaves, up)[0]
        x6, w6 = x.detach().double(), w.detach().double()
        z, mag = x6 @ w6 + b.detach().double(), x6.abs() @ w6.abs() + b.detach().double().abs()
        row_off = (sums(k) * mag).amax(1)
        keep = t >= 0
        weight = keep * up.double() / (max(1, int(keep.sum())) if reduction == "mean" else 1)
        p = torch.softmax(z, 1)
        off = (weight.abs()[:, None] * p * (2 * row_off + 2.0 ** -16)[:, None]).sum(0)
        p.scatter_add_(1, t.clamp_min(0)[:, None], -torch.ones_like(p[:, :1]))
        p *= weight[:, None]
        close(got, p.sum(0), off + 2.0 ** -19 * p.abs().sum(0) + 2.0 ** -23 * p.sum(0).abs(), size)


@pytest.mark.parametrize("out_major", [False, True])
@pytest.mark.parametrize("size", [(70, 8, 300), (150, 8, 41), (300, 5, 64), (513, 8, 1500), (1, 8, 5000), (2, 4, 70001)])
def test_fp32_losses_to_the_accuracy_of_fp32(size, out_major):
    """Short sums of k, so that the softmax's own error shows. In units of 2^-24:
    arguments up to 32 rounded once (32), the sum's chain of up to 64 additions
    in a lane, 4 waves and 16 joins with an exponential each, 8 tiles a thread with
    two (100 additions, 40 exponentials of 4): below 2^-15 of a row's loss, and of
    a probability with twice the logits' own error."""
    n, k, v = size
    x, w, b, t = inputs(n, k, v, torch.float32, out_major, 0.8, 41)
    leaves = [a.requires_grad_() for a in (x, w, b)]
    up = torch.full((), 1.5, device="cuda")
    rows = rsc.linear_cross_entropy(x, w, t, b, reduction="none")
    loss = rsc.linear_cross_entropy(x, w, t, b)
    x6, w6 = x.detach().double(), w.detach().double()
    z, mag = x6 @ w6 + b.detach().double(), x6.abs() @ w6.abs() + b.detach().double().abs()
    assert float((z.amax(1) - z.amin(1)).max()) <= 32
    row_off = (sums(k) * mag).amax(1)
    keep, at = t >= 0, t.clamp_min(0)[:, None]
    want = torch.where(keep, torch.logsumexp(z, 1) - z.gather(1, at)[:, 0], 0.0)
    bound = 2 * row_off + 2.0 ** -15 + 2.0 ** -23 * want.abs()
    close(rows.detach(), want, bound, "rows")
    count = max(1, int(keep.sum()))
    close(loss.detach(), want.sum() / count, (bound * keep).sum() / count + 2.0 ** -23 * want.sum() / count, "loss")
    weight = (keep * 1.5 / count)[:, None]
    p = torch.softmax(z, 1)
    off = weight * p * (2 * row_off + 2.0 ** -15)[:, None]
    p = weight * p.scatter_add(1, at, -torch.ones_like(p[:, :1]))
    off = off + 2.0 ** -22 * p.abs()      # the differences and factors, held in fp32
    gx, gw, gb = torch.autograd.grad(loss, leaves, up)
    close(gx, p @ w6.t(), off @ w6.abs().t() + (sums(v) + 2.0 ** -22) * (p.abs() @ w6.abs().t()), "dx")
    close(gw, x6.t() @ p, x6.abs().t() @ off + (sums(n) + 2.0 ** -22) * (x6.abs().t() @ p.abs()), "dw")
    close(gb, p.sum(0), off.sum(0) + 2.0 ** -22 * p.abs().sum(0), "db")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(96, 48, 300), (64, 1000, 41), (66000, 16, 2300), (2, 64, 300)])
def test_upstream_gradients_of_any_size_keep_their_rows(size, dtype):
    """Reduction "none", the rows' upstream gradients from 2^12 down to 2^-10: each
    row of dX is right beside its own upstream gradient, not only the largest."""
    n, k, v = size
    x, w, b, t = inputs(n, k, v, dtype, True, 0.9, 51)
    for a in (x, w, b):
        a.requires_grad_()
    g = torch.Generator(device="cuda").manual_seed(2)
    up = torch.randn(n, generator=g, device="cuda") * 2.0 ** (12 - torch.arange(n, device="cuda") % 23)
    up[0] = 2.0 ** 12
    up[1] = 0.0
    loss = rsc.linear_cross_entropy(x, w, t, b, reduction="none")
    _, _, grad, grad_off, grad_mag, _ = reference(x, w, b, t, -100, "none", up)
    got = torch.autograd.grad(loss, [x, w, b], up)
    # fp16: half of the smallest step, 2^-25 over 2^10, beside the row's own upstream gradient
    tiny = up.abs().double()[:, None] * 2.0 ** -34 if dtype == torch.float16 else 0.0
    grad_off = grad_off + (half(dtype) * grad_mag + tiny * (grad_mag > 0)) * (1 if dtype != torch.float32 else 0.5) \
        + 2.0 ** -22 * grad_mag
    x6, w6 = x.detach().double(), w.detach().double()
    small = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps   # a result's own smallest step
    want, mag = grad @ w6.t(), (grad_mag + grad_off) @ w6.abs().t()
    off = grad_off @ w6.abs().t() + (sums(v) + 4 * 2.0 ** -23) * mag
    close(got[0], want, off + half(dtype) * (want.abs() + off) + small, "dx")
    assert not got[0][t == -100].any() and not got[0][1].any()
    # in the sums over rows what is lost is beside the largest one
    if dtype == torch.float16:
        grad_off = grad_off + up.abs().max().double() * 2.0 ** -34 * (grad_mag > 0)
    want, off = x6.t() @ grad, x6.abs().t() @ grad_off + (sums(n) + 2.0 ** -23) * (x6.abs().t() @ (grad_mag + grad_off))
    close(got[1], want, off + half(dtype) * (want.abs() + off) + small, "dw")
    want, off = grad.sum(0), grad_off.sum(0)
    close(got[2], want, off + half(b.dtype) * (want.abs() + off) + small, "db")


def test_fp16_upstream_gradients_that_are_not_finite_stay_in_their_rows():
    x, w, b, t = inputs(40, 32, 300, torch.float16, True, 1.0, 52)
    x.requires_grad_()
    up = torch.full((40,), 8.0, device="cuda")
    want, = torch.autograd.grad(rsc.linear_cross_entropy(x, w, t, b, reduction="none"), x, up)
    up[3], up[7] = float("inf"), float("nan")
    got, = torch.autograd.grad(rsc.linear_cross_entropy(x, w, t, b, reduction="none"), x, up)
    rest = torch.tensor([i not in (3, 7) for i in range(40)], device="cuda")
    assert torch.equal(got[rest], want[rest]) and not got[3].isfinite().any() and bool(got[7].isnan().all())
