"""The layer product and its gradients against the formula in 64 bits.

Tolerances: a sum of k products in fp32 is off by at most 2 (k + 8) 2^-24 of
the sum of magnitudes (a rounding an addition, twice for the order inside the
matrix instruction, 8 for the split of fp32 values and the epilogue); a result
is rounded once, by eps / 2 of its type."""
import math

import pytest
import torch

import paper_2210_10737_amd as rsc
from paper_2210_10737_amd import update

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 1, 1), (1, 8, 8), (3, 5, 7), (17, 64, 33), (33, 100, 257), (130, 129, 131), (300, 257, 70), (64, 1000, 41),
         (257, 64, 512), (1, 4096, 1024), (1000, 40, 300), (513, 2048, 129), (5000, 31, 19), (2, 9000, 3)]


@pytest.fixture(scope="module", autouse=True)
def _gpu(gpu):
    yield


def half(dtype):
    return torch.finfo(dtype).eps / 2


def sums(k):
    return 2 * (k + 8) * 2.0 ** -24


def rand(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def act64(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0), (z > 0).double()
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    return z, torch.ones_like(z)


def close(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, what
    bad = (got - want).abs() - bound
    assert bool((bad <= 0).all()), (what, float(bad.max()), float(want.abs().max()))


def inputs(n, k, m, dtype, out_major, seed, bias_dtype=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = rand((n, k), dtype, g)
    w = rand((m, k), dtype, g, 1 / math.sqrt(k)).t() if out_major else rand((k, m), dtype, g, 1 / math.sqrt(k))
    return x, w, rand((m,), bias_dtype or dtype, g), rand((n, m), dtype, g), rand((n, m), dtype, g)


def check(n, k, m, dtype, act, out_major, bias, residual, alpha, beta, bias_dtype=None, seed=3):
    x, w, b, r, dy = inputs(n, k, m, dtype, out_major, seed + n + 7 * k + 31 * m, bias_dtype)
    b, r = b if bias else None, r if residual else None
    leaves = [t.requires_grad_() if t is not None else None for t in (x, w, b, r)]
    y = rsc.linear(x, w, b, residual=r, act=act, alpha=alpha, beta=beta)
    assert y.dtype == dtype and tuple(y.shape) == (n, m)
    x6, w6 = x.detach().double(), w.detach().double()
    z = alpha * (x6 @ w6)
    mag = abs(alpha) * (x6.abs() @ w6.abs())
    if bias:
        z, mag = z + b.detach().double(), mag + b.detach().double().abs()
    if residual:
        z, mag = z + beta * r.detach().double(), mag + abs(beta) * r.detach().double().abs()
    want, _ = act64(z, act)
    z_off = sums(k) * mag
    close(y.detach(), want, 1.2 * z_off + half(dtype) * want.abs() + 1e-7, ("y", n, k, m, act))
    wanted = [t for t in leaves if t is not None]
    grads = dict(zip([i for i, t in enumerate(leaves) if t is not None], torch.autograd.grad(y, wanted, dy)))
    # the slope from what the forward pass kept: Y > 0, or Z rounded (|act''| <= 1.13)
    if act == "relu":
        slope = (y.detach() > 0).double()
        s_off = torch.zeros_like(z)
    else:
        _, slope = act64(z, act)
        s_off = 0.0 * z if act == "none" else 1.13 * (z_off + half(dtype) * z.abs()) + 2.0 ** -22
    dz = dy.double() * slope
    dz_off = dy.double().abs() * s_off + (0 if act == "none" else half(dtype)) * dz.abs() + 1e-7 * (act != "none")
    dz_mag = dz.abs() + dz_off
    want = alpha * (dz @ w6.t())
    off = abs(alpha) * (dz_off @ w6.abs().t() + sums(m) * (dz_mag @ w6.abs().t()))
    close(grads[0], want, off + half(dtype) * (want.abs() + off) + 1e-7, ("dx", n, k, m, act))
    want = alpha * (x6.t() @ dz)
    off = abs(alpha) * (x6.abs().t() @ dz_off + sums(n) * (x6.abs().t() @ dz_mag))
    close(grads[1], want, off + half(dtype) * (want.abs() + off) + 1e-7, ("dw", n, k, m, act))
    assert grads[1].stride(0) == 1 or not out_major or k == 1 or m == 1
    if bias:
        want, off = dz.sum(0), dz_off.sum(0) + 2.0 ** -23 * dz_mag.sum(0)
        assert grads[2].dtype == b.dtype
        close(grads[2], want, off + half(b.dtype) * (want.abs() + off) + 1e-7, ("db", n, k, m, act))
    if residual:
        off = abs(beta) * dz_off + half(dtype) * abs(beta) * dz_mag
        close(grads[3], beta * dz, off + 1e-7, ("dr", n, k, m, act))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out_major", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_product_and_gradients(size, out_major, dtype):
    check(*size, dtype, "none", out_major, bias=True, residual=False, alpha=1.0, beta=1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("size,alpha,beta", [((70, 50, 90), 1.0, 1.0), ((257, 129, 40), 0.25, -0.5)])
def test_epilogues(size, alpha, beta, act, dtype):
    check(*size, dtype, act, False, bias=True, residual=True, alpha=alpha, beta=beta)
    check(*size, dtype, act, True, bias=False, residual=True, alpha=alpha, beta=beta)
    check(*size, dtype, act, True, bias=True, residual=False, alpha=alpha, beta=beta, bias_dtype=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(700, 520, 600), (2500, 300, 512), (40000, 70, 130), (1500, 1030, 2050)])
def test_larger_products(size, dtype):
    """Several tiles of every shape, split and unsplit sums."""
    check(*size, dtype, "gelu", False, bias=True, residual=False, alpha=1.0, beta=1.0)
    check(*size, dtype, "none", True, bias=False, residual=True, alpha=1.0, beta=0.5)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strided_operands(dtype):
    """Rows apart, columns apart, misaligned bases, expanded gradients; what
    lies beside an operand (NaN) is never used and outputs' padding is kept."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n, k, m = 75, 43, 29
    big = torch.full((n + 2, 4 * k + 16), float("nan"), dtype=dtype, device="cuda")
    wide = torch.full((k, m + 35), float("nan"), dtype=dtype, device="cuda")
    forms = [big[:n, :k], big[1:n + 1, 3:3 + k], big[:n, 0:2 * k:2], big[:, 8:8 + k][:n]]
    x0, w0 = rand((n, k), dtype, g), rand((k, m), dtype, g)
    want = rsc.linear(x0, w0)
    for x in forms:
        big.fill_(float("nan"))
        x.copy_(x0)
        for w in (wide[:, :m], wide[:, 5:5 + m], wide[:, 0:2 * m:2], torch.empty((m, k + 3), dtype=dtype, device="cuda")[:, :k].t()):
            w.copy_(w0)
            assert torch.equal(rsc.linear(x, w), want)
    out = torch.full((n, 40), 7.0, dtype=dtype, device="cuda")
    assert rsc.linear(x0, w0, out=out[:, :m]).data_ptr() == out.data_ptr()
    assert torch.equal(out[:, :m], want) and bool((out[:, m:] == 7).all())
    x, w = x0.clone().requires_grad_(), w0.clone().requires_grad_()
    a = torch.autograd.grad(rsc.linear(x, w).sum(), [x, w])          # a gradient of stride 0
    b = torch.autograd.grad(rsc.linear(x, w), [x, w], torch.ones((n, m), dtype=dtype, device="cuda"))
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    # in place on the residual
    r = rsc.linear(x0, w0)
    r2 = r.clone()
    assert torch.equal(rsc.linear(x0, w0, residual=r, out=r), rsc.linear(x0, w0, residual=r2))


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows(dtype):
    x = torch.empty((0, 12), dtype=dtype, device="cuda", requires_grad=True)
    w = torch.ones((12, 5), dtype=dtype, device="cuda", requires_grad=True)
    b = torch.ones(5, dtype=dtype, device="cuda", requires_grad=True)
    y = rsc.linear(x, w, b, act="silu")
    assert tuple(y.shape) == (0, 5)
    gx, gw, gb = torch.autograd.grad(y, [x, w, b], torch.empty((0, 5), dtype=dtype, device="cuda"))
    assert tuple(gx.shape) == (0, 12) and not gw.any() and not gb.any() and tuple(gw.shape) == (12, 5)


def test_gradients_against_differences():
    """fp32, central differences of a smooth scalar: steps of 2^-7, the second
    derivatives of this sum keep their error below 2e-3 of the scale."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w, b, r = rand((9, 21), torch.float32, g), rand((21, 13), torch.float32, g, 0.2), rand((13,), torch.float32, g), \
        rand((9, 13), torch.float32, g)
    dy = rand((9, 13), torch.float32, g)
    leaves = [t.requires_grad_() for t in (x, w, b, r)]
    grads = torch.autograd.grad(rsc.linear(x, w, b, residual=r, act="gelu", alpha=0.7, beta=1.5), leaves, dy)
    h = 2.0 ** -7
    for t, gr in zip(leaves, grads):
        d = rand(tuple(t.shape), torch.float32, g)
        at = lambda s: (rsc.linear(*[v.detach() + s * h * d if v is t else v.detach() for v in leaves[:3]],  # noqa: E731
                                   residual=(r.detach() + s * h * d if t is r else r.detach()), act="gelu", alpha=0.7,
                                   beta=1.5).double() * dy.double()).sum()
        slope = float((at(1) - at(-1)) / (2 * h))
        want = float((gr.double() * d.double()).sum())
        assert abs(slope - want) <= 2e-3 * max(1.0, float(gr.double().norm() * d.double().norm()) ** 0.5 * 3), (slope, want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_special_values(dtype):
    """NaN stays in its row or column; a bias of -inf and the type's lowest
    value pass through; a ReLU keeps NaN."""
    x = torch.ones((40, 30), dtype=dtype, device="cuda")
    w = torch.full((30, 50), 0.5, dtype=dtype, device="cuda")
    b = torch.zeros(50, dtype=dtype, device="cuda")
    b[3] = -float("inf")
    b[4] = torch.finfo(dtype).min
    x[7, 2] = float("nan")
    y = rsc.linear(x, w, b)
    assert bool(y[7].isnan().all()) and not y[torch.arange(40, device="cuda") != 7].isnan().any()
    assert bool((y[:7, 3] == -float("inf")).all())
    assert bool((y[:7, 4].double() <= torch.finfo(dtype).min * 0.99).all())
    y = rsc.linear(x, w, b, act="relu")
    assert bool(y[7].isnan().all()) and bool((y[:7, 3] == 0).all()) and bool((y[:7, 5] == 15).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(300, 200, 150), (64, 5000, 64)])
def test_results_repeat_and_streams(size, dtype):
    x, w, b, r, dy = inputs(*size, dtype, False, 9)
    first = rsc.linear(x, w, b, residual=r, act="silu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            again = rsc.linear(x, w, b, residual=r, act="silu")
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(first, again)


def test_largest_fp32_magnitudes():
    """The three-part form holds values near the ends of fp32's range."""
    x = torch.tensor([[3e38, 1e-30, 1.0]], device="cuda")
    w = torch.tensor([[1e-30, 0.0, 0.0], [0.0, 1e30, 0.0], [0.0, 0.0, 2.0 ** -100]], device="cuda")
    y = rsc.linear(x, w).double().cpu()
    want = x.double().cpu() @ w.double().cpu()
    assert bool(((y - want).abs() <= 2.0 ** -21 * want.abs()).all()), (y, want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured_forward_and_backward(dtype):
    x, w, b, r, dy = inputs(200, 150, 120, dtype, False, 5)
    leaves = [t.requires_grad_() for t in (x, w, b, r)]

    def work():
        y = rsc.linear(x, w, b, residual=r, act="gelu")
        return [y.detach(), *torch.autograd.grad(y, leaves, dy)]

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
            dy.add_(0.01 * i)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(held, work()):
            assert torch.equal(got, want), i


def test_refusals():
    x, w = torch.ones((4, 8), device="cuda"), torch.ones((8, 6), device="cuda")
    for bad in (dict(act="tanh"), dict(bias=torch.ones(5, device="cuda")), dict(residual=torch.ones((4, 5), device="cuda")),
                dict(bias=torch.ones(6, device="cuda", dtype=torch.float16)), dict(bias=torch.ones(6)),
                dict(residual=torch.ones((4, 6), device="cuda", dtype=torch.bfloat16)),
                dict(out=torch.ones((4, 6), device="cuda")), dict(out=torch.ones((4, 8), device="cuda"))):
        with pytest.raises(ValueError):
            rsc.linear(x, w, **bad)
    for args in ((x.cpu(), w), (x.double(), w.double()), (x, w.half()), (x, w[:7]), (x[0], w), (x, w[:, :0])):
        with pytest.raises(ValueError):
            rsc.linear(*args)
    with pytest.raises(rsc.RscError) as e:
        rsc.linear(x, torch.ones((8, 8), device="cuda"), out=x)
    assert rsc.STATUS[e.value.status] == "RSC_ERR_INVALID_ARGUMENT"
    xg = x.clone().requires_grad_()
    with pytest.raises(ValueError):
        rsc.linear(xg, w, out=torch.empty((4, 8), device="cuda")[:, :6])
    y = rsc.linear(xg, w)
    gx, = torch.autograd.grad(y.sum(), xg, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(gx.sum(), xg)


def test_offsets_past_32_bits():
    """An operand of 4.5 GB: its last rows, and the sum over all of them."""
    n, k, m = 2_200_003, 1024, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((n, k), dtype=torch.bfloat16, device="cuda")
    for i in range(0, n, 200_000):
        part = x[i:i + 200_000]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    w = rand((k, m), torch.bfloat16, g, 1 / 32).requires_grad_()
    y = rsc.linear(x, w)
    dy = rand((n, m), torch.bfloat16, g)
    dw, = torch.autograd.grad(y, w, dy)
    w6 = w.detach().double()
    for a in (0, n // 2, n - 300):
        xs = x[a:a + 300].double()
        want = xs @ w6
        close(y.detach()[a:a + 300], want, sums(k) * (xs.abs() @ w6.abs()) + half(torch.bfloat16) * want.abs(), a)
    want, mag = (torch.zeros((k, m), dtype=torch.float64, device="cuda") for _ in range(2))
    for i in range(0, n, 100_000):
        xs, ds = x[i:i + 100_000].double(), dy[i:i + 100_000].double()
        want += xs.t() @ ds
        mag += xs.abs().t() @ ds.abs()
    # a split's chain of additions is at most n long
    close(dw, want, sums(n) * mag + half(torch.bfloat16) * want.abs(), "dw")
    # against weights of 4.5 GB, a column for each of their rows
    wide = x[:2_200_000].view(275_000, 8192).t()
    for rows, form in ((2, "few rows"), (40, "tiles")):
        a = rand((rows, 8192), torch.bfloat16, g)
        last = wide[:, -100:].double()
        want = a.double() @ last
        close(rsc.linear(a, wide)[:, -100:], want, sums(8192) * (a.double().abs() @ last.abs())
              + half(torch.bfloat16) * want.abs(), form)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out_major", [False, True])
@pytest.mark.parametrize("size", [(5003, 1021, 1045), (900, 3001, 700), (64, 9000, 300), (2, 3000, 4000), (1, 700, 9000)])
def test_relu_masks_are_those_of_64_bits(size, out_major, dtype):
    """Every result of a pass that keeps gradients is above zero where the sum
    in 64 bits is (of ten million random ones a few come out of fp32 sums with
    the other sign, or round to 0 in fp16)."""
    n, k, m = size
    x, w, b, r, _ = inputs(n, k, m, dtype, out_major, 77)
    for residual, beta in ((None, 1.0), (r, 0.5)):
        y = rsc.linear(x.clone().requires_grad_(), w, b, residual=residual, act="relu", alpha=0.5, beta=beta)
        z = 0.5 * (x.double() @ w.double()) + b.double() + (0 if residual is None else beta * residual.double())
        assert torch.equal(y.detach() > 0, z > 0)


def test_relu_masks_of_cancelled_sums():
    """The residual takes all of the sum away but its rounding: 30 results that
    32 bits cannot tell from zero. Rows of zeros and exact sums stay zero."""
    g = torch.Generator(device="cuda").manual_seed(8)
    x, w = rand((3, 50), torch.float32, g), rand((50, 10), torch.float32, g)
    exact = x.double() @ w.double()
    r = -exact.float()
    y = rsc.linear(x.clone().requires_grad_(), w, residual=r, act="relu").detach()
    z = exact + r.double()
    assert torch.equal(y > 0, z > 0)
    # one rounding to 32 bits, and on either side a 64-bit sum of 50 terms: up to
    # 50 roundings of 2^-53 of the sum of magnitudes (here about 40: 2e-13)
    sums64 = 2 * 50 * 2.0 ** -53 * (x.double().abs() @ w.double().abs())
    assert bool(((y.double() - z.clamp_min(0)).abs() <= 2.0 ** -24 * z.abs() + sums64).all())
    x, w = torch.zeros((500, 64), device="cuda"), rand((64, 300), torch.float32, g)
    assert not rsc.linear(x.requires_grad_(), w, act="relu").any()
    x = torch.randint(-1, 2, (500, 64), generator=g, device="cuda").float()
    w = torch.randint(-1, 2, (64, 300), generator=g, device="cuda").float()
    assert torch.equal(rsc.linear(x.clone().requires_grad_(), w, act="relu").detach(), torch.relu((x.double() @ w.double()).float()))
    # results that lie on the residual
    for size in ((700, 1021, 300), (64, 9000, 300), (2, 300, 400)):   # tiles, a split k, few rows
        x, w, b, r, _ = inputs(*size, torch.float32, False, 5)
        r = (-(x.double() @ w.double()) - b.double()).float().contiguous()
        want = rsc.linear(x.clone().requires_grad_(), w, b, residual=r, act="relu").detach()
        y, _, _, _ = update._linear_forward(x, w, b, r, 1, 1.0, 1.0, r, True)
        assert y is r and torch.equal(y, want), size


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(700, 520, 301), (300, 64, 41), (9000, 130, 300), (3000, 64, 5)])
def test_relu_with_gradients_does_not_depend_on_what_lies_beside_the_weights(size, dtype):
    """Large values beside the weights' rows, as an uninitialised or a wider
    buffer may hold them: results are those beside zeros, bit for bit."""
    n, k, m = size
    x, w, b, r, _ = inputs(n, k, m, dtype, False, 12)
    wide = torch.zeros((k, (m + 31) // 16 * 16), dtype=dtype, device="cuda")
    wide[:, :m] = w
    assert update._ld(wide[:, :m]) is not None       # used as it lies
    got = []
    for beside in (0.0, 1e30 if dtype != torch.float16 else 6e4, float("inf"), float("nan")):
        wide[:, m:] = beside
        for residual in (None, r):
            got.append(rsc.linear(x.clone().requires_grad_(), wide[:, :m], b, residual=residual, act="relu").detach())
    for i, y in enumerate(got[2:]):
        assert torch.equal(y, got[i % 2]), i


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(4992, 300, 320), (704, 1021, 320), (64, 9000, 320), (320, 300, 64)])
def test_relu_masks_beside_rows_of_another_scale(size, dtype):
    """One row in 32 is 2^14 times as large as the others, whose sums are 0.06 or
    so. Every fourth column's bias takes the sum of one ordinary row away but its
    rounding: that row's result is decided in 64 bits, as among rows of one scale."""
    n, k, m = size
    g = torch.Generator(device="cuda").manual_seed(21)
    x, w = rand((n, k), dtype, g, 2.0 ** -4), rand((k, m), dtype, g, 1 / math.sqrt(k))
    x[::32] *= 2.0 ** 14
    b = rand((m,), torch.float32, g, 2.0 ** -4)
    exact = x.double() @ w.double()
    column = torch.arange(0, m, 4, device="cuda")
    row = (column * 32 + 16 + column % 16) % (n // 32 * 32)
    b[column] = -exact[row, column].float()
    y = rsc.linear(x.clone().requires_grad_(), w, b, act="relu").detach()
    z = exact + b.double()
    assert bool((z[row, column].abs() <= 2.0 ** -24 * exact[row, column].abs()).all())
    assert torch.equal(y > 0, z > 0)


def test_out_is_a_write_in_place_to_autograd():
    """A backward pass that saved `out`'s old values raises, and a tensor that
    requires gradients is no place for a result without them."""
    g = torch.Generator(device="cuda").manual_seed(6)
    x, w = rand((9, 16), torch.float32, g), rand((16, 24), torch.float32, g)
    buffer, a = rand((9, 24), torch.float32, g), torch.ones((9, 24), device="cuda", requires_grad=True)
    y = (buffer * a).sum()
    rsc.linear(x, w, out=buffer)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    (buffer * a).sum().backward()
    assert torch.equal(a.grad, rsc.linear(x, w))
    for out in (a, a * 2):
        with pytest.raises(ValueError):
            rsc.linear(x, w, out=out)
    with torch.no_grad():
        rsc.linear(x, w, out=a)
    assert torch.equal(a.detach(), buffer)
    with torch.inference_mode():
        held = torch.empty((9, 24), device="cuda")
        assert torch.equal(rsc.linear(x, w, out=held), buffer)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [40, 41, 1])
@pytest.mark.parametrize("n", [50, 1])
def test_results_can_be_changed_in_place(n, m, dtype):
    """With whole and with ragged rows, results and gradients alike; a ReLU's
    result is what its backward pass reads, so that one raises."""
    x, w, b, _, dy = inputs(n, 24, m, dtype, False, 14)
    x2, w2 = x.clone(), w.clone()
    for t in (x, w, b):
        t.requires_grad_()
    y = rsc.linear(x, w, b, act="gelu")
    want = torch.autograd.grad(y, [x, w, b], 2 * dy)
    y = rsc.linear(x, w, b, act="gelu")
    before = y.detach().clone()
    y.mul_(2).add_(1)
    assert torch.equal(y.detach(), 2 * before + 1) and not y.is_leaf
    got = torch.autograd.grad(y, [x, w, b], dy)
    for p, q in zip(got, want):
        assert torch.equal(p, q) and not p._is_view()
        p.mul_(2)
        assert torch.equal(p, 2 * q)
    y = rsc.linear(x, w, b, act="relu")
    y.mul_(2)
    with pytest.raises(RuntimeError, match="inplace"):
        torch.autograd.grad(y, x, dy)
    # the weights' gradient in the order of weights stored the other way
    w3 = w2.t().contiguous().t().requires_grad_()
    g, = torch.autograd.grad(rsc.linear(x2, w3), w3, dy)
    assert not g._is_view() and (g.stride(0) == 1 or m == 1)
    y = rsc.linear(x2, w2)      # (without gradients)
    y.mul_(2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(4992, 300, 320), (320, 300, 64), (5, 300, 640)])
def test_relu_masks_of_columns_of_another_scale(size, dtype):
    """One column in 64 is 2^8 times as large as the others, and its bias takes the
    sum of one row away but its rounding: decided in 64 bits, though the row's
    other results are small."""
    n, k, m = size
    g = torch.Generator(device="cuda").manual_seed(22)
    x, w = rand((n, k), dtype, g), rand((k, m), dtype, g, 1 / math.sqrt(k))
    w[:, 5::64] *= 2.0 ** 8
    b = rand((m,), torch.float32, g)
    exact = x.double() @ w.double()
    column = torch.arange(5, m, 64, device="cuda")
    for first in range(0, min(n, 96), 3):      # many rows, one after the other
        row = (first + column) % n
        b[column] = -exact[row, column].float()
        y = rsc.linear(x.clone().requires_grad_(), w, b, act="relu").detach()
        assert torch.equal(y > 0, exact + b.double() > 0), first
