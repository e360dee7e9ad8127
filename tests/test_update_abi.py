"""The update phase's C ABI without a GPU: bad arguments are refused with the
documented status before anything is launched, and the workspace sizes of the
documented sizes are finite and monotone."""
import ctypes
import os

import pytest

import paper_2210_10737_amd as rsc

BAD, UNSUPPORTED, CAPACITY = "RSC_ERR_INVALID_ARGUMENT", "RSC_ERR_UNSUPPORTED", "RSC_ERR_CAPACITY"
no_gpu = pytest.mark.skipif(__import__("torch").cuda.is_available(), reason="a GPU is visible")
WS = 0x100000


def name(status):
    return rsc.STATUS[status]


def layer(dtype=0, act=0, n=10, k=20, m=12, out_major=0, alpha=1.0, beta=1.0):
    return rsc.LinearStruct(dtype, act, n, k, m, out_major, alpha, beta)


def forward(p=None, X=0x1000, ldx=32, W=0x2000, ldw=32, bias=None, bias_dtype=0, R=None, ldr=16, Y=0x4000, ldy=16,
            pre=None, ldpre=16, ws=WS, ws_bytes=1 << 30):
    p = layer() if p is None else p
    return name(rsc.lib().rsc_linear(ctypes.byref(p) if p else None, X, ldx, W, ldw, bias, bias_dtype, R, ldr, Y, ldy,
                                     pre, ldpre, ws, ws_bytes, None))


def test_linear_refusals():
    assert forward(p=False) == BAD
    for bad in (dict(dtype=3), dict(dtype=-1), dict(act=4), dict(act=-1), dict(n=-1), dict(k=0), dict(m=0)):
        assert forward(layer(**bad)) == BAD, bad
    assert forward(X=None) == BAD and forward(W=None) == BAD and forward(Y=None) == BAD
    assert forward(ldx=16) == BAD                         # ld < k
    assert forward(ldw=8) == BAD and forward(layer(out_major=1), ldw=16) == BAD
    assert forward(ldx=22) == UNSUPPORTED                 # no whole 16 bytes
    assert forward(layer(dtype=1), ldx=28) == UNSUPPORTED
    assert forward(ldx=(1 << 20) + 4) == UNSUPPORTED      # rows over 4 MiB
    assert forward(X=0x1004) == UNSUPPORTED and forward(Y=0x4008) == UNSUPPORTED
    assert forward(bias=0x1001) == UNSUPPORTED
    assert forward(bias=0x1000, bias_dtype=1) == BAD      # a bf16 bias of an fp32 layer
    assert forward(R=0x5000, ldr=8) == BAD
    assert forward(pre=0x4000) == BAD                     # pre is Y
    assert forward(Y=0x1000, ldy=32) == BAD               # Y is X
    assert forward(layer(n=1 << 30, m=1 << 18), ldy=1 << 18, ldw=1 << 18) == UNSUPPORTED   # too many tiles
    assert forward(layer(n=2 ** 31 - 1)) == UNSUPPORTED
    big = layer(n=64, k=8192, m=64)
    need = rsc.lib().rsc_linear_workspace_bytes(ctypes.byref(big))
    assert need > 0                                       # few tiles, a long sum: split
    assert forward(big, ldx=8192, ldw=64, ldy=64, ws_bytes=need - 1) == CAPACITY
    assert forward(big, ldx=8192, ldw=64, ldy=64, ws=None) == BAD
    assert forward(big, ldx=8192, ldw=64, ldy=64, ws=WS + 16) == UNSUPPORTED


def test_linear_backward_refusals():
    def call(p=None, dY=0x1000, lddy=16, saved=None, lds=16, X=0x2000, ldx=32, W=0x3000, ldw=16, dX=0x5000, lddx=32,
             dW=0x6000, lddw=16, db=None, db_dtype=0, dR=None, lddr=16, ws=WS, ws_bytes=1 << 30):
        p = layer() if p is None else p
        return name(rsc.lib().rsc_linear_backward(ctypes.byref(p), dY, lddy, saved, lds, X, ldx, W, ldw, dX, lddx, dW,
                                                  lddw, db, db_dtype, dR, lddr, ws, ws_bytes, None))

    assert call(dY=None) == BAD
    assert call(layer(act=1)) == BAD                      # nothing saved for a ReLU
    assert call(layer(act=2), saved=0x7004) == UNSUPPORTED
    assert call(X=None) == BAD and call(W=None) == BAD
    assert call(dX=0x5004) == UNSUPPORTED and call(lddw=8) == BAD and call(dR=0x8000, lddr=13) == UNSUPPORTED
    assert call(db=0x8000, db_dtype=2) == BAD
    need = rsc.lib().rsc_linear_backward_workspace_bytes(ctypes.byref(layer(act=1)), 1, 1, 1)
    assert call(layer(act=1), saved=0x7000, db=0x8000, ws_bytes=need - 1) == CAPACITY


def loss(dtype=0, n=10, k=20, v=12, out_major=0, reduction=2, i32=0, bias_dtype=0, ignore=-100):
    return rsc.XentStruct(dtype, n, k, v, out_major, reduction, i32, bias_dtype, ignore)


def test_xent_refusals():
    def call(p=None, X=0x1000, ldx=32, W=0x2000, ldw=16, bias=None, t=0x3000, out=0x4000, lse=0x5000, count=0x6000,
             ws=WS, ws_bytes=1 << 30, G=None, ldg=16):
        p = loss() if p is None else p
        return name(rsc.lib().rsc_xent(ctypes.byref(p), X, ldx, W, ldw, bias, t, out, lse, count, G, ldg, ws, ws_bytes,
                                       None))

    for bad in (dict(dtype=3), dict(n=-1), dict(k=0), dict(v=0), dict(reduction=3), dict(reduction=-1)):
        assert call(loss(**bad)) == BAD, bad
    for null in ("X", "W", "t", "out", "lse", "count"):
        assert call(**{null: None}) == BAD, null
    assert call(t=0x3004) == UNSUPPORTED and call(t=0x3002, p=loss(i32=1)) == UNSUPPORTED
    assert call(out=0x4002) == UNSUPPORTED and call(ldx=22) == UNSUPPORTED and call(ldw=8) == BAD
    assert call(loss(bias_dtype=1), bias=0x7000) == BAD
    assert call(loss(v=65), ldw=68, G=0x8000, ldg=68) == UNSUPPORTED and call(loss(reduction=0), G=0x8000) == UNSUPPORTED
    assert call(G=0x8004) == UNSUPPORTED and call(G=0x8000, ldg=8) == BAD
    need = rsc.lib().rsc_xent_workspace_bytes(ctypes.byref(loss()))
    assert call(ws_bytes=need - 1) == CAPACITY and call(ws=None) == BAD and call(ws=WS + 8) == UNSUPPORTED

    def back(p=None, d=0x9000, X=0x1000, W=0x2000, t=0x3000, lse=0x5000, count=0x6000, dX=0xa000, lddx=32, dW=0xb000,
             lddw=16, db=None, ws=WS, ws_bytes=1 << 30, G=None, ldg=16):
        p = loss() if p is None else p
        return name(rsc.lib().rsc_xent_backward(ctypes.byref(p), d, X, 32, W, 16, None, t, lse, count, G, ldg, dX, lddx,
                                                dW, lddw, db, ws, ws_bytes, None))

    for null in ("d", "X", "W", "t", "lse", "count"):
        assert back(**{null: None}) == BAD, null
    assert back(lddx=16) == BAD and back(dW=0xb004) == UNSUPPORTED
    need = rsc.lib().rsc_xent_backward_workspace_bytes(ctypes.byref(loss()), 1, 1, 0)
    assert back(ws_bytes=need - 1) == CAPACITY
    assert back(loss(reduction=0), G=0x8000) == UNSUPPORTED and back(G=0x8000, ldg=13) == UNSUPPORTED


def tensor(param=0x1000, grad=0x2000, m=0x3000, v=0x4000, master=None, ms=None, vs=None, n=100):
    return (ctypes.c_uint64 * 8)(param or 0, grad or 0, m or 0, v or 0, master or 0, ms or 0, vs or 0, n & (2 ** 64 - 1))


def test_adamw_refusals():
    def call(t=None, count=1, step=0x8000, ws=WS, ws_bytes=256, **opts):
        o = {**dict(dtype=0, bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.01), **opts}
        p = rsc.AdamwStruct(o["dtype"], o["bits"], o["lr"], o["b1"], o["b2"], o["eps"], o["wd"], 0)
        return name(rsc.lib().rsc_adamw_step(ctypes.byref(p), tensor() if t is None else t, count, step, ws, ws_bytes, None))

    for bad in (dict(dtype=5), dict(bits=16), dict(b1=1.0), dict(b2=-0.1), dict(eps=-1e-8), dict(lr=float("nan")),
                dict(lr=float("inf")), dict(wd=float("nan")), dict(b1=float("nan")), dict(count=-1), dict(step=None),
                dict(t=tensor(param=None)), dict(t=tensor(grad=None)), dict(t=tensor(m=None)), dict(t=tensor(n=-1)),
                dict(bits=8), dict(ws=None)):
        assert call(**bad) == BAD, bad
    for bad in (dict(step=0x8004), dict(t=tensor(param=0x1002)), dict(t=tensor(v=0x4001)), dict(t=tensor(master=0x1001)),
                dict(t=tensor(n=1 << 34)), dict(bits=8, t=tensor(ms=0x5002, vs=0x6000)), dict(ws=WS + 4)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(ws_bytes=255) == CAPACITY
    L = rsc.lib()
    outs = (ctypes.c_uint64 * 1)(0)
    assert name(L.rsc_adamw_moments(tensor(ms=0x5000, vs=0x6000), 1, outs, outs, None)) == BAD
    assert name(L.rsc_adamw_moments(tensor(), 1, outs, outs, None)) == BAD
    assert name(L.rsc_adamw_moments(None, 1, outs, outs, None)) == BAD


@no_gpu
def test_without_a_device():
    assert forward() == "RSC_ERR_NO_DEVICE"


def test_workspaces_hold_any_documented_size():
    L = rsc.lib()
    for dtype in (0, 1, 2):
        for n in (0, 1, 7, 300, 5000, 700000, 3000000):
            for k, m in ((1, 1), (64, 41), (300, 512), (4096, 4096), (1024, 131072)):
                for out_major in (0, 1):
                    if -(-n // 32) * -(-m // 64) > 1 << 24:
                        assert L.rsc_linear_backward_workspace_bytes(ctypes.byref(layer(n=n, k=k, m=m)), 1, 1, 1) == 0
                        continue
                    p = layer(dtype=dtype, act=1, n=n, k=k, m=m, out_major=out_major)
                    all_of = L.rsc_linear_backward_workspace_bytes(ctypes.byref(p), 1, 1, 1)
                    for flags in ((0, 0, 1), (0, 1, 0), (1, 0, 0)):
                        assert L.rsc_linear_backward_workspace_bytes(ctypes.byref(p), *flags) <= all_of < 1 << 42
                    q = loss(dtype=dtype, n=n, k=k, v=m, out_major=out_major)
                    some = L.rsc_xent_backward_workspace_bytes(ctypes.byref(q), 0, 1, 0)
                    assert 0 < some <= L.rsc_xent_backward_workspace_bytes(ctypes.byref(q), 1, 1, 0) < 1 << 42
                    assert 0 < L.rsc_xent_workspace_bytes(ctypes.byref(q)) < 1 << 42


def test_python_checks_without_a_device():
    torch = __import__("torch")
    x, w = torch.ones(3, 4), torch.ones(4, 5)
    with pytest.raises(ValueError):
        rsc.linear(x, w, act="tanh")
    with pytest.raises(ValueError):
        rsc.linear_cross_entropy(x, w, torch.zeros(3), reduction="mean")
    with pytest.raises(ValueError):
        rsc.AdamW([torch.nn.Parameter(x)], state_bits=4)
    assert os.path.exists(rsc.LIB_PATH)


def test_results_on_operands_are_refused():
    """Also where only their ends, or some of their columns, meet."""
    # X: 10 x 20 in rows of 32 (1,280 bytes), W: 20 x 12, ldw 32 (2,480 up to the last value)
    assert forward(Y=0x1000 + 9 * 128 + 64) == BAD            # Y's first row in X's last one
    assert forward(Y=0x2000 - 64 * 9 - 32, ldy=16) == BAD     # Y's last row in W's first one
    assert forward(R=0x4040) == BAD                           # R a row further on than Y
    assert forward(R=0x4000, ldr=32) == BAD                   # R is Y, in other rows
    assert forward(bias=0x4000 + 64 * 4 + 16) == BAD
    assert forward(pre=0x4000 + 64 * 3) == BAD
    assert forward(X=0x1000, ldx=32, Y=0x1000 + 64, ldy=32) == BAD    # columns 16 to 27 of X's rows, X has 20

    def back(p=None, dY=0x1000, X=0x2000, W=0x3000, dX=0x5000, lddx=32, dW=0x6000, db=None, dR=None, saved=None):
        p = layer(act=1) if saved else layer()
        return name(rsc.lib().rsc_linear_backward(ctypes.byref(p), dY, 16, saved, 16, X, 32, W, 16, dX, lddx, dW, 16, db, 0,
                                                  dR, 16, WS, 1 << 30, None))

    for bad in (dict(dX=0x1000), dict(dX=0x2000), dict(dX=0x3000), dict(dW=0x3000), dict(dW=0x2000 + 128), dict(dW=0x5000),
                dict(dR=0x1000), dict(dR=0x6000), dict(db=0x3000), dict(db=0x5010), dict(saved=0x7000, dR=0x7000),
                dict(saved=0x7000, dX=0x7000)):
        assert back(**bad) == BAD, bad

    def xent(out=0x4000, lse=0x5000, count=0x6000, G=None, X=0x1000, t=0x3000):
        return name(rsc.lib().rsc_xent(ctypes.byref(loss()), X, 32, 0x2000, 16, None, t, out, lse, count, G, 16, WS, 1 << 30,
                                       None))

    for bad in (dict(out=0x5004), dict(lse=0x5000, count=0x5024), dict(lse=0x3010), dict(G=0x1000), dict(G=0x2000),
                dict(out=0x1000), dict(G=0x8000, count=0x8000)):
        assert xent(**bad) == BAD, bad

    def xback(dX=0xa000, dW=0xb000, db=None, G=None):
        return name(rsc.lib().rsc_xent_backward(ctypes.byref(loss()), 0x9000, 0x1000, 32, 0x2000, 16, None, 0x3000, 0x5000,
                                                0x6000, G, 16, dX, 32, dW, 16, db, WS, 1 << 30, None))

    for bad in (dict(dX=0x1000), dict(dW=0x2000), dict(dX=0x2000), dict(dX=0xb000), dict(db=0xa000), dict(db=0x5000),
                dict(G=0x8000, dX=0x8010)):
        assert xback(**bad) == BAD, bad


@no_gpu
def test_column_ranges_of_one_matrix_are_apart():
    ok = "RSC_ERR_NO_DEVICE"
    assert forward(X=0x10000, ldx=32, Y=0x10000 + 80, ldy=32) == ok       # columns 20 to 31 beside X's 0 to 19
    assert forward(X=0x10000 + 48, ldx=32, Y=0x10000, ldy=32) == ok       # and before them
    assert forward(R=0x4000) == ok                                        # in place
    assert forward(layer(n=1), R=0x4000, ldr=32) == ok
    assert forward(Y=0x1000 + 9 * 128 + 80) == ok                         # right behind X's last value
