"""The 4-bit calls refuse bad arguments on the host, before any HIP call."""
import ctypes

import pytest
import torch

import paper_2502_01637_amd as S

# fake device addresses: only where no GPU is visible (see test_abi_cpu.py)
pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: for a process without a GPU")

E, H, OK = S.scone.EINVAL, S.scone.EHIP, S.scone.OK
BF16, F16, F32, MX4 = S.scone.BF16, S.scone.FP16, S.scone.FP32, S.scone.MX4


def at(k, off=0):
    return ctypes.c_void_p((k << 36) + off)


def test_quantize_refusals():
    Q = S.scone.lib().scone_quantize_mx4

    def q(x=at(1), t=BF16, n=10, cols=100, ld=100, rows=at(2)):
        return Q(x, t, n, cols, ld, rows, None)

    assert q() == H                       # past the checks: the first HIP call fails here
    assert q(n=0, x=None, rows=None) == OK
    for bad in (dict(t=MX4), dict(t=9), dict(t=-1), dict(n=-1), dict(cols=0), dict(cols=-3),
                dict(cols=(1 << 22) + 1, ld=1 << 23), dict(ld=99), dict(ld=1 << 60),
                dict(x=None), dict(rows=None), dict(x=at(1, 1)), dict(x=at(1, 2), t=F32),
                dict(rows=at(2, 8))):
        assert q(**bad) == E, bad
    # rows of 80 bytes over x, from either side; next to it they are fine
    assert q(rows=at(1, 16 * 124)) == E and q(x=at(2, 798)) == E
    assert q(rows=at(1, 2000)) == H and q(x=at(2, 800)) == H


def test_gather_refusals():
    G = S.scone.lib().scone_gather_mx4

    def g(ids=at(1), n=10, rows=at(2), n_rows=20, cols=100, out=at(3), t=BF16, place=0):
        return G(ids, n, rows, n_rows, cols, out, t, place, None)

    assert g() == H and g(place=1) == H and g(ids=None) == H
    assert g(n=0, ids=None, rows=None, out=None) == OK
    for bad in (dict(t=MX4), dict(t=7), dict(n=-1), dict(n_rows=-1), dict(cols=0),
                dict(cols=(1 << 22) + 1), dict(place=2), dict(out=None), dict(rows=None),
                dict(ids=None, n=21), dict(n=1 << 60), dict(out=at(3, 1)),
                dict(out=at(3, 2), t=F32), dict(rows=at(2, 4)),
                dict(out=at(1, 36)), dict(ids=at(3, 1996)), dict(out=at(2, 1598)),
                dict(rows=at(3, 1984))):
        assert g(**bad) == E, bad


def test_decode_step_refusals():
    D = S.scone.lib().scone_decode_step_mx4
    tbl = ctypes.create_string_buffer(64)

    def d(tb=tbl, ctx=at(1), clen=at(2), cap=4, new=at(3), n=5, max_n=3, rows=at(4), n_rows=20,
          cols=100, place=0, out=at(5), t=BF16, ids=at(6), lens=at(7)):
        return D(tb, ctx, clen, cap, new, n, max_n, rows, n_rows, cols, place, out, t, ids, lens,
                 None)

    assert d() == H and d(ids=None, lens=None) == H and d(n=0) == OK
    for bad in (dict(tb=None), dict(n=-1), dict(max_n=0), dict(cap=64), dict(cols=0),
                dict(cols=(1 << 22) + 1), dict(place=3), dict(t=MX4), dict(out=None),
                dict(clen=None), dict(new=None), dict(rows=None), dict(n_rows=-1),
                dict(out=at(5, 1)), dict(rows=at(4, 8)), dict(out=at(1, 78)), dict(ids=at(5)),
                dict(lens=at(6, 3)), dict(out=at(4, 1598)), dict(new=at(2, 16)),
                dict(n=1 << 61)):
        assert d(**bad) == E, bad


def test_linear_refusals():
    lib = S.scone.lib()
    W = lib.scone_linear_mx4_workspace
    need = W(200, 30, 100, BF16)
    assert need >= 230 * 68                   # both operands in 4 bits

    def f(x=at(1), t=BF16, ld=100, M=200, K=100, w=at(2), N=30, bias=at(3), bt=BF16, act=1,
          res=None, out=at(4), ot=BF16, ldo=30, ws=at(5), wsb=need):
        return lib.scone_linear_mx4(x, t, ld, M, K, w, N, bias, bt, act, res, out, ot, ldo, ws,
                                    wsb, None)

    assert f() == H and f(bias=None, bt=99) == H and f(res=at(4)) == H and f(res=at(6)) == H
    assert f(t=MX4, ld=0) == H and f(M=10, ws=None, wsb=0) == H
    assert f(M=0, x=None) == OK and f(N=0, w=None, ldo=0) == OK
    for bad in (dict(t=5), dict(t=-1), dict(ot=MX4), dict(ot=8), dict(M=-1), dict(N=-1),
                dict(K=0), dict(K=(1 << 22) + 1, ld=1 << 23), dict(M=1 << 31), dict(N=1 << 31),
                dict(act=2), dict(act=-1), dict(bt=MX4), dict(ld=99), dict(ldo=29),
                dict(ld=(1 << 28) + 1), dict(ldo=(1 << 28) + 1), dict(x=None), dict(w=None),
                dict(out=None), dict(w=at(2, 8)), dict(x=at(1, 1)), dict(x=at(1, 2), t=F32),
                dict(x=at(1, 8), t=MX4), dict(out=at(4, 1)), dict(bias=at(3, 1)),
                dict(res=at(6, 1)), dict(ws=None), dict(wsb=need - 1), dict(ws=at(5, 8)),
                # the output over x, the weights, the biases, the scratch; a residual
                # that lies over it without being it
                dict(out=at(1, 39998)), dict(out=at(2, 2398)), dict(out=at(3, 58)),
                dict(out=at(5, 798)), dict(res=at(4, 2)),
                # the scratch over what is read
                dict(ws=at(1, 16)), dict(ws=at(2, 2384)), dict(ws=at(3, 48)),
                dict(ws=at(6), res=at(6, 16))):
        assert f(**bad) == E, bad
    assert W(200, 30, 100, MX4) == need
    assert W(1, 30, 100, F32) == W(0, 30, 100, F32) == W(200, 0, 100, F32) == 0
    for a in ((-1, 3, 3, BF16), (3, -1, 3, BF16), (3, 3, 0, BF16), (3, 3, 3, 4),
              (1 << 31, 3, 3, BF16), (3, 3, (1 << 22) + 1, MX4)):
        assert W(*a) == -1


def test_binding_refusals():
    x = torch.zeros(3, 4)
    with pytest.raises(TypeError):
        S.quantize_mx4(x)
    with pytest.raises(TypeError):
        S.Mx4Rows(torch.zeros((3, 80), dtype=torch.uint8), 100)
    with pytest.raises(TypeError):
        S.linear_mx4(x, x)
    with pytest.raises(TypeError):
        S.gather_mx4(torch.zeros(3, dtype=torch.int32), x)
    with pytest.raises(TypeError):
        S.dequantize_mx4(x)
    assert S.linear_mx4_workspace_bytes(200, 30, 100, torch.float16) >= 230 * 68
    assert S.linear_mx4_workspace_bytes(10, 30, 100) == 0
    with pytest.raises(ValueError):
        S.linear_mx4_workspace_bytes(-1, 30, 100)
    with pytest.raises(TypeError):
        S.linear_mx4_workspace_bytes(1, 30, 100, torch.int32)


def test_model_refusals():
    L = S.scone.lib()
    Q, F = L.scone_fgram_model_quantize, L.scone_fgram_model_forward_mx4
    B, W = L.scone_fgram_model_mx4_bytes, L.scone_fgram_model_workspace_mx4
    row = 16 * 17                                     # 512 elements
    assert B(512, 8, 1024, 3) == 3 * ((4 * 512 + 1024) * row + 512 * 2 * row)
    assert B(512, 8, 1024, 0) == 0
    assert B(500, 8, 1024, 1) == B(512, 8, 1000, 1) == B(512, 8, 1024, -1) == -1
    assert W(100, 3, 512, 8, 1024) > L.scone_fgram_model_workspace(100, 3, 512, 8, 1024)
    assert W(-1, 3, 512, 8, 1024) == W(100, 9, 512, 8, 1024) == -1
    n = B(512, 8, 1024, 2)
    assert Q(at(1), 512, 8, 1024, 2, 3, at(2), None) == H
    assert Q(None, 512, 8, 1024, 0, 3, None, None) == OK
    for bad in ((None, 512, 8, 1024, 2, 3, at(2)), (at(1), 512, 8, 1024, 2, 3, None),
                (at(1), 500, 8, 1024, 2, 3, at(2)), (at(1), 512, 8, 1024, 2, 8, at(2)),
                (at(1, 8), 512, 8, 1024, 2, 3, at(2)), (at(1), 512, 8, 1024, 2, 3, at(2, 4)),
                (at(1), 512, 8, 1024, 2, 3, at(1, 4096))):
        assert Q(*bad, None) == E, bad

    def f(n=5, weights=at(5), rows=at(6), ws=at(7), wsb=1 << 34, params=at(4)):
        return F(at(1), at(2), at(3), n, 3, at(8), 100, params, weights, 512, 8, 1024, 2, rows, 90,
                 ws, wsb, None)

    assert f(n=0, weights=None) == OK
    for bad in (dict(weights=None), dict(weights=at(5, 8)), dict(rows=at(5, n - 16)),
                dict(ws=at(5, -256)), dict(wsb=1000), dict(ws=at(7, 16)), dict(n=-1),
                dict(params=None)):
        assert f(**bad) == E, bad
