"""The 4-bit operators on the GPU against the plain 64-bit forms of oracle/mx4.py.

Codes, scales and values are compared bit for bit.  Sums: products of two codes are
exact, so where every product is a multiple of 2^-a and sum |x| |w| < 2^(24 - a) no
fp32 sum rounds, whatever its order, and results are equal to the bit; elsewhere each of
the K additions is off by at most one unit of the last place (2^-23, rounded or cut) of
a partial sum no larger than sum |x| |w|, the bias counted in.  GELU's polynomial is
2.5e-7 off (for results of 16 bits 6.1e-6, or 4.4e-5 of its value) and its slope at most
1.13; each rounding to the output's type is off by half
a unit."""
import numpy as np
import pytest
import torch

import oracle
import paper_2502_01637_amd as S
from gpu_util import as_bytes, build_gpu, dev
from oracle import mx4
from workloads import CONFIGS, make_workload, scaled

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
EPS = {t: torch.finfo(t).eps / 2 for t in TYPES}


def rng_tensor(seed, shape, dtype, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def f64(t):
    return t.double().cpu().numpy()


def packed(seed, n, cols, lo=120, hi=130):
    """Random 4-bit rows: any code, scale bytes in [lo, hi)."""
    rng = np.random.default_rng(seed)
    g = -(-cols // 128)
    r = np.zeros((n, mx4.row_bytes(cols)), np.uint8)
    codes = rng.integers(0, 16, (n, 128 * g), dtype=np.uint8)
    codes[:, cols:] = 0
    r[:, :64 * g] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    r[:, 64 * g:64 * g - (-cols // 32)] = rng.integers(lo, hi, (n, -(-cols // 32)))
    return r


# ---------------------------------------------------------------- quantise ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,cols,pad,shift", [
    (1, 1, 0, 0), (3, 31, 0, 0), (5, 32, 3, 0), (2, 33, 0, 1), (4, 127, 1, 1), (7, 128, 0, 0),
    (3, 129, 2, 3), (6, 500, 0, 0), (33, 520, 8, 8), (5, 1000, 1, 1), (130, 1024, 0, 0),
    (9, 2049, 0, 0)])
def test_quantize(dtype, n, cols, pad, shift):
    wide = rng_tensor(n * 10000 + cols, n * (cols + pad) + shift, torch.float32, 0.02)
    # rows of very different sizes, single large elements, zeros of both signs
    wide *= torch.exp2(torch.randint(-30, 15, wide.shape, device="cuda",
                                     generator=torch.Generator("cuda").manual_seed(cols)) // 6)
    wide[::7] = 0.0
    wide[3::11] *= -0.0
    x = wide.to(dtype)[shift:].view(n, cols + pad)[:, :cols]
    guard = torch.full((n + 2, S.mx4_row_bytes(cols)), 0xA5, dtype=torch.uint8, device="cuda")
    out = S.Mx4Rows(guard[1:n + 1], cols)
    S.quantize_mx4(x, out=out)
    want = mx4.quantize(x.float().cpu().numpy())
    assert not (out.data.cpu().numpy() != want).sum()
    assert (guard[0] == 0xA5).all() and (guard[-1] == 0xA5).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_special_values(dtype):
    fi = torch.finfo(dtype)
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0]
    row = [0.0, -0.0, fi.max, -fi.max, fi.tiny, fi.smallest_normal / 4, 1.0, -1.0]
    rows = [row + [0.0] * 24,
            mids + [-m for m in mids] + [4.0] + [0.0] * 13,
            [m * (1 + fi.eps) for m in mids] + [-m * (1 - fi.eps / 2) for m in mids] + [4.0] * 14,
            [fi.tiny / 2, -fi.tiny] + [0.0] * 30, [-0.0] * 32,
            [1.0] * 31 + [float("nan")], [float("inf")] + [1.0] * 31, [-float("inf")] * 32]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype).cuda()
    x = torch.cat([x, torch.ones_like(x)], 1).contiguous()   # the next block stays finite
    q = S.quantize_mx4(x)
    assert not (q.data.cpu().numpy() != mx4.quantize(x.float().cpu().numpy())).sum()
    v = S.dequantize_mx4(q, torch.float32)
    assert torch.isnan(v[5:, :32]).all() and (v[:, 32:] == 1).all() and not torch.isnan(v[:5]).any()


# ------------------------------------------------------------------ gather ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,n_tok", [(1, 5), (8, 1), (31, 77), (64, 512), (100, 33), (129, 64),
                                        (1000, 21), (1024, 130), (2048, 9), (5003, 7)])
def test_gather(dtype, cols, n_tok):
    n_rows = 50
    rows = packed(cols, n_rows, cols, 0, 256)     # every scale, NaN among them
    ids = np.random.default_rng(n_tok).integers(0, n_rows, n_tok).astype(np.int32)
    ids[::5] = ids[0]
    want = torch.from_numpy(mx4.values(rows, cols)[ids]).to(dtype)
    table = S.Mx4Rows(dev(rows), cols)
    host = S.HostRows(n_rows, (table.row_bytes,), torch.uint8)
    host.tensor().copy_(torch.from_numpy(rows))
    for t in (table, S.Mx4Rows(host, cols)):
        # an output that starts one element into its memory, with guards around
        buf = torch.full((n_tok * cols + 2,), 77.0, dtype=dtype, device="cuda")
        out = buf[1:-1].view(n_tok, cols)
        assert S.gather_mx4(dev(ids), t, out=out) is out
        S.check_ok()
        assert torch.equal(out.cpu().nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))
        assert buf[0] == 77.0 and buf[-1] == 77.0
        v = S.dequantize_mx4(t, dtype)
        all_want = torch.from_numpy(mx4.values(rows, cols)).to(dtype)
        assert torch.equal(v.cpu().nan_to_num(nan=12345.0), all_want.nan_to_num(nan=12345.0))
    host.close()


def test_gather_bad_ids_and_no_rows():
    rows = packed(1, 4, 200)
    ids = dev(np.array([[3, -1, 0], [4, 2, 2 ** 31 - 1]], np.int32))
    out = S.gather_mx4(ids, S.Mx4Rows(dev(rows), 200), torch.float32)
    assert S.check() == S.scone.EROW and S.check() == S.scone.OK
    want = mx4.values(rows, 200)
    got = f64(out)
    assert out.shape == (2, 3, 200)
    assert np.array_equal(got[0, 0], want[3]) and np.array_equal(got[0, 2], want[0])
    assert np.array_equal(got[1, 1], want[2])
    assert not got[0, 1].any() and not got[1, 0].any() and not got[1, 2].any()
    none = S.Mx4Rows(torch.empty((0, 144), dtype=torch.uint8, device="cuda"), 200)
    out = S.gather_mx4(ids, none)
    assert S.check() == S.scone.EROW and not out.any()
    assert S.gather_mx4(ids[:0], none).shape == (0, 3, 200) and S.check() == S.scone.OK
    assert S.dequantize_mx4(none).shape == (0, 200)


def test_gather_far_rows():
    """Rows and outputs beyond 2^32 bytes."""
    cols, n = 1024, 8_100_000                     # 544 bytes each, 4.4 GB
    table = torch.zeros((n, 544), dtype=torch.uint8, device="cuda")
    at = torch.tensor([0, 7_895_160, 7_895_161, n - 1], device="cuda")
    rows = packed(3, 4, cols)
    table[at] = dev(rows)
    out = S.gather_mx4(at.int(), S.Mx4Rows(table, cols), torch.float32)
    S.check_ok()
    assert np.array_equal(f64(out), mx4.values(rows, cols))
    ids = torch.zeros(2_200_000, dtype=torch.int32, device="cuda")   # 4.5 GB of bf16
    ids[-3:] = at[1:].int()
    out = S.gather_mx4(ids, S.Mx4Rows(table, cols))
    S.check_ok()
    want = torch.from_numpy(mx4.values(rows, cols)).to(torch.bfloat16)
    assert torch.equal(out[-3:].cpu(), want[1:]) and torch.equal(out[-4].cpu(), want[0])
    assert torch.equal(out[1_048_575:1_048_577].cpu(), want[:1].expand(2, -1))


# ------------------------------------------------------------- decode step ----

@pytest.mark.parametrize("K,max_n,cols,n_seq,dtype", [
    (2, 2, 64, 1, torch.float32), (3, 3, 1000, 17, torch.bfloat16), (5, 5, 2048, 8, torch.bfloat16),
    (5, 3, 300, 5, torch.float16), (7, 7, 37, 64, torch.float32), (3, 1, 129, 3, torch.float16),
    (7, 9, 4100, 2, torch.bfloat16)])
@pytest.mark.parametrize("place", ["hbm", "host"])
def test_decode_step(K, max_n, cols, n_seq, dtype, place):
    """The step over 4-bit rows is decode_step over the rows' values, for a few steps."""
    V, n = 40, 300
    rng = np.random.default_rng(K * 100 + cols)
    fg = np.unique(rng.integers(0, V, (2 * n, K)).astype(np.int32), axis=0)
    ln = rng.integers(2, K + 1, len(fg)).astype(np.int32)
    seen, keep = set(), []
    for i, (f, l) in enumerate(zip(fg, ln)):
        if tuple(f[:l]) not in seen:
            seen.add(tuple(f[:l]))
            keep.append(i)
    fg, ln = fg[keep], ln[keep]
    table = build_gpu(fg, ln, np.arange(V, V + len(fg)))
    rows = packed(cols, V + len(fg), cols)
    values = torch.from_numpy(mx4.values(rows, cols)).to(dtype).cuda()
    mx = S.Mx4Rows(dev(rows), cols)
    if place == "host":
        host = S.HostRows(rows.shape[0], (rows.shape[1],), torch.uint8)
        host.tensor().copy_(torch.from_numpy(rows))
        mx = S.Mx4Rows(host, cols)
    cap = max(min(K, max_n) - 1, 1)
    state = [torch.zeros((n_seq, cap), dtype=torch.int32, device="cuda") for _ in range(2)]
    lens = [torch.zeros(n_seq, dtype=torch.int32, device="cuda") for _ in range(2)]
    for step in range(K + 2):
        new = dev(rng.integers(0, V, n_seq).astype(np.int32))
        res = []
        for i in range(2):
            ids = torch.full((n_seq,), -9, dtype=torch.int32, device="cuda")
            ml = torch.zeros(n_seq, dtype=torch.int8, device="cuda")
            out = torch.full((n_seq + 1, cols), 7.0, dtype=dtype, device="cuda")
            if i:
                S.decode_step_mx4(table, state[i], lens[i], new, max_n, mx, out[:n_seq], ids, ml)
            else:
                S.decode_step(table, state[i], lens[i], new, max_n, values, out[:n_seq], ids, ml)
            res.append((out, ids, ml, state[i], lens[i]))
        S.check_ok()
        for a, b in zip(*res):
            assert torch.equal(a, b), step


def test_decode_step_bad_rows_and_tokens():
    table = build_gpu([[1, 2]], [2], [9])
    mx = S.Mx4Rows(dev(packed(5, 6, 70)), 70)
    ctx = dev(np.array([[1], [1], [1]], np.int32))
    clen = torch.ones(3, dtype=torch.int32, device="cuda")
    out = torch.ones((3, 70), dtype=torch.float32, device="cuda")
    S.decode_step_mx4(table, ctx, clen, dev(np.array([2, 5, 3], np.int32)), 2, mx, out)
    assert S.check() == S.scone.EROW and not out[0].any()    # id 9 of 6 rows
    assert torch.equal(out[1:], S.dequantize_mx4(mx, torch.float32)[[5, 3]])
    S.decode_step_mx4(table, ctx, clen, dev(np.array([2, 70000, -1], np.int32)), 2, mx, out)
    assert S.check() == S.scone.ETOKEN


# ------------------------------------------------------------------ linear ----

def linear_case(seed, M, N, K, exact):
    """x, w packed (numpy) with products that are multiples of 1/16 where `exact`."""
    lo, hi = (126, 129) if exact else (117, 131)
    return packed(seed, M, K, lo, hi), packed(seed + 1, N, K, lo, hi)


SIZES = [(1, 1, 1), (1, 16, 128), (1, 100, 1000), (1, 513, 4100), (2, 17, 31), (3, 64, 129),
         (5, 300, 256), (15, 15, 500), (16, 33, 384), (17, 128, 640), (33, 31, 1024), (48, 257, 77),
         (64, 100, 2000), (65, 512, 128), (100, 1, 300), (127, 129, 127), (128, 256, 512),
         (129, 130, 900), (200, 1000, 160), (257, 513, 1030), (300, 260, 2304), (600, 384, 260),
         (1030, 770, 1280)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_sums_to_the_bit(M, N, K):
    """No sum can round: every product is a multiple of 1/16, and sum |x| |w| below 2^20."""
    x, w = linear_case(M * 7 + N, M, N, K, True)
    xv, wv = mx4.values(x, K), mx4.values(w, K)
    want, size = mx4.linear(xv, wv)
    assert size.max() < 2 ** 20
    got = S.linear_mx4(S.Mx4Rows(dev(x), K), S.Mx4Rows(dev(w), K), dtype=torch.float32)
    assert np.array_equal(f64(got), want)


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("x_type,out_type,bias_type,gelu,resid", [
    (torch.bfloat16, torch.bfloat16, torch.bfloat16, True, None),
    (torch.float16, torch.float16, None, False, "new"),
    (torch.float32, torch.float32, torch.float32, True, "in place"),
    (None, torch.float32, torch.float16, False, "in place"),
    (None, torch.bfloat16, torch.bfloat16, False, None)])
def test_linear(M, N, K, x_type, out_type, bias_type, gelu, resid):
    x, w = linear_case(M + 3 * N + K, M, N, K, False)
    if x_type is None:
        xin, xv = S.Mx4Rows(dev(x), K), mx4.values(x, K)
    else:
        xin = rng_tensor(M * N, (M, K + 3), x_type)[:, 1:K + 1]
        xv = mx4.values(mx4.quantize(xin.float().cpu().numpy()), K)
    bias = None if bias_type is None else rng_tensor(N, (N,), bias_type)
    # an output whose rows are longer than N, the elements between them guarded
    ld = N + 5 if M % 2 else N
    buf = torch.full((M + 1, ld), 9.0, dtype=out_type, device="cuda")
    out = buf[:M, :N]
    res = None
    if resid:
        res = rng_tensor(K, (M, ld), out_type)[:, :N]
        if resid == "in place":
            out.copy_(res)
    want, size = mx4.linear(xv, mx4.values(w, K), None if bias is None else f64(bias), gelu,
                            None if res is None else f64(res))
    S.linear_mx4(xin, S.Mx4Rows(dev(w), K), bias, gelu=gelu,
                 residual=out if resid == "in place" else res, out=out)
    got = f64(out)
    tol = (K + 2) * 2.0 ** -23 * size * (1.13 if gelu else 1.0)
    if gelu:
        y = want if res is None else want - f64(res)
        tol = tol + (3e-7 if out_type == torch.float32 else 6.1e-6 + 4.4e-5 * np.abs(y))
    if res is not None:
        tol = tol + 2.0 ** -24 * (np.abs(want) + np.abs(f64(res)))
    tol = tol + EPS[out_type] * (np.abs(want) + tol) + (2.0 ** -25 if out_type == torch.float16
                                                        else 0.0)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) - tol)
    assert (buf[M] == 9.0).all() and (buf[:M, N:] == 9.0).all()


# enough tiles of 128 x 256 for those, with ragged edges, over one to nine groups
BIG = [(4100, 2100, 100), (4100, 2100, 200), (4096, 2048, 384), (2049, 4097, 512),
       (4099, 2305, 640), (4100, 2100, 1100)]


@pytest.mark.parametrize("M,N,K", BIG)
def test_linear_big_tiles(M, N, K):
    """To the bit without a residual; with one, a bias and GELU within the bounds."""
    x, w = linear_case(M + K, M, N, K, True)
    xq, wq = S.Mx4Rows(dev(x), K), S.Mx4Rows(dev(w), K)
    xv = torch.from_numpy(mx4.values(x, K)).cuda()
    wv = torch.from_numpy(mx4.values(w, K)).cuda()
    want, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    assert float(size.max()) < 2 ** 20
    assert torch.equal(S.linear_mx4(xq, wq, dtype=torch.float32).double(), want)
    for dtype in TYPES:
        bias, res = rng_tensor(N, (N,), dtype), rng_tensor(K, (M, N), dtype, 50.0)
        # weights 1/64 as large: GELU where it bends
        small = S.Mx4Rows(wq.data.clone(), K)
        small.data[:, 64 * (-(-K // 128)):64 * (-(-K // 128)) - (-K // 32)] -= 6
        got = S.linear_mx4(xq, small, bias, gelu=True, residual=res, dtype=dtype)
        b64 = bias.double()
        pre = want / 64 + b64
        y = 0.5 * pre * torch.special.erfc(-pre * 0.5 ** 0.5)
        full = y + res.double()
        # the sum with the bias rounds K times at most; GELU's polynomial for results of
        # 16 bits is 6.1e-6 off, or 4.4e-5 of its value
        tol = 1.13 * (K + 2) * 2.0 ** -23 * (size / 64 + b64.abs())
        tol = tol + (3e-7 if dtype == torch.float32 else 6.1e-6 + 4.4e-5 * y.abs())
        tol = tol + 2.0 ** -24 * (full.abs() + res.double().abs())
        tol = tol + EPS[dtype] * (full.abs() + tol) + (2.0 ** -25 if dtype == torch.float16 else 0)
        assert ((got.double() - full).abs() <= tol).all(), dtype
        inplace = res.clone()
        S.linear_mx4(xq, small, bias, gelu=True, residual=inplace, out=inplace)
        assert torch.equal(inplace, got)


@pytest.mark.parametrize("M,N,K", [(1, 40, 300), (16, 64, 1024), (70, 90, 500), (300, 300, 640)])
def test_linear_nan_and_zero_blocks(M, N, K):
    """A NaN block of a row reaches that row (or column) of the output and no other."""
    x, w = linear_case(5, M, N, K, True)
    g = -(-K // 128)
    x[M // 2, 64 * g + 1] = 255
    w[N // 3, 64 * g + 2] = 255
    x[-1, :64 * g] = 0                    # a row of zeros
    got = f64(S.linear_mx4(S.Mx4Rows(dev(x), K), S.Mx4Rows(dev(w), K), dtype=torch.float32))
    xv, wv = mx4.values(x, K), mx4.values(w, K)
    bad = np.zeros((M, N), bool)
    bad[M // 2] = True
    bad[:, N // 3] = True
    want = np.nan_to_num(xv, nan=0.0) @ np.nan_to_num(wv, nan=0.0).T
    assert np.array_equal(np.isnan(got), bad)
    assert np.array_equal(got[~bad], want[~bad])


def test_linear_scales_at_the_ends():
    """Scale bytes 0 and 254: 2^-127 and 2^127, whose products are exact."""
    K = 256
    for M in (1, 20, 300):
        x, w = packed(1, M, K, 0, 1), packed(2, 40, K, 254, 255)
        got = f64(S.linear_mx4(S.Mx4Rows(dev(x), K), S.Mx4Rows(dev(w), K), dtype=torch.float32))
        assert np.array_equal(got, mx4.values(x, K) @ mx4.values(w, K).T)


@pytest.mark.parametrize("M", [3, 70])
def test_linear_products_past_the_range(M):
    """Products past fp32's range are infinities of their sign; codes of 0 stay 0 under
    the largest scales.  Codes are 6 and 0, so that 36 x 2^250 is a product's size."""
    x = torch.zeros((M, 200), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((5, 200), dtype=torch.bfloat16, device="cuda")
    x[:, 0] = 3e38
    w[0, 0], w[1, 1], w[2, 0], w[3, 130], w[4, 0] = 3e38, 3e38, -3e38, 3e38, 2.0 ** -100
    got = f64(S.linear_mx4(x, S.quantize_mx4(w), dtype=torch.float32))
    assert np.array_equal(got, np.tile([np.inf, 0, -np.inf, 0, 6 * 2.0 ** 25], (M, 1)))


def test_linear_empty_sizes():
    w = S.Mx4Rows(dev(packed(1, 8, 100)), 100)
    none = S.Mx4Rows(torch.empty((0, 80), dtype=torch.uint8, device="cuda"), 100)
    x = rng_tensor(1, (3, 100), torch.bfloat16)
    assert S.linear_mx4(x[:0], w).shape == (0, 8)
    assert S.linear_mx4(x, none).shape == (3, 0)
    assert S.linear_mx4(none, w).shape == (0, 8)
    y = S.linear_mx4(rng_tensor(1, (2, 3, 100), torch.bfloat16), w)
    assert y.shape == (2, 3, 8)
    assert torch.equal(y[0], S.linear_mx4(rng_tensor(1, (2, 3, 100), torch.bfloat16)[0], w))
    assert S.linear_mx4(x[0], w).shape == (8,)


def test_linear_far_output():
    """Output offsets beyond 2^31 elements; rows near the end against a small call."""
    M, N, K = 70_000, 32_000, 128
    x, w = rng_tensor(1, (M, K), torch.bfloat16), rng_tensor(2, (N, K), torch.bfloat16)
    wq = S.quantize_mx4(w)
    y = S.linear_mx4(x, wq)
    for m in (0, 33_553, 67_109, M - 64):
        assert torch.equal(y[m:m + 64], S.linear_mx4(x[m:m + 64].contiguous(), wq))


# --------------------------------------------- refusals, streams and graphs ----

def test_a_resized_tensor_of_rows_is_refused():
    rows = S.quantize_mx4(rng_tensor(2, (6, 100), torch.bfloat16))
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    S.gather_mx4(ids, rows)
    rows.data.resize_((2, rows.row_bytes))
    for call in (lambda: S.gather_mx4(ids, rows), lambda: S.dequantize_mx4(rows),
                 lambda: S.linear_mx4(rng_tensor(1, (4, 100), torch.bfloat16), rows)):
        with pytest.raises(ValueError):
            call()


def test_binding_refuses_mismatches():
    x = rng_tensor(1, (4, 100), torch.bfloat16)
    w = S.quantize_mx4(rng_tensor(2, (6, 100), torch.bfloat16))
    bad = [
        (TypeError, lambda: S.quantize_mx4(x.double())),
        (TypeError, lambda: S.quantize_mx4(x.int())),
        (ValueError, lambda: S.quantize_mx4(x[0])),
        (ValueError, lambda: S.quantize_mx4(x[:, ::2])),
        (ValueError, lambda: S.quantize_mx4(x[:1].expand(4, 100))),
        (ValueError, lambda: S.quantize_mx4(x[:, :0])),
        (ValueError, lambda: S.quantize_mx4(x, out=w)),
        (ValueError, lambda: S.Mx4Rows(w.data, 200)),
        (ValueError, lambda: S.Mx4Rows(w.data.view(torch.int8), 100)),
        (ValueError, lambda: S.Mx4Rows(w.data[:, ::2], 100)),
        (TypeError, lambda: S.gather_mx4(torch.zeros(3, dtype=torch.int32, device="cuda"), w,
                                         torch.float64)),
        (ValueError, lambda: S.gather_mx4(torch.zeros(3, dtype=torch.int32, device="cuda"), w,
                                          out=x)),
        (TypeError, lambda: S.gather_mx4(torch.zeros(3, dtype=torch.int64, device="cuda"), w)),
        (ValueError, lambda: S.linear_mx4(x[:, :99], w)),
        (ValueError, lambda: S.linear_mx4(x.t(), w)),
        (ValueError, lambda: S.linear_mx4(x, w, x[0])),
        (ValueError, lambda: S.linear_mx4(x, w, torch.zeros(6))),
        (TypeError, lambda: S.linear_mx4(x, w, torch.zeros(6, dtype=torch.float64, device="cuda"))),
        (ValueError, lambda: S.linear_mx4(x, w, out=x)),
        (ValueError, lambda: S.linear_mx4(x, w, residual=x)),
        (ValueError, lambda: S.linear_mx4(x, w, residual=torch.zeros((4, 6), device="cuda"))),
        (ValueError, lambda: S.linear_mx4(x, w, residual=torch.zeros(
            (4, 7), dtype=torch.bfloat16, device="cuda")[:, :6])),
        (TypeError, lambda: S.linear_mx4(x, w, dtype=torch.float64)),
        (ValueError, lambda: S.linear_mx4(x.view(2, 2, 100)[:, :, :], w,
                                          out=torch.empty((4, 6), device="cuda"))),
        (ValueError, lambda: S.linear_mx4(rng_tensor(1, (2, 4, 100), torch.bfloat16)[:, ::2], w)),
        (S.SconeError, lambda: S.linear_mx4(x.repeat(50, 1), w, workspace=torch.empty(
            16, dtype=torch.uint8, device="cuda"))),
        (ValueError, lambda: S.linear_mx4(x, w, workspace=torch.empty(4096, device="cuda"))),
    ]
    for k, (kind, call) in enumerate(bad):
        with pytest.raises(kind):
            call()
            pytest.fail(f"call {k} was not refused")


def test_streams_and_graph_replay():
    """The whole chain on a side stream, and captured with new inputs at each replay."""
    M, N, K = 70, 260, 600
    w = S.quantize_mx4(rng_tensor(2, (N, K), torch.bfloat16))
    bias = rng_tensor(3, (N,), torch.float32)
    x = rng_tensor(4, (M, K), torch.bfloat16)
    ids = torch.arange(M, dtype=torch.int32, device="cuda") % 7

    def chain(stream=None):
        q = S.quantize_mx4(x, stream=stream)
        v = S.gather_mx4(ids, q, stream=stream)
        y = S.linear_mx4(v, w, bias, gelu=True, stream=stream)
        one = S.linear_mx4(y[:1, :].contiguous() if stream is None else y[:1], wy, stream=stream)
        return v, y, one

    wy = S.quantize_mx4(rng_tensor(5, (50, N), torch.bfloat16))
    want = chain()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for st in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            got = chain(st)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = chain()
    for seed in range(4):
        x.copy_(rng_tensor(10 + seed, (M, K), torch.bfloat16))
        want = chain()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(res, want)), seed


def test_calls_repeat_to_the_bit():
    x = rng_tensor(1, (333, 1500), torch.float16)
    for M in (1, 16, 40, 333):
        w = S.quantize_mx4(rng_tensor(2, (4001, 1500), torch.float16))
        first = S.linear_mx4(x[:M], w)
        for _ in range(3):
            assert torch.equal(S.linear_mx4(x[:M], w), first)


# --------------------------------------------------------- used together ----

def test_table_in_four_bits_end_to_end():
    """A table quantised once, then served: prefill (lookup and gather, or the byte
    calls and a dequantisation), split placement, decoding steps, and a product."""
    cfg = scaled(CONFIGS["tiny"], B=6, T=70)
    wl = make_workload(cfg)
    table = build_gpu(wl.fgrams, wl.lengths, wl.ids)
    d = 320
    E = rng_tensor(1, (cfg.n_rows, d), torch.bfloat16, 0.02)
    q = S.quantize_mx4(E)
    assert np.array_equal(q.data[:50].cpu().numpy(), mx4.quantize(E[:50].float().cpu().numpy()))
    tok = dev(wl.tokens)
    exp_ids, _ = oracle.OracleTable(wl.fgrams, wl.lengths, wl.ids).lookup(wl.tokens, cfg.max_n)
    want = torch.from_numpy(mx4.values(q.data.cpu().numpy(), d)).to(torch.bfloat16)[
        torch.from_numpy(exp_ids).long()]
    ids, _ = S.lookup(table, tok, cfg.max_n)
    out = S.gather_mx4(ids, q)
    assert torch.equal(out.cpu(), want)
    raw = S.embed(table, tok, cfg.max_n, q.data)              # the packed rows as bytes
    flat = S.dequantize_mx4(S.Mx4Rows(raw.view(-1, q.row_bytes), d))
    assert torch.equal(flat.view_as(out), out)
    far = S.HostRows(cfg.n_rows - cfg.V, (q.row_bytes,), torch.uint8)
    far.tensor().copy_(q.data[cfg.V:])
    ws = torch.empty(S.split_workspace_bytes(ids.numel(), q.row_bytes), dtype=torch.uint8,
                     device="cuda")
    split = S.gather_split(ids, q.data[:cfg.V], far, ws)
    flat = S.dequantize_mx4(S.Mx4Rows(split.view(-1, q.row_bytes), d))
    assert torch.equal(flat.view_as(out), out)
    ctx = torch.zeros((cfg.B, max(cfg.max_n - 1, 1)), dtype=torch.int32, device="cuda")
    clen = torch.zeros(cfg.B, dtype=torch.int32, device="cuda")
    step = torch.empty((cfg.B, d), dtype=torch.bfloat16, device="cuda")
    for t in range(5):
        S.decode_step_mx4(table, ctx, clen, tok[:, t].contiguous(), cfg.max_n, q, step)
        assert torch.equal(step, out[:, t])
    S.check_ok()
    w = S.quantize_mx4(rng_tensor(2, (77, d), torch.bfloat16, 0.05))
    y = S.linear_mx4(out, w, dtype=torch.float32)
    xq = S.quantize_mx4(out.view(-1, d))
    # the values of 4-bit rows are held as they are
    assert torch.equal(S.dequantize_mx4(xq), out.view(-1, d))
    assert torch.equal(S.linear_mx4(xq, w, dtype=torch.float32), y.view(-1, 77))
    assert as_bytes(out).size == out.numel() * 2
    far.close()
