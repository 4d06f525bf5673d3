"""GELU behind the 4-bit linear map, value by value, in every kernel and output type.

Weights of zeros leave the biases as the sums, so that a row of results is GELU of the
biases.  The form is max(x, 0) - z 2^P(z) with z = |x|, held at z = 7: over [0, 7] P lies
within 1.41e-4 of log2 Phi(-z) (9.74e-5 of the value 2^P) and the roundings of its float
steps are at most 1.2e-5 of it, the exponential's and the product's 2^-22 together, so
that negative results down to x = -7 are off by 1.1e-4 of themselves at most; beyond -7
GELU and the result both lie within 9.1e-12 of 0.  Positive results are off by 2.5e-7.
The rounding to 16 bits adds half a unit of the last place, for fp16's subnormal
results half of 2^-24."""
import numpy as np
import pytest
import torch
from scipy.special import erfc

import paper_2502_01637_amd as S

pytestmark = pytest.mark.gpu


def bound(x, y, dtype):
    tol = np.where(x > 0, 2.5e-7, np.where(x < -7, 9.1e-12, 1.1e-4 * np.abs(y)))
    sub = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}[dtype]
    return tol + torch.finfo(dtype).eps / 2 * (np.abs(y) + tol) + sub


# rows up to 64 and up to 128 large tiles take other kernels than those beyond
@pytest.mark.parametrize("M,N", [(1, 4096), (40, 512), (100, 1024), (2048, 4096), (1100, 8191)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
def test_gelu_of_every_value(M, N, dtype, residual):
    K = 64
    w = S.quantize_mx4(torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"))
    x = torch.randn((M, K), generator=torch.Generator("cuda").manual_seed(M), device="cuda")
    # a residual of zeros leaves the values as they are
    res = torch.zeros((M, N), dtype=dtype, device="cuda") if residual else None
    for lo, hi in [(-8.0, -3.0), (-3.0, 0.0), (0.0, 8.0), (-40.0, -8.0)]:
        b = torch.linspace(lo, hi, N, dtype=torch.float64).float()
        got = S.linear_mx4(x, w, b.cuda(), gelu=True, residual=res, dtype=dtype)
        v = b.double().numpy()
        y = 0.5 * v * erfc(-v * np.sqrt(0.5))
        err = np.abs(got.double().cpu().numpy() - y)
        over = (err - bound(v, y, dtype)).max(axis=0)
        at = np.argmax(over)
        assert over[at] <= 0, (v[at], y[at], over[at])


@pytest.mark.parametrize("M", [1, 100, 2048])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_gelu_of_infinities_and_nan(M, dtype):
    """As x Phi(x) computes them: inf stays, -inf (times 0) and NaN give NaN."""
    N, K = 4096, 64
    w = S.quantize_mx4(torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"))
    b = torch.zeros(N)
    b[3], b[700], b[4095] = float("inf"), -float("inf"), float("nan")
    got = S.linear_mx4(torch.zeros((M, K), device="cuda"), w, b.cuda(), gelu=True,
                       dtype=dtype).cpu()
    assert (got[:, 3] == float("inf")).all() and torch.isnan(got[:, [700, 4095]]).all()
    got[:, [3, 700, 4095]] = 0
    assert not got.any()


@pytest.mark.parametrize("M,N", [(100, 1024), (1100, 8191)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_a_value_does_not_depend_on_its_tile(M, N, dtype):
    """Equal rows give equal results in whole tiles and in tiles over an edge, and their
    16-bit results are the fp32 ones rounded to nearest."""
    K = 64
    w = S.quantize_mx4(torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"))
    x = torch.zeros((M, K), device="cuda")
    for lo, hi in [(-8.0, 0.0), (0.0, 8.0)]:
        b = torch.linspace(lo, hi, N, dtype=torch.float64).float().cuda()
        got = S.linear_mx4(x, w, b, gelu=True, dtype=dtype)
        assert torch.equal(got, S.linear_mx4(x, w, b, gelu=True, dtype=torch.float32).to(dtype))
        assert torch.equal(got, got[:1].expand(M, N))
