"""Few rows of x that the 4-bit linear map quantises itself: at every width of a row and
every alignment of its start the codes are those of quantize_mx4."""
import pytest
import torch

import paper_2502_01637_amd as S

pytestmark = pytest.mark.gpu

WIDTHS = list(range(1, 140)) + [255, 256, 257, 383, 500, 1000, 1023, 1025, 1500, 2047, 4100]


@pytest.mark.parametrize("M,dtype", [(M, t) for t in (torch.bfloat16, torch.float16, torch.float32)
                                     for M in (1, 5, 16, 19, 32, 33) if M <= 32 or t.itemsize == 2])
def test_rows_are_quantised_as_by_quantize_mx4(M, dtype):
    """Both sides sum in the same order, so that equal codes give equal results; what
    lies around the rows is NaN."""
    for K in [K for K in WIDTHS if M <= 16 or K <= 2048]:   # beyond, tiles take them
        g = torch.Generator("cuda").manual_seed(K * 100 + M)
        pad = K % 5
        buf = torch.full((M * (K + pad) + 9,), float("nan"), dtype=dtype, device="cuda")
        x = buf[K % 7:][:M * (K + pad)].view(M, K + pad)[:, :K]
        x.copy_(torch.randn((M, K), generator=g, device="cuda")
                * torch.exp2(torch.randint(-8, 9, (M, K), generator=g, device="cuda").float()))
        w = S.quantize_mx4(torch.randn((20, K), generator=g, device="cuda"))
        got = S.linear_mx4(x, w, dtype=torch.float32)
        assert torch.equal(got, S.linear_mx4(S.quantize_mx4(x), w, dtype=torch.float32)), K
        assert torch.isfinite(got).all(), K


@pytest.mark.parametrize("M", [9, 16, 17, 32, 33, 64, 65])
@pytest.mark.parametrize("N,K", [(1024, 4100), (4001, 1500), (8300, 2100), (16400, 500)])
@pytest.mark.parametrize("dtype", [None, torch.bfloat16, torch.float32])
def test_both_sides_of_the_row_limits(M, N, K, dtype):
    """Products whose sums no order of adding rounds, whichever kernel takes them: x of
    whole numbers up to 6 (one scale), w of halves and scales of 1."""
    g = torch.Generator("cuda").manual_seed(M + K)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    x, w = (grid[torch.randint(0, 8, (n, K), generator=g, device="cuda")]
            * (torch.randint(0, 2, (n, K), generator=g, device="cuda") * 2 - 1) for n in (M, N))
    x[:, ::32], w[:, ::32] = 6.0, 4.0          # every block's largest: scale 1
    xin = S.quantize_mx4(x) if dtype is None else x.to(dtype)
    got = S.linear_mx4(xin, S.quantize_mx4(w), dtype=torch.float32)
    assert 36 * K < 2 ** 22                    # multiples of 1/4 below 2^22: 24 bits
    assert torch.equal(got.double(), x.double() @ w.double().t())


@pytest.mark.parametrize("M,N,K", [(1530, 4000, 1100), (1600, 4000, 1100), (1020, 4001, 4100),
                                   (1100, 4001, 4100), (12000, 520, 300), (8300, 1000, 200)])
@pytest.mark.parametrize("residual", [False, True])
def test_both_sides_of_the_tile_limits(M, N, K, residual):
    """As above, around 192 and (over a long K) 128 large tiles."""
    g = torch.Generator("cuda").manual_seed(M + K)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    x, w = (grid[torch.randint(0, 8, (n, K), generator=g, device="cuda")]
            * (torch.randint(0, 2, (n, K), generator=g, device="cuda") * 2 - 1) for n in (M, N))
    x[:, ::32], w[:, ::32] = 6.0, 4.0
    bias = torch.randint(-8, 9, (N,), generator=g, device="cuda").float()
    res = torch.randint(-99, 99, (M, N), generator=g, device="cuda").float() if residual else None
    got = S.linear_mx4(x, S.quantize_mx4(w), bias, residual=res)
    want = x.double() @ w.double().t() + bias.double()
    assert torch.equal(got.double(), want if res is None else want + res.double())
