"""Few rows of x that the 4-bit linear map quantises itself: at every width of a row and
every alignment of its start the codes are those of quantize_mx4."""
import pytest
import torch

import paper_2502_01637_amd as S

pytestmark = pytest.mark.gpu

WIDTHS = list(range(1, 140)) + [255, 256, 257, 383, 500, 1000, 1023, 1025, 1500, 2047, 4100]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("M", [1, 5, 16, 19, 33])
def test_rows_are_quantised_as_by_quantize_mx4(dtype, M):
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
