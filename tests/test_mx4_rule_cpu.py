"""The scratch that the 4-bit linear map asks for goes by what its launch takes."""
import ctypes

import pytest
import torch

import paper_2502_01637_amd as S

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: for a process without a GPU")

BF16, F16, F32, MX4 = S.scone.BF16, S.scone.FP16, S.scone.FP32, S.scone.MX4


def at(k):
    return ctypes.c_void_p(k << 40)


@pytest.mark.parametrize("t", [BF16, F16, F32, MX4])
def test_scratch_is_asked_for_where_it_is_needed(t):
    """Without scratch a call is refused where the size is not 0, and gets past the checks
    (to a device that is not there) where it is."""
    lib = S.scone.lib()
    for M in (1, 8, 9, 16, 17, 32, 33, 64, 65, 1000):
        for N, K in ((1, 1), (512, 512), (4096, 1024), (1024, 4096), (16384, 4096), (65536, 128)):
            need = lib.scone_linear_mx4_workspace(M, N, K, t)
            rc = [lib.scone_linear_mx4(at(1), t, K, M, K, at(2), N, None, 0, 0, None, at(3), BF16,
                                       N, ws, size, None)
                  for ws, size in ((None, 0), (at(4), need))]
            assert rc == [S.scone.EINVAL if need else S.scone.EHIP, S.scone.EHIP], (M, N, K)


def test_rows_count_by_what_their_quantisation_costs():
    """Rows that are in 4 bits already, that nothing has to quantise again, take the form
    without scratch for longer than those of 16 bits, and these for longer than fp32."""
    def size(M, N, K, t):
        return S.scone.lib().scone_linear_mx4_workspace(M, N, K, t)

    assert size(64, 4096, 4096, MX4) == 0 < size(64, 4096, 4096, BF16)
    assert size(32, 16384, 4096, MX4) == 0 < size(32, 16384, 4096, F16)
    assert size(64, 4096, 1024, BF16) == 0 < size(64, 4096, 1024, F32)
    assert size(16, 16384, 4096, BF16) == 0 < size(16, 16384, 4096, F32)
