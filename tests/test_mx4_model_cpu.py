"""The 4-bit model without layers, which has no 4-bit weights."""
import ctypes

import pytest
import torch

import paper_2502_01637_amd as S

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: for a process without a GPU")


def at(k):
    return ctypes.c_void_p(k << 36)


def test_no_layers_need_no_weights():
    L = S.scone.lib()
    assert L.scone_fgram_model_mx4_bytes(512, 8, 1024, 0) == 0

    def forward(weights, layers):
        return L.scone_fgram_model_forward_mx4(
            at(1), at(2), at(3), 5, 3, at(8), 100, at(4), weights, 512, 8, 1024, layers, at(6), 90,
            at(7), 1 << 34, None)

    assert forward(at(5), 0) == S.scone.EHIP       # past the checks: no GPU here
    assert forward(None, 0) == S.scone.EHIP
    assert forward(None, 2) == S.scone.EINVAL
