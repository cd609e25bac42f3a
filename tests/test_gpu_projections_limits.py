"""Sizes that experts refuse, as the header states them: before anything is launched, so the pointers are good for far less."""
import pytest
import torch

from test_gpu_projections import _layers, snn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count,c_out,rows", [
    (16, 32, 1 << 30),             # (2^27 + 1) * 16
    (1000, 8, 8 * 2147483),        # 2147484 * 1000, the first above
    (3, 512, (1 << 30) - 24),      # (2^27 - 3 + 3) * 16
    (1, 1024, (1 << 29) - 8),      # (2^26 - 1 + 1) * 32
    (1, 8, (1 << 30) + 1),
])
def test_refused(snn, count, c_out, rows):  # noqa: F811
    assert rows > 1 << 30 or (rows // 8 + 1) * count >= 1 << 31 or (rows // 8 + count) * -(-c_out // 32) >= 1 << 31
    layers, _, _ = _layers(snn, 1, 8, c_out, 3, 2600)
    ex = snn.SnnConvExperts(layers * count)   # (the same layer may be several experts)
    p = torch.zeros(4096, device="cuda").data_ptr()
    before, lib = snn.kernel_launches(), snn.load_library()
    st = lib.snn_conv_experts_forward(ex._h, p, snn.ACT_F16, 16, 8, None, p, rows, p, snn.OUT_F32, c_out, None)
    assert st == 2 and b"split the call" in lib.snn_last_error() and snn.kernel_launches() == before
