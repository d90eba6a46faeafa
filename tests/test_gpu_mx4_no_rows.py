"""Each microscaled 4-bit operator with tensors of no rows, in each of its forms."""
import pytest
import torch

import paper_2605_28803_amd as oq

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_forms(dtype):
    z = torch.empty((0, 1088), dtype=dtype, device=DEV)
    codes = [(0, 544), (0, oq.mx4_step_bytes(1088))]
    shapes = lambda pair: [tuple(t.shape) for t in pair]  # noqa: E731
    a = oq.mx4_quantize(z, 64)
    assert shapes(a) == codes and oq.mx4_dequantize(*a).shape == (0, 1088)
    w = oq.mx4_quantize(torch.ones((9, 1088), dtype=dtype, device=DEV))
    assert oq.mx4_linear(*a, *w).shape == (0, 9)
    assert oq.gated_activation(z).shape == (0, 544)
    half = [(0, 272), (0, oq.mx4_step_bytes(544))]
    assert shapes(oq.gated_activation(z, oq.ACT_SILU, mx4=True)) == half
    assert shapes(oq.gated_activation(z, mx4=True, H=oq.mx4_quantize(z[:, :544]))) == half
    row = torch.empty((0,), dtype=torch.int32, device=DEV)
    gate = torch.ones((2, 1088), dtype=dtype, device=DEV)
    for mx4 in (False, True):
        r, h = oq.residual_norm(z, z, oq.Norm("layer"), oq.Norm("rms"), gate=gate, mod_row=row, mx4=mx4)
        assert r.shape == (0, 1088) and (shapes(h) == codes if mx4 else h.shape == (0, 1088))
