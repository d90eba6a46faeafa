"""Residual norm without r': h and the codes are those of the call that writes it."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests.test_gpu_residual_norm import B, DEV, F32, H, make, norms

pytestmark = pytest.mark.gpu

# Every choice of launch_norm: up to 1024 rows and more, from one wave for four rows to sixteen for one.
SIZES = [(1, 8), (7, 520), (1030, 256), (1030, 1000), (1030, 1536), (900, 2048), (1030, 2560), (40, 4096), (1030, 8192), (30, 8192),
         (1030, 9216), (20, 16384)]
FORMS = [(M, D, mx4) for M, D in SIZES for mx4 in (False, True) if not mx4 or D % 32 == 0]


def same(a, b, mx4, D):
    if not mx4:
        return torch.equal(a, b)
    return torch.equal(a[0], b[0]) and torch.equal(a[1][:, : D // 32], b[1][:, : D // 32])


@pytest.mark.parametrize("rt", [B, F32])
@pytest.mark.parametrize("M,D,mx4", FORMS)
def test_without_the_residual_s_output(M, D, mx4, rt):
    t = make(M, D, B, rt, M + D, 3)
    p, q, _, _ = norms(t, "layer", "rms")
    dev = {n: t[n].to(DEV) for n in ("R", "Y", "gate", "scale", "shift", "row")}
    kw = dict(pre=p, post=q, alpha=0.75, gate=dev["gate"], scale=dev["scale"], shift=dev["shift"], mod_row=dev["row"], mx4=mx4)
    x = dev["R"].clone()
    _, want = oq.residual_norm(dev["R"], dev["Y"], **kw)
    none, got = oq.residual_norm(dev["R"], dev["Y"], R_out=False, **kw)
    assert none is None and same(got, want, mx4, D) and torch.equal(dev["R"], x)
    # A first norm: the residual stays what it is; and a block's output without a residual.
    for r, y in ((dev["R"], None), (None, dev["Y"])):
        _, want = oq.residual_norm(r, y, pre=p, mx4=mx4, dtype=B)
        none, got = oq.residual_norm(r, y, pre=p, mx4=mx4, dtype=B, R_out=False)
        assert none is None and same(got, want, mx4, D)


def test_nothing_to_write_is_refused():
    x = torch.ones((4, 64), dtype=H, device=DEV)
    with pytest.raises(ValueError, match="no output"):
        oq.residual_norm(x, x, R_out=False)
