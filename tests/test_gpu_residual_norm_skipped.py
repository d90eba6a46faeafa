"""Each form of the residual norm (waves of a row, pieces of a thread) with skipped rows
among others."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import mx4_ref as R
from tests.test_gpu_residual_norm import DEV, F32, H, make, norms, pick
from tests.test_gpu_residual_norm_only_h import FORMS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rt", [H, F32])
@pytest.mark.parametrize("M,D,mx4", FORMS)
def test_skipped_rows_in_each_form(M, D, mx4, rt):
    """Runs of one, two and three skipped rows, so that the four rows of a workgroup (up to
    512 channels) are skipped and kept in every mixture, and neighbours are where a row has
    its own."""
    t = make(M, D, H, rt, M + D, 3)
    p, q, rp, rq = norms(t, "layer", "layer")
    skip = torch.isin(torch.arange(M) % 13, torch.tensor([1, 4, 5, 9, 10, 11]))
    t["row"] = torch.where(skip, torch.tensor([-1, 3, 2 ** 31 - 1, -2 ** 31])[torch.arange(M) % 4], t["row"]).to(torch.int32)
    out = torch.full((M, D), 5.0, dtype=rt, device=DEV)
    h = (torch.full((M, D // 2), 0xA5, dtype=torch.uint8, device=DEV), torch.full((M, oq.mx4_step_bytes(D)), 0xA5, dtype=torch.uint8, device=DEV)) \
        if mx4 else torch.full((M, D), 6.0, dtype=H, device=DEV)
    oq.residual_norm(t["R"].to(DEV), t["Y"].to(DEV), p, q, 1.5, t["gate"].to(DEV), t["scale"].to(DEV), t["shift"].to(DEV), t["row"].to(DEV),
                     mx4, out, h)
    keep = ~skip
    assert bool((out.cpu()[skip] == 5).all())
    for x, v in zip(h if mx4 else [h], (0xA5, 0xA5) if mx4 else (6,)):
        assert bool((x.cpu()[skip] == v).all())
    for n in ("R", "Y", "row"):
        t[n] = t[n][keep]
    wr, er, wh, eh = R.residual_norm(t["R"], t["Y"], rp, rq, 1.5, pick(t, "gate"), pick(t, "scale"), pick(t, "shift"))
    R.check(out.cpu()[keep], wr, er, rt)
    if mx4:
        R.check_codes([c.cpu()[keep] for c in h], wh)
    else:
        R.check(h.cpu()[keep], wh, eh, H)
