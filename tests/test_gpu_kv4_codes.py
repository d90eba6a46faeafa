"""Codes of rotated rows whose quotients lie on a half integer but for elements
2^33 times smaller: decided exactly, against integer arithmetic."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import serving_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _exact(x, d):
    """Codes of rows x (integers, a list of rows) rotated by H_d, in integers."""
    H = R.hadamard(d).long().tolist()
    out = []
    for row in x:
        there = [i for i, a in enumerate(row) if a]
        u = [sum(row[i] * h[i] for i in there) for h in H]
        top = max(abs(a) for a in u)
        codes = []
        for a in u:
            q, r = divmod(7 * abs(a), top)
            q += 2 * r > top or (2 * r == top and q % 2)
            codes.append(q if a >= 0 else -q)
        out.append(codes)
    return torch.tensor(out)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,below", [(torch.float16, 12), (torch.bfloat16, 12), (torch.bfloat16, 28)])
def test_small_elements_decide_ties(dtype, below, d):
    """19 and 9 give quotients of 7 (19 - 9) / (19 + 9) = 5 / 2 in half of the
    channels, 13 and 15 of 1 / 2; elements of 2^-below make them more or less, or leave them."""
    rows = []
    for p, r in ((19, 9), (13, 15), (-9, 19)):
        for small in ((0, 0), (1, 0), (-1, 0), (1, 1), (1, -1), (3, -2)):
            x = [0] * d
            x[0], x[d // 2 + 1] = p << below, r << below
            x[2], x[d - 1] = small
            rows.append(x)
    k = (torch.tensor(rows).double() * 2.0 ** -below).to(dtype)
    assert torch.equal(k.double() * 2.0 ** below, torch.tensor(rows).double())
    n = len(rows)
    cache = oq.KV4Cache.empty(1, 1, d, 32, rotate_k=True)
    oq.kv4_append(cache, k[:, None].to(DEV), torch.zeros((n, 1, d), dtype=dtype, device=DEV), torch.arange(n, device=DEV))
    got = R.unpack(cache.k_codes.cpu()[0, 0, :n]).long()
    assert torch.equal(got, _exact(rows, d))
