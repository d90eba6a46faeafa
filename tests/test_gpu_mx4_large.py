"""Calls whose rows do not fit one launch, or whose offsets do not fit 32 bits: the last
rows are those of a call on them alone, and so are those on either side of a border."""
import pytest
import torch

import paper_2605_28803_amd as oq

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def fill(shape, dtype):
    x = torch.empty(shape, dtype=dtype, device=DEV)
    return x.normal_(generator=torch.Generator(device=DEV).manual_seed(shape[0]))


def same(got, want):
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_residual_norm_rows():
    M, D = (1 << 21) + 5, 32
    Y, R = fill((M, D), torch.bfloat16), fill((M, D), torch.float32)
    gate = fill((3, D), torch.bfloat16)
    row = (torch.arange(M, device=DEV) % 4).to(torch.int32)  # (3: left as it was)
    pre = oq.Norm("rms")
    for mx4 in (False, True):
        r, h = oq.residual_norm(R, Y, pre=pre, gate=gate, mod_row=row, mx4=mx4, R_out=R.clone())
        used = [h[0], h[1][:, :1]] if mx4 else [h]
        for a, b in ((0, 40), (M - 40, M)):
            keep = row[a:b] < 3
            r2, h2 = oq.residual_norm(R[a:b], Y[a:b], pre=pre, gate=gate, mod_row=row[a:b], mx4=mx4, R_out=R[a:b].clone())
            same([r[a:b]], [r2])
            same([t[a:b][keep] for t in used], [t[keep] for t in ([h2[0], h2[1][:, :1]] if mx4 else [h2])])


@pytest.mark.parametrize("had", [1, 64])
def test_codes_of_many_rows(had):
    M, K = (1 << 17) + 3, 65536  # 17 GB; without rotation two launches
    X = fill((M, K), torch.bfloat16)
    q, s = oq.mx4_quantize(X, had)
    v = oq.mx4_dequantize(q, s, X=X)  # (in X's place, whose rows are no longer needed but the last)
    for a, b in ((0, 2), (65535, 65537), (131070, M)):
        x = fill((M, K), torch.bfloat16)[a:b].clone()
        q2, s2 = oq.mx4_quantize(x, had)
        same([q[a:b], s[a:b], v[a:b]], [q2, s2, oq.mx4_dequantize(q2, s2)])
    h = oq.gated_activation(X[:, : K // 2 * 2], mx4=True)
    for a, b in ((0, 2), (131070, M)):
        same([t[a:b] for t in h], oq.gated_activation(X[a:b].contiguous(), mx4=True))


def test_linear_past_32_bits():
    M, N, K = 70000, 65536, 32
    g = torch.Generator(device=DEV).manual_seed(1)
    q = lambda n: (torch.randint(0, 256, (n, K // 2), generator=g, device=DEV, dtype=torch.uint8),  # noqa: E731
                   torch.randint(120, 134, (n, 16), generator=g, device=DEV, dtype=torch.uint8))
    x, w = q(M), q(N)
    y = oq.mx4_linear(*x, *w)
    for a, b in ((0, 300), (32700, 32800), (65500, 65600), (M - 300, M)):
        same([y[a:b]], [oq.mx4_linear(x[0][a:b], x[1][a:b], *w)])
