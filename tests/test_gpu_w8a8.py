"""W8A8 on the GPU: exact int32 accumulators, the dequantized outputs against
float64, weights in 8 bits, ragged edges, every kernel and tiling."""
import numpy as np
import pytest
import torch

import paper_2605_28803_amd as oq
from oracle import quant
from tests import parity

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")

CASES = [
    (1, 2560, 2048), (1, 64, 64), (16, 2048, 16384), (17, 200, 2048), (50, 3000, 1024), (50, 8192, 1024), (40, 9000, 2048),
    (64, 520, 4160), (3, 100, 64), (65, 320, 1536), (130, 1000, 1024), (256, 4096, 4096), (1000, 2048, 2112), (50, 1024, 4096),
    (700, 4104, 192), (129, 257, 320), (2000, 2056, 704), (300, 8200, 64), (64, 20000, 128), (5, 33000, 1088), (20, 520, 4160),
    (1000, 4096, 320), (3000, 3000, 1024), (4100, 4096, 1024), (4096, 4104, 1024),
    (2, 300, 16384), (30, 4096, 8256), (16, 4104, 4160), (13, 6000, 16384), (1, 5000, 64), (27, 1000, 1088), (9, 5000, 2176),
]


def _codes(g, n, K, extreme=False):
    q = torch.randint(-127, 128, (n, K), generator=g, dtype=torch.int64)
    if extreme:
        q = torch.where(q >= 0, 127, -128)
    return q


def _product(a, b):
    # float64 sums of integer products below 2^53 are exact
    return (a.double() @ b.double().T).to(torch.int64)


@pytest.mark.parametrize("M,N,K", CASES)
def test_accumulators_and_outputs(M, N, K):
    g = torch.Generator().manual_seed(M + 3 * N + 5 * K)
    a, b = _codes(g, M, K), _codes(g, N, K)
    A, B = a.to(torch.int8).to(DEV), b.to(torch.int8).to(DEV)
    want = _product(a, b)
    # (A single row's leading dimension is its width, a multiple of 8 here.)
    ld, ldy = (N + 3) // 4 * 4, (N + 7) // 8 * 8
    acc = torch.full((M, ld), 77, dtype=torch.int32, device=DEV)
    oq.w8a8_gemm_i32(A, B, acc=acc[:, :N])
    torch.cuda.synchronize()
    assert torch.equal(acc[:, :N].cpu().long(), want)
    assert (acc[:, N:] == 77).all()
    xs, ws = torch.rand(M, generator=g) * 0.01 + 1e-3, torch.rand(N, generator=g) * 1e-3 + 1e-4
    bias = torch.randn(N, generator=g).half()
    for out, dt, u in ((oq.OUT_F16, torch.float16, 2.0 ** -11), (oq.OUT_BF16, torch.bfloat16, 2.0 ** -8)):
        for bb in (None, bias):
            full = torch.full((M, ldy), 7.0, dtype=dt, device=DEV)
            Y = full[:, :N]
            oq.w8a8_linear(A, xs.to(DEV), B, ws.to(DEV), None if bb is None else bb.to(DEV), out, Y=Y)
            assert (full[:, N:] == 7.0).all()
            torch.cuda.synchronize()
            y = Y.cpu().double()
            ref = want.double() * xs.double()[:, None] * ws.double()[None, :]
            size = ref.abs()
            if bb is not None:
                ref, size = ref + bb.double(), size + bb.double().abs()
            # the output's rounding, three fp32 roundings of the product, one of the sum
            assert ((y - ref).abs() <= u * ref.abs() + 5 * 2.0 ** -24 * size + 2.0 ** -25).all()


@pytest.mark.parametrize("M,N,K", [(8, 64, 16384), (200, 256, 16384), (64, 64, 16384)])
def test_extreme_codes(M, N, K):
    g = torch.Generator().manual_seed(1)
    a, b = _codes(g, M, K, True), _codes(g, N, K, True)
    a[0], b[0] = -128, -128
    acc = oq.w8a8_gemm_i32(a.to(torch.int8).to(DEV), b.to(torch.int8).to(DEV))
    assert torch.equal(acc.cpu().long(), _product(a, b))
    assert acc[0, 0].item() == 16384 * K


@pytest.mark.parametrize("N,K,b", [(33, 1024, 1024), (7, 1536, 512), (5, 128, 1)])
def test_weights_in_8_bits(N, K, b):
    w = (np.random.default_rng(N).standard_normal((N, K)) * 0.02).astype(np.float16)
    Wq, ws = oq.quantize_weights_i8(torch.from_numpy(w).to(DEV), b)
    torch.cuda.synchronize()
    q_o, ws_o, r_o = quant.rotate_quantize_act(w.astype(np.float64), b, 1.0, quant.QMAX8)
    parity.check_codes(Wq.cpu().numpy().astype(np.int64), q_o, r_o, parity.tau_rows(w, b, 127), qmax=127)
    assert np.allclose(ws.cpu().numpy(), ws_o, rtol=1e-6, atol=0)


def test_whole_linear_is_closer_than_w4a8():
    rng = np.random.default_rng(3)
    M, N, K = 96, 512, 1024
    x = rng.standard_normal((M, K)).astype(np.float16)
    w = (rng.standard_normal((N, K)) * 0.02).astype(np.float16)
    X, W = torch.from_numpy(x).to(DEV), torch.from_numpy(w).to(DEV)
    Xq, xs = oq.rotate_quantize_act_i8(X, K)
    y8 = oq.w8a8_linear(Xq, xs, *oq.quantize_weights_i8(W, K)).double().cpu().numpy()
    y4 = oq.w4a8_linear(Xq, xs, *oq.quantize_weights(W, K)).double().cpu().numpy()
    ref = x.astype(np.float64) @ w.astype(np.float64).T
    e8, e4 = parity.rel_l2(y8, ref), parity.rel_l2(y4, ref)
    # Steps of max / 127 on both sides: each side's error is at most half a step,
    # max / 254, against an rms of about max / 4.
    assert e8 <= 0.02 and e8 < e4 / 4


def test_no_rows():
    W = torch.zeros((64, 64), dtype=torch.int8, device=DEV)
    y = oq.w8a8_linear(torch.zeros((0, 64), dtype=torch.int8, device=DEV), torch.zeros(0, device=DEV), W, torch.ones(64, device=DEV))
    assert y.shape == (0, 64)
