"""Microscaled 4-bit codes and their product on the GPU against the plain 64-bit
definitions: codes and steps exactly, products within a bound on their sums."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import mx4_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = [torch.float16, torch.bfloat16]
OUT = {torch.float16: oq.OUT_F16, torch.bfloat16: oq.OUT_BF16, torch.float32: oq.OUT_F32}


def rows(M, K, dtype, seed, ld=None):
    """Rows with channels x 30, blocks of zeros, of tiny and of large numbers."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, K), generator=g, dtype=torch.float64)
    x = torch.where(torch.rand((K,), generator=g) < 0.01, 30 * x, x)
    b = x.view(M, -1, 32)
    pick = torch.rand(b.shape[:2], generator=g)
    b[pick < 0.05] = 0
    b[(pick > 0.05) & (pick < 0.1)] *= 2.0 ** -18 if dtype is torch.float16 else 2.0 ** -126
    b[(pick > 0.1) & (pick < 0.15)] *= 2.0 ** 8 if dtype is torch.float16 else 2.0 ** 100
    x = x.to(dtype)
    wide = torch.full((M, ld or K), float("nan"), dtype=dtype)
    wide[:, :K] = x
    return wide.to(DEV)[:, :K], x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,had,ld", [(1, 32, 1, None), (3, 96, 1, 104), (5, 544, 1, None), (300, 2048, 1, 2056), (1, 32, 32, None),
                                        (7, 96, 32, 96), (5, 192, 64, 200), (3, 128, 128, None), (33, 640, 128, 648), (2, 16384, 64, None),
                                        (2, 65536, 1, None), (129, 2560, 32, None)])
def test_quantize(dtype, M, K, had, ld):
    X, x = rows(M, K, dtype, M + K, ld)
    q = torch.full((M + 1, K // 2), 0xA5, dtype=torch.uint8, device=DEV)
    s = torch.full((M + 1, oq.mx4_step_bytes(K)), 0xA5, dtype=torch.uint8, device=DEV)
    oq.mx4_quantize(X, had, q[:M], s[:M])
    R.check_codes((q[:M], s[:M]), R.rotate(x.double(), had))
    # What is not the call's is left as it was.
    assert bool((q[M] == 0xA5).all()) and bool((s[M] == 0xA5).all()) and bool((s[:M, K // 32:] == 0xA5).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_every_16_bit_number(dtype):
    """Every finite number of the type, in a block whose maximum is near it and
    in one whose maximum is 2^k above it; borders among them."""
    h = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(dtype)
    h = h[torch.isfinite(h)]
    n = h.numel() // 2
    x = torch.cat([h, h.flip(0)])
    x = torch.cat([x, x[: -x.numel() % 32]]).view(-1, 32)
    mixed = h[(torch.arange(64 * 32).view(64, 32) * 7919 + torch.arange(32) * (n // 40)) % h.numel()].view(64, 32)
    for t in (x, mixed):
        R.check_codes(oq.mx4_quantize(t.to(DEV).contiguous()), t.double())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("had", [1, 32, 128])
def test_blocks_that_are_not_finite(dtype, had):
    X, x = rows(4, 256, dtype, 5)
    for r, c, v in ((0, 3, float("inf")), (1, 40, float("nan")), (2, 255, float("-inf")), (2, 254, float("inf"))):
        X[r, c] = x[r, c] = v
    got = oq.mx4_quantize(X, had)
    index, byte = R.unpack(*got)
    # The blocks of 32 of a rotation block with such a value are NaN, the others are theirs.
    bad = ~torch.isfinite(x.double()).view(4, -1, max(had, 32)).all(-1).repeat_interleave(max(had, 32) // 32, 1)
    assert torch.equal(byte == 255, bad)
    clean = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).double()
    wi, wb = R.quantize(R.rotate(clean, had))
    assert torch.equal(byte[~bad], wb[~bad])
    assert torch.equal(index.view(4, -1, 32)[~bad] % 8, wi.view(4, -1, 32)[~bad] % 8)
    assert not bool(index.view(4, -1, 32)[bad].any())
    v = oq.mx4_dequantize(*got).cpu().view(4, -1, 32)
    assert torch.equal(torch.isnan(v).all(-1), bad) and torch.equal(torch.isnan(v).any(-1), bad)


@pytest.mark.parametrize("out", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,ld", [(1, 32, None), (9, 544, 552), (256, 128, None)])
def test_dequantize(out, M, K, ld):
    """Every code with every step."""
    g = torch.Generator().manual_seed(K)
    index = torch.randint(0, 16, (M, K), generator=g)
    byte = (torch.arange(M * (K // 32)).view(M, -1) * (1 if M == 256 else 37)) % 256
    want = R.values(index, byte)
    X = torch.full((M, ld or K), -7.0, dtype=out, device=DEV)
    oq.mx4_dequantize(*R.pack(index, byte, DEV), OUT[out], X[:, :K])
    assert torch.equal(X[:, :K].cpu().nan_to_num(nan=123.0), want.to(torch.float32).to(out).nan_to_num(nan=123.0))
    assert bool((X[:, K:] == -7).all())


def operands(M, N, K, seed, spread=6):
    g = torch.Generator().manual_seed(seed)
    out = []
    for n in (M, N):
        out += [torch.randint(0, 16, (n, K), generator=g), 127 - torch.randint(0, spread + 1, (n, K // 32), generator=g)]
    return out


# One token to several hundred, columns and K off every tile, one block to 2048 of them.
SHAPES = [(1, 1, 32), (1, 16, 64), (1, 2560, 2048), (2, 24, 512), (3, 17, 96), (5, 100, 544), (16, 300, 1024), (17, 33, 4096),
          (33, 128, 480), (50, 1024, 4096), (64, 65, 1056), (65, 64, 2048), (100, 520, 992), (128, 256, 512), (129, 257, 160),
          (200, 1000, 2080), (256, 512, 16384), (257, 129, 32), (300, 2049, 1536), (512, 768, 256), (700, 800, 1024), (8, 72, 65536)]


# Enough rows and columns for the large tiles, alone and with a rest in a launch of its own.
LARGE = [(2100, 8200, 1056), (8000, 2050, 1056), (4100, 2050, 544), (4100, 2050, 4160), (200, 8200, 4160), (4100, 1000, 544),
         (4100, 1000, 4160), (65, 8200, 4160), (65, 8200, 1056), (200, 8200, 96)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("out", [torch.float16, torch.bfloat16, torch.float32])
def test_linear(M, N, K, out):
    xi, xb, wi, wb = operands(M, N, K, M + N + K)
    bias = torch.randn((N,), generator=torch.Generator().manual_seed(N)).half() if N % 2 else None
    want, bound = R.linear(xi, xb, wi, wb, bias)
    ld = (N + 7) // 8 * 8 + 8
    Y = torch.full((M + 1, ld), 77.0, dtype=out, device=DEV)
    oq.mx4_linear(*R.pack(xi, xb, DEV), *R.pack(wi, wb, DEV), None if bias is None else bias.to(DEV), OUT[out], Y[:M, :N])
    R.check(Y[:M, :N], want, bound, out)
    assert bool((Y[M] == 77).all()) and bool((Y[:, N:] == 77).all())
    again = oq.mx4_linear(*R.pack(xi, xb, DEV, fill=0), *R.pack(wi, wb, DEV, fill=200), None if bias is None else bias.to(DEV), OUT[out])
    assert again.shape == (M, N) and torch.equal(again, Y[:M, :N])  # (the steps' unused bytes do not matter)


@pytest.mark.parametrize("M,N,K", LARGE)
def test_linear_large(M, N, K):
    xi, xb, wi, wb = operands(M, N, K, M + N + K)
    bias = torch.randn((N,), generator=torch.Generator().manual_seed(N)).half() if M % 20 else None
    want, bound = R.linear(xi, xb, wi, wb, bias)
    for out in (torch.float16, torch.float32) if M % 20 else (torch.bfloat16,):
        Y = torch.full((M + 1, (N + 7) // 8 * 8 + 8), 77.0, dtype=out, device=DEV)
        oq.mx4_linear(*R.pack(xi, xb, DEV), *R.pack(wi, wb, DEV), None if bias is None else bias.to(DEV), OUT[out], Y[:M, :N])
        R.check(Y[:M, :N], want, bound, out)
        assert bool((Y[M] == 77).all()) and bool((Y[:, N:] == 77).all())


@pytest.mark.parametrize("M,N,K", [(3, 40, 1024), (130, 300, 544), (600, 520, 2048), (4100, 2050, 544), (4100, 2050, 2080)])
def test_linear_where_each_block_goes(M, N, K):
    """Blocks of one operand that are 1 in a single channel: the product reads the
    other operand's channel, whatever block order the kernel has inside."""
    g = torch.Generator().manual_seed(K)
    wi, wb = torch.randint(0, 16, (N, K), generator=g), 127 - torch.randint(0, 40, (N, K // 32), generator=g)
    at = torch.randint(0, K, (M,), generator=g)
    at[0], at[1] = 0, K - 1
    xi = torch.zeros((M, K), dtype=torch.int64)
    xi[torch.arange(M), at] = 2
    xb = 127 + torch.randint(0, 20, (M, K // 32), generator=g)
    Y = oq.mx4_linear(*R.pack(xi, xb, DEV), *R.pack(wi, wb, DEV), out_dtype=oq.OUT_F32)
    want = R.values(wi, wb)[:, at].T * 2.0 ** (xb[torch.arange(M), at // 32].double() - 127)[:, None]
    assert torch.equal(Y.cpu().double(), want)


@pytest.mark.parametrize("M,N,K", [(2, 40, 1024), (70, 300, 544), (600, 520, 2048)])
def test_linear_with_blocks_that_are_not_finite(M, N, K):
    xi, xb, wi, wb = operands(M, N, K, 3)
    xb[M // 2, (K // 32) // 3] = 255
    wb[N - 2, K // 32 - 1] = 255
    Y = oq.mx4_linear(*R.pack(xi, xb, DEV), *R.pack(wi, wb, DEV), out_dtype=oq.OUT_F32).cpu()
    bad = torch.zeros((M, N), dtype=torch.bool)
    bad[M // 2], bad[:, N - 2] = True, True
    assert torch.equal(torch.isnan(Y), bad)
    xb[M // 2, (K // 32) // 3], wb[N - 2, K // 32 - 1] = 127, 127
    want, bound = R.linear(xi, xb, wi, wb)
    R.check(torch.where(bad, want.float(), Y), want, bound, torch.float32)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_linear_extreme_steps(M):
    """Steps from 2^-127 to 2^127 whose products meet in the middle, and zeros."""
    N, K = 48, 1024
    g = torch.Generator().manual_seed(M)
    e = torch.randint(0, 255, (K // 32,), generator=g)
    e[0], e[1] = 0, 254
    xi, wi = torch.randint(0, 16, (M, K), generator=g), torch.randint(0, 16, (N, K), generator=g)
    xb, wb = e.expand(M, -1).clone(), (254 - e).expand(N, -1).clone()
    want, bound = R.linear(xi, xb, wi, wb)
    R.check(oq.mx4_linear(*R.pack(xi, xb, DEV), *R.pack(wi, wb, DEV), out_dtype=oq.OUT_F32), want, bound, torch.float32)
    zero = oq.mx4_linear(*R.pack(0 * xi, 0 * xb, DEV), *R.pack(wi, wb, DEV), out_dtype=oq.OUT_F32)
    assert not bool(zero.any())


def test_quantized_linear():
    """A weight and activations through quantization, rotated alike: near the plain product."""
    M, N, K = 70, 200, 1024
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn((M, K), generator=g).half(), (0.02 * torch.randn((N, K), generator=g)).half()
    for had in (1, 32, 128):
        a, b = oq.mx4_quantize(x.to(DEV), had), oq.mx4_quantize(w.to(DEV), had)
        Y = oq.mx4_linear(*a, *b, out_dtype=oq.OUT_F32)
        want, bound = R.linear(*R.unpack(*a), *R.unpack(*b))
        R.check(Y, want, bound, torch.float32)
        plain = x.double() @ w.double().T
        # 4-bit codes: a relative error of at most 1/4 of each value, independent over 1024 channels and two operands.
        assert (Y.cpu().double() - plain).norm() < 0.25 * plain.norm()


def test_no_rows():
    a = oq.mx4_quantize(torch.empty((0, 64), dtype=torch.float16, device=DEV))
    b = oq.mx4_quantize(torch.ones((8, 64), dtype=torch.float16, device=DEV))
    assert oq.mx4_linear(*a, *b).shape == (0, 8) and oq.mx4_dequantize(*a).shape == (0, 64)
