"""The gated activation where e^-t leaves the range of a float: far negative gates
beside ups that bring act(g) u back, among ordinary channels of one block."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import mx4_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
H, B = torch.float16, torch.bfloat16
ACTS = [oq.ACT_GELU_TANH, oq.ACT_SILU]
F = R.F


def far_gates(act, n, g):
    """Gates whose t lies between about -75 and -210."""
    lo, hi = (-14.0, -9.3) if act == oq.ACT_GELU_TANH else (-210.0, -75.0)
    return lo + (hi - lo) * torch.rand((n,), generator=g)


def signed_powers(shape, lo, hi, g):
    return 2.0 ** (lo + (hi - lo) * torch.rand(shape, generator=g)) * (1 - 2 * torch.randint(0, 2, shape, generator=g))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("at,gate,up", [(0, -100.0, -3e38), (0, -100.0, 3e38), (17, -88.0, 2.0 ** 125), (31, -88.0, -2.0 ** 125),
                                        (5, -10.5, -3e38), (5, -10.5, 3e38), (30, -10.0, -2.0 ** 126), (8, -12.0, -3e38)])
@pytest.mark.parametrize("rest", [1e-6, 1.0, 1e-25])
def test_codes_of_one_far_gate(act, at, gate, up, rest):
    x = torch.cat([torch.full((32,), 1.0), torch.full((32,), rest)])
    x[at], x[32 + at] = gate, up
    x = x.to(B)[None]
    R.check_codes(oq.gated_activation(x.to(DEV), act, mx4=True), R.activation(x, act)[0])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,F_,far", [(1, 32, 1), (700, 96, 1), (300, 544, 5), (64, 4096, 40)])
def test_codes_of_mixed_magnitudes(act, M, F_, far):
    g = torch.Generator().manual_seed(M + far)
    gates, ups = torch.randn((M, F_), generator=g), signed_powers((M, F_), -100, 3, g)
    ups *= 2.0 ** torch.randint(-60, 1, (M, 1), generator=g)
    at = torch.randint(0, F_, (M, far), generator=g)
    gates.scatter_(1, at, far_gates(act, M * far, g).view(M, far))
    ups.scatter_(1, at, signed_powers((M, far), 20, 127.9, g))
    x = torch.cat([gates, ups], 1).to(B)
    R.check_codes(oq.gated_activation(x.to(DEV), act, mx4=True), R.activation(x, act)[0])


@pytest.mark.parametrize("dtype", [H, B])
@pytest.mark.parametrize("act", ACTS)
def test_16_bits(act, dtype):
    """Every finite gate with ups from the smallest to the largest.  t and its product
    with log2 e have at most nine roundings, which move the result by as much as t,
    relative (past |t| = 200 it is u g, or below half the smallest number); the power
    and the reciprocal 2 F each, the sum and three products one each: 10 F with one to
    spare.  A product below 2^-126 is off by 2^-150, times a gate below 2^8."""
    gates = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(dtype)
    gates = gates[torch.isfinite(gates)]
    gates = gates[gates.double().abs() < 1e36]  # (g^3 within a double of the reference)
    gates = gates[: gates.numel() // 8 * 8]
    top = torch.finfo(dtype).max
    ups = [top, -top, 1.0, 3e-4, -1e-7, 0.0] + ([2.0 ** 125, -1e35, 1e30, -1e20, 1e10, 1e-20, -1e-38, 1e-40] if dtype is B else [])
    x = torch.cat([gates.repeat(len(ups), 1), torch.tensor(ups, dtype=dtype)[:, None].expand(-1, gates.numel())], 1)
    want, _ = R.activation(x, act)
    t = x[:, : gates.numel()].double()
    if act == oq.ACT_GELU_TANH:
        t = 1.6 * (t + 0.044715 * t ** 3)
    bound = want.abs() * (9 * F * t.abs().clamp(max=200) + 10 * F) + 2.0 ** -142
    got = oq.gated_activation(x.to(DEV), act).cpu()
    past, within = want.abs() > 1.01 * top, want.abs() < 0.99 * top
    assert bool((got[past].double() == want[past].sign() * float("inf")).all())
    zero = torch.zeros((), dtype=dtype)
    R.check(torch.where(within, got, zero), torch.where(within, want, zero.double()), torch.where(within, bound, zero.double()), dtype)


@pytest.mark.parametrize("act", ACTS)
def test_16_bits_of_far_gates(act):
    """Dense in the range that the tails above only touch; ragged rows."""
    g = torch.Generator().manual_seed(act)
    M, F_ = 203, 1000
    x = torch.cat([far_gates(act, M * F_, g).view(M, F_), signed_powers((M, F_), -30, 127.9, g)], 1).to(B)
    want, _ = R.activation(x, act)
    R.check(oq.gated_activation(x.to(DEV), act), want, want.abs() * ((9 * 215 + 10) * F) + 2.0 ** -142, B)
