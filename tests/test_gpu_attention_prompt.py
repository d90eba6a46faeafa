"""Attention over packed prompts against float64: lengths from one token, odd
and empty sequences, grouped heads, strides, both types, unused rows."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import serving_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _run(lens, hq, hk, d, causal, dtype, lead=0, tail=0, scale=None, packed=True, seed=0, spike=0.0):
    T = lead + sum(lens) + tail
    g = torch.Generator().manual_seed(seed + 7 * T + d)
    qkv = torch.randn((max(T, 1), hq + 2 * hk, d), generator=g).to(dtype)[:T]
    if spike:
        qkv[:, :, 0] *= spike
    cu = torch.tensor([lead] + [lead + sum(lens[:i + 1]) for i in range(len(lens))], dtype=torch.int32)
    x = qkv.to(DEV)
    # Rows of no sequence hold NaN: they may not be used.
    x[:lead] = float("nan")
    x[T - tail:] = float("nan") if tail else x[T - tail:]
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    O = torch.full((T, hq, d), 3.0, dtype=dtype, device=DEV)
    r = oq.attention_prompt(q, k, v, cu.to(DEV), causal=causal, scale=scale, O=O)
    assert r is O
    torch.cuda.synchronize()
    got = O.cpu()
    assert (got[:lead] == 3.0).all() and (got[T - tail:] == 3.0).all() or not (lead or tail)
    s = d ** -0.5 if scale is None else scale
    at = lead
    for n in lens:
        rows = slice(at, at + n)
        at += n
        see = torch.ones((n, n), dtype=torch.bool)
        see = see.tril() if causal else see
        for h in range(hq):
            qq, kk, vv = (qkv[rows, i].double() for i in (h, hq + h // (hq // hk), hq + hk + h // (hq // hk)))
            o, spread, _ = R.attend(qq, kk, vv, s, see)
            R.check(got[rows, h], o, spread, 2 * R.score_error(qq, kk, s), dtype, R.U[dtype])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged(d, causal, dtype):
    _run([1, 31, 0, 130, 64, 257, 2], 4, 2, d, causal, dtype, lead=3, tail=5)


@pytest.mark.parametrize("hq,hk", [(1, 1), (8, 1), (5, 5), (15, 3)])
def test_heads(hq, hk):
    _run([100, 33], hq, hk, 128, True, torch.bfloat16)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 300, 816, 1025])
def test_one_sequence(n):
    _run([n], 2, 1, 128, True, torch.float16, packed=False)
    _run([n], 2, 1, 256, False, torch.bfloat16)
    _run([n], 2, 1, 64, True, torch.bfloat16)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_workgroup_shapes(d, causal):
    """Every shape of workgroup over several steps: few and many heads, one long
    sequence and several."""
    _run([500], 4, 1, d, causal, torch.float16)             # key groups
    _run([700], 44, 2, d, causal, torch.bfloat16)           # one group, many steps (d = 64: two)
    _run([700], 100, 4, d, causal, torch.float16)           # more heads
    _run([200, 170], 4, 2, d, causal, torch.bfloat16)       # few short rows
    _run([300, 290, 310], 12, 3, d, causal, torch.float16)
    if causal:
        _run([2100], 20, 1, d, causal, torch.float16)       # few long rows



def test_many_sequences():
    _run([(7 * i) % 40 for i in range(150)], 2, 2, 64, True, torch.float16, tail=70)


def test_large_scores():
    # One channel dominates: nearly one-hot rows, maxima that grow along the row.
    _run([200], 2, 2, 64, False, torch.bfloat16, spike=30.0)
    _run([200], 2, 2, 64, True, torch.float16, spike=12.0, scale=0.5)


@pytest.mark.parametrize("below", [10.0, 13.0, 15.0])
def test_many_small_probabilities(below):
    """One key far above the others, whose probabilities are below fp16's normal
    numbers but of weight together; in all channels but one they alone are the output."""
    n, d = 4096, 64
    q, k, v = (torch.zeros((n, 1, d), dtype=torch.float16) for _ in range(3))
    q[:, 0, 0], k[5, 0, 0] = 1.0, 8.0
    v[:], v[5], v[5, 0, 0] = 1.0, 0.0, 1.0
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    o = oq.attention_prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu, causal=False, scale=below / 8)
    row = slice(0, 1)  # (every row is the same)
    ref, spread, _ = R.attend(q[row, 0].double(), k[:, 0].double(), v[:, 0].double(), below / 8, torch.ones((1, n), dtype=torch.bool))
    got = o.cpu()[:, 0]
    R.check(got, ref.expand(n, d), spread.expand(n, d), 2.0 ** -16, torch.float16, 2.0 ** -11)


def test_equal_to_itself_and_on_another_stream():
    qkv = torch.randn((500, 8, 128), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).half()
    cu = torch.tensor([0, 200, 500], dtype=torch.int32, device=DEV)
    a = oq.attention_prompt(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], cu)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = oq.attention_prompt(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], cu, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_captured():
    qkv = torch.randn((300, 6, 64), device=DEV).to(torch.bfloat16)
    cu = torch.tensor([0, 300], dtype=torch.int32, device=DEV)
    O = torch.empty((300, 4, 64), dtype=torch.bfloat16, device=DEV)
    oq.attention_prompt(qkv[:, :4], qkv[:, 4:5], qkv[:, 5:], cu, O=O)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        oq.attention_prompt(qkv[:, :4], qkv[:, 4:5], qkv[:, 5:], cu, O=O)
    for i in range(3):
        qkv.copy_(torch.randn((300, 6, 64), device=DEV, generator=torch.Generator(device=DEV).manual_seed(i)))
        cu.copy_(torch.tensor([0, 300 - 50 * i], dtype=torch.int32))
        want = oq.attention_prompt(qkv[:, :4], qkv[:, 4:5], qkv[:, 5:], cu)
        g.replay()
        torch.cuda.synchronize()
        n = 300 - 50 * i
        assert torch.equal(O[:n], want[:n])


def test_sequence_bounds_are_clamped():
    # Bounds outside the rows, and a decreasing pair, read and write nothing outside.
    qkv = torch.randn((100, 3, 64), device=DEV).half()
    O = torch.full((100, 1, 64), 3.0, dtype=torch.float16, device=DEV)
    cu = torch.tensor([-5, 40, 30, 1000], dtype=torch.int32, device=DEV)
    oq.attention_prompt(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], cu, O=O)
    torch.cuda.synchronize()
    assert torch.isfinite(O).all()
