"""The microscaled 4-bit product's ring kernel, its calls of two launches and a layer
that takes them, captured into graphs and on streams of their own.  (Which kernel a
shape takes is checked on the host, in test_mx4_forms.py.)"""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import mx4_ref as R
from tests.test_gpu_mx4_layer import D, Layer, flat

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")

# (M, N, K): every tiling of the ring, and whole rounds of large tiles with the rest beside or below.
RING = {0: (2000, 8190, 1056), 1: (1000, 4090, 4096), 2: (2000, 2060, 1024), 3: (300, 2049, 1536), 4: (400, 4096, 4096)}
SPLIT = {"columns": (2000, 8200, 1056), "rows": (2100, 8200, 1056)}
CASES = list(RING.values()) + list(SPLIT.values())
LAYER_ROWS = 700


def operands(M, N, K, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [t for n in (M, N) for t in (torch.randint(0, 256, (n, K // 2), generator=g, device=DEV, dtype=torch.uint8),
                                        torch.randint(120, 128, (n, oq.mx4_step_bytes(K)), generator=g, device=DEV, dtype=torch.uint8))]


def plain(x, xs, w, ws):
    """In 64 bits on the GPU: (product, sum of the products' magnitudes)."""
    def values(q, s):
        v = R.GRID.to(DEV)[torch.stack((q & 7, (q >> 4) & 7), -1).flatten(1).long()]
        v = torch.where((torch.stack((q, q >> 4), -1).flatten(1) & 8) > 0, -v, v)
        return v * (2.0 ** (s[:, : v.shape[1] // 32].double() - 127)).repeat_interleave(32, 1)
    a, b = values(x, xs), values(w, ws)
    return torch.mm(a, b.T.contiguous()), torch.mm(a.abs(), b.abs().T.contiguous())


@pytest.mark.parametrize("M,N,K", CASES)
@pytest.mark.parametrize("out", [oq.OUT_F32, oq.OUT_BF16])
def test_product_captured(M, N, K, out):
    """Two graphs of one product, replayed in turn with new operands between them and the
    eager product among the replays; the first against the 64-bit one."""
    x, xs, w, ws = operands(M, N, K, 1)
    call = lambda: oq.mx4_linear(x, xs, w, ws, out_dtype=out)  # noqa: E731
    first = call()
    want, mag = plain(x, xs, w, ws)
    # As the reference's bound: an instruction's sum within 2^-23 of the magnitudes, one behind the other.
    tol = (K / 64 + 17) * 2 * R.F * mag
    tol = tol + R.U[first.dtype] * (want.abs() + tol)
    assert bool(((first.double() - want).abs() <= tol).all())
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = call()
        graphs.append((graph, y))
    for turn in range(4):
        for t, u in zip((x, xs, w, ws), operands(M, N, K, 2 + turn)):
            t.copy_(u)
        eager = call()
        for graph, y in graphs if turn % 2 else graphs[::-1]:
            y.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, eager)


@pytest.mark.parametrize("M,N,K", CASES)
def test_product_on_another_stream(M, N, K):
    """On a stream of its own while the current one is busy: the values of a call on the
    current one, in memory that is not shared with it."""
    x, xs, w, ws = operands(M, N, K, 9)
    want = oq.mx4_linear(x, xs, w, ws)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = torch.empty_like(want)
    at = freed.data_ptr()
    del freed
    busy = torch.zeros((4096, 4096), device=DEV)
    torch.mm(busy, busy)
    got = oq.mx4_linear(x, xs, w, ws, stream=side)
    with torch.cuda.stream(side):
        again = oq.mx4_linear(x, xs, w, ws)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(again, want) and at not in (got.data_ptr(), again.data_ptr())


def test_two_streams_at_once():
    """Products of different shapes under way together, several times over."""
    sets = [operands(M, N, K, 20 + i) for i, (M, N, K) in enumerate(CASES)]
    want = [oq.mx4_linear(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[oq.mx4_linear(*s, stream=streams[(turn + i) % 2]) for i, s in enumerate(sets)] for turn in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for turn in got for a, b in zip(turn, want))


def test_layer_of_many_rows_captured():
    """A layer whose products take the ring."""
    T = LAYER_ROWS
    layer = Layer(torch.bfloat16, 2)
    g = torch.Generator(device=DEV).manual_seed(T)
    x, row = torch.empty((T, D), device=DEV), torch.arange(T, dtype=torch.int32, device=DEV) % 2
    cu = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    attend = lambda q, k, v: oq.attention_prompt(q, k, v, cu)  # noqa: E731
    x.normal_(generator=g)
    layer.check(x, row, layer(x, row, attend))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(x, row, attend)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s = layer(x, row, attend)
        graphs.append((graph, s))
    for turn in range(4):
        x.normal_(generator=g)
        want = [t.clone() for t in flat(layer(x, row, attend))]
        for graph, s in graphs if turn % 2 else graphs[::-1]:
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(flat(s), want))
