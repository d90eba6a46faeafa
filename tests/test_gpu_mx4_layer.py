"""A backbone layer in microscaled 4-bit floating point as a program runs it: norm,
q|k|v, attention over packed prompts and then over a 4-bit cache, output projection,
the norms between, the gated MLP, every linear on codes that the step before wrote.
Each step is checked on the GPU's own input; the whole layer captured into a graph
and replayed gives what it gives eagerly, on another stream too."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import mx4_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
D, HQ, HK, HD, F = 256, 4, 1, 64, 640


class Layer:
    """Sandwich norms (before and behind each block), rotated o projection."""

    def __init__(self, dtype, mods):
        g = torch.Generator(device=DEV).manual_seed(11)
        rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.dtype, self.out = dtype, oq.OUT_F16 if dtype is torch.float16 else oq.OUT_BF16
        w = lambda n, k, had=1: oq.mx4_quantize((0.06 * rnd(n, k)).to(dtype), had)  # noqa: E731
        self.qkv, self.o = w((HQ + 2 * HK) * HD, D), w(D, HQ * HD, 64)
        self.gate_up, self.down = w(2 * F, D), w(D, F)
        self.norms = [oq.Norm("rms", (0.1 * rnd(D)).to(dtype), eps=1e-5, gain_offset=1.0) for _ in range(4)]
        self.gate = (1 + 0.1 * rnd(mods, D)).to(dtype)
        self.scale, self.shift = (0.1 * rnd(mods, D)).to(dtype), (0.1 * rnd(mods, D)).to(dtype)

    def __call__(self, x, row, attend, stream=None):
        """x fp32 [T, D], the residual stream; row int32 [T]; attend(q, k, v).  Returns every step."""
        n, s, kw = self.norms, {}, dict(stream=stream)
        _, s["a"] = oq.residual_norm(x, pre=n[0], mx4=True, dtype=self.dtype, **kw)
        s["qkv"] = oq.mx4_linear(*s["a"], *self.qkv, out_dtype=self.out, **kw)
        qkv = s["qkv"].view(-1, HQ + 2 * HK, HD)
        s["att"] = attend(qkv[:, :HQ], qkv[:, HQ:HQ + HK], qkv[:, HQ + HK:])
        s["b"] = oq.mx4_quantize(s["att"].reshape(-1, HQ * HD), 64, **kw)
        s["o"] = oq.mx4_linear(*s["b"], *self.o, out_dtype=self.out, **kw)
        s["r1"], s["c"] = oq.residual_norm(x, s["o"], pre=n[2], post=n[1], gate=self.gate, scale=self.scale, shift=self.shift,
                                           mod_row=row, mx4=True, **kw)
        s["gu"] = oq.mx4_linear(*s["c"], *self.gate_up, out_dtype=self.out, **kw)
        s["d"] = oq.gated_activation(s["gu"], mx4=True, **kw)
        s["y"] = oq.mx4_linear(*s["d"], *self.down, out_dtype=self.out, **kw)
        s["r2"], _ = oq.residual_norm(s["r1"], s["y"], post=n[3], **kw)
        return s

    def check(self, x, row, s):
        cpu = lambda t: t.cpu()  # noqa: E731
        norm = [("rms", cpu(n.gain), None, 1.0, 1e-5) for n in self.norms]
        pick = lambda t: cpu(t)[cpu(row).long()]  # noqa: E731

        def linear(codes, w, y):
            want, bound = R.linear(*R.unpack(*codes), *R.unpack(*w))
            R.check(y, want, bound, self.dtype)

        R.check_codes(s["a"], R.residual_norm(cpu(x), None, norm[0], None, 1.0, None, None, None)[2])
        linear(s["a"], self.qkv, s["qkv"])
        R.check_codes(s["b"], R.rotate(cpu(s["att"]).double().reshape(-1, HQ * HD), 64))
        linear(s["b"], self.o, s["o"])
        wr, er, wh, _ = R.residual_norm(cpu(x), cpu(s["o"]), norm[2], norm[1], 1.0, pick(self.gate), pick(self.scale), pick(self.shift))
        R.check(s["r1"], wr, er, torch.float32)
        R.check_codes(s["c"], wh)
        linear(s["c"], self.gate_up, s["gu"])
        R.check_codes(s["d"], R.activation(cpu(s["gu"]), oq.ACT_GELU_TANH)[0])
        linear(s["d"], self.down, s["y"])
        wr, er, _, _ = R.residual_norm(cpu(s["r1"]), cpu(s["y"]), None, norm[3], 1.0, None, None, None)
        R.check(s["r2"], wr, er, torch.float32)


def flat(s):
    """Every tensor of the steps; of codes and steps, the bytes in use."""
    return [t for v in s.values() for t in ((v[0], v[1][:, :v[0].shape[1] // 16]) if isinstance(v, tuple) else (v,))]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_prompt_then_decode(dtype):
    g = torch.Generator(device=DEV).manual_seed(2)
    lens, page = [70, 1, 33], 32
    n, T = len(lens), sum(lens)
    layer = Layer(dtype, n)
    cu = torch.tensor([0, 70, 71, 104], dtype=torch.int32, device=DEV)
    seq = torch.arange(n, device=DEV).repeat_interleave(torch.tensor(lens, device=DEV))
    cache = oq.KV4Cache.empty(4 * n, HK, HD, page)
    table = torch.randperm(4 * n, device=DEV, generator=g).to(torch.int32).view(n, 4)
    pos = torch.arange(T, device=DEV) - cu[:-1].long()[seq]

    def prompt(q, k, v):
        oq.kv4_append(cache, k, v, table[seq, pos // page].long() * page + pos % page)
        return oq.attention_prompt(q, k, v, cu)

    x = torch.randn((T, D), generator=g, device=DEV) * 3
    row = seq.to(torch.int32)
    layer.check(x, row, layer(x, row, prompt))
    length = torch.tensor(lens, device=DEV)
    one = torch.arange(n, device=DEV)
    for _ in range(2):
        x = torch.randn((n, D), generator=g, device=DEV) * 3

        def decode(q, k, v):
            oq.kv4_append(cache, k, v, table[one, length // page].long() * page + length % page)
            return oq.attention_kv4(q, cache, table, (length + 1).to(torch.int32), max_len=128)

        layer.check(x, one.to(torch.int32), layer(x, one.to(torch.int32), decode))
        length = length + 1


@pytest.mark.parametrize("T", [1, 90])
def test_captured_and_on_another_stream(T):
    """Replays with new inputs between them, the eager layer's results among them; and
    two graphs of one layer, replayed in turn."""
    layer = Layer(torch.bfloat16, 2)
    g = torch.Generator(device=DEV).manual_seed(T)
    x, row = torch.empty((T, D), device=DEV), torch.arange(T, dtype=torch.int32, device=DEV) % 2
    cu = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    attend = lambda q, k, v: oq.attention_prompt(q, k, v, cu)  # noqa: E731
    x.normal_(generator=g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(x, row, attend)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append([graph, None])
            graphs[-1][1] = layer(x, row, attend)
    for turn in range(4):
        x.normal_(generator=g)
        want = [t.clone() for t in flat(layer(x, row, attend))]
        for graph, s in graphs if turn % 2 else graphs[::-1]:
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(flat(s), want))
    # On a stream of its own, while the current one is busy.
    torch.mm(torch.zeros((4096, 4096), device=DEV), torch.zeros((4096, 4096), device=DEV))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s = layer(x, row, attend)
    other = layer(x, row, lambda q, k, v: oq.attention_prompt(q, k, v, cu, stream=side), stream=side)
    torch.cuda.synchronize()
    assert torch.equal(s["r2"], want[-1]) and torch.equal(other["r2"], want[-1])


def _calls():
    g = torch.Generator(device=DEV).manual_seed(4)
    x, w = (torch.randn((n, 1024), generator=g, device=DEV).half() for n in (96, 320))
    (xq, xs), (wq, ws) = oq.mx4_quantize(x), oq.mx4_quantize(w)
    norm = oq.Norm("layer")
    torch.cuda.synchronize()
    return {
        "mx4_quantize": lambda s: oq.mx4_quantize(x, 64, stream=s),
        "mx4_dequantize": lambda s: oq.mx4_dequantize(xq, xs, oq.OUT_F32, stream=s),
        "mx4_linear": lambda s: oq.mx4_linear(xq, xs, wq, ws, stream=s),
        "mx4_linear, split": lambda s: oq.mx4_linear(xq[:1], xs[:1], wq, ws, out_dtype=oq.OUT_F32, stream=s),
        "gated_activation": lambda s: oq.gated_activation(x, stream=s),
        "gated_activation, codes": lambda s: oq.gated_activation(x, mx4=True, stream=s),
        "residual_norm": lambda s: oq.residual_norm(x, x, pre=norm, stream=s),
        "residual_norm, codes": lambda s: oq.residual_norm(x, x, pre=norm, mx4=True, stream=s),
    }


def _list(out):
    return [out] if torch.is_tensor(out) else [t for t in out for t in (t if isinstance(t, tuple) else (t,))]


def test_outputs_belong_to_the_call_s_stream():
    """Blocks just freed on the current stream are not what a call on another one
    writes, and what it made does not come back on the current one; values as ever."""
    s = torch.cuda.Stream()
    for name, call in _calls().items():
        want = _list(call(None))
        torch.cuda.synchronize()
        freed = [torch.empty_like(t) for t in want]
        at = {t.data_ptr() for t in freed}
        del freed
        got = _list(call(s))
        torch.cuda.synchronize()
        # (1024 channels: every step's byte is in use.)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
        assert not at & {t.data_ptr() for t in got}, name
        like, at = [(t.shape, t.dtype) for t in got], {t.data_ptr() for t in got}
        del got
        again = [torch.empty(n, dtype=dt, device=DEV) for n, dt in like for _ in range(4)]
        assert not at & {t.data_ptr() for t in again}, name
        del again


def test_a_stream_of_another_device_is_refused():
    import types
    other = types.SimpleNamespace(device_index=1, cuda_stream=0, device=torch.device("cuda", 1))
    x = torch.ones((4, 64), dtype=torch.float16, device=DEV)
    q = (torch.empty((4, 32), dtype=torch.uint8, device=DEV), torch.empty((4, 16), dtype=torch.uint8, device=DEV))
    for call in (lambda: oq.mx4_quantize(x, 1, *q, stream=other), lambda: oq.mx4_dequantize(*q, X=x, out_dtype=oq.OUT_F16, stream=other),
                 lambda: oq.mx4_linear(*q, *q, Y=x[:, :4], stream=other),
                 lambda: oq.gated_activation(x, H=x[:, :32], stream=other),
                 lambda: oq.residual_norm(x, x, pre=oq.Norm("rms"), R_out=x, H=x, stream=other)):
        with pytest.raises(ValueError, match="not on cuda:0"):
            call()


def test_norm_keeps_its_parameters():
    """A norm's values are its tensors' memory: written in place they are seen; another
    tensor in their place is not taken up, and the memory stays."""
    x = torch.ones((2, 64), dtype=torch.float16, device=DEV)
    gain = torch.nn.Parameter(torch.full((64,), 2.0, dtype=torch.float16, device=DEV))
    norm = oq.Norm("rms", gain)  # (eps 1e-6: 3 (1 - 5e-7) is 3 in fp16)
    with torch.no_grad():
        gain.fill_(3.0)
    gain.data = torch.zeros_like(gain)
    fill = torch.zeros((64,), dtype=torch.float16, device=DEV)
    _, h = oq.residual_norm(x, pre=norm, dtype=torch.float16)
    assert bool((h == 3).all()) and bool((fill == 0).all())
    with pytest.raises(AttributeError):
        norm.gain = fill
