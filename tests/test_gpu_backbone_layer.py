"""The serving operators as a backbone uses them together: a layer's q|k|v
linear in 8 bits over packed prompts, attention within the prompts, their keys
and values into the cache, then decoding steps over it; and the DiT head's
prefix read back from such a cache."""
import math

import numpy as np
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import serving_ref as R
from workloads import configs, dit_inputs

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.mark.parametrize("hq,hk,d,D", [(8, 1, 256, 2048), (8, 4, 64, 512)])
def test_prompt_then_decode(hq, hk, d, D):
    g = torch.Generator(device=DEV).manual_seed(hk)
    lens, page, steps = [70, 1, 130], 32, 3
    T, n = sum(lens), len(lens)
    w = torch.randn((hq * d + 2 * hk * d, D), device=DEV, generator=g).half() * 0.05
    W, ws = oq.quantize_weights_i8(w, D)
    wd = oq.w8a8_gemm_i32(W, torch.eye(D, device=DEV).to(torch.int8)).double() * ws.double()[:, None]  # its values

    def linear(x):
        Xq, xs = oq.rotate_quantize_act_i8(x, D)
        qkv = oq.w8a8_linear(Xq, xs, W, ws)
        ref = (Xq.double() * xs.double()[:, None]) @ wd.t()
        assert (qkv.double() - ref).norm() <= 2.0 ** -11 * ref.norm()
        return qkv.view(-1, hq + 2 * hk, d)

    cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=DEV)
    qkv = linear(torch.randn((T, D), device=DEV, generator=g).half())
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    o = oq.attention_prompt(q, k, v, cu)
    # Cache: pages dealt out in any order, room for the steps.
    wide = -(-(max(lens) + steps) // page)
    table = torch.randperm(n * wide, device=DEV, generator=g).to(torch.int32).view(n, wide)
    cache = oq.KV4Cache.empty(n * wide, hk, d, page, rotate_k=True)

    def slots_of(seq, pos):
        return table[seq, pos // page].long() * page + pos % page

    seq = torch.arange(n, device=DEV).repeat_interleave(torch.tensor(lens, device=DEV))
    pos = torch.arange(T, device=DEV) - cu[:-1].long()[seq]
    oq.kv4_append(cache, k, v, slots_of(seq, pos))
    for s in range(n):
        a, b = int(cu[s]), int(cu[s + 1])
        see = torch.ones((b - a, b - a), dtype=torch.bool).tril()
        for h in range(hq):
            x = [t[a:b, i].double().cpu() for t, i in ((q, h), (k, h // (hq // hk)), (v, h // (hq // hk)))]
            want, spread, _ = R.attend(*x, d ** -0.5, see)
            R.check(o[a:b, h].cpu(), want, spread, 2 * R.score_error(x[0], x[1], d ** -0.5), torch.float16, 2.0 ** -11)
    length = torch.tensor(lens, device=DEV)
    one = torch.arange(n, device=DEV)
    for _ in range(steps):
        qkv = linear(torch.randn((n, D), device=DEV, generator=g).half())
        oq.kv4_append(cache, qkv[:, hq:hq + hk], qkv[:, hq + hk:], slots_of(one, length))
        length = length + 1
        o = oq.attention_kv4(qkv[:, :hq], cache, table, length.to(torch.int32))
        for s in range(n):
            L = int(length[s])
            kk, vv = oq.kv4_gather(cache, slots_of(torch.full((L,), s, device=DEV), torch.arange(L, device=DEV)), oq.OUT_F32)
            for h in range(hq):
                x = [t.double().cpu() for t in (qkv[s:s + 1, h], kk[:, h // (hq // hk)], vv[:, h // (hq // hk)])]
                want, spread, p = R.attend(*x, d ** -0.5, torch.ones((1, L), dtype=torch.bool))
                # Keys and queries are used rotated: 72 sum(q) in steps, 22 bits and log2 d sums (Cauchy-Schwarz).
                one_ = math.sqrt(d) * x[0].norm().item() * d ** -0.5
                step = x[1].norm(dim=-1).max().item() / math.sqrt(d) * 4 / 7
                extra = 2 * R.score_error(x[0], x[1], d ** -0.5) + 2 * one_ * step * (80 * (d + 8) * 2.0 ** -24 + 7 * 12 * 2.0 ** -22)
                spread = spread + L * 7 * 2.0 ** -16 * (p[:, :, None] * x[2].abs()[None]).amax((1, 2))[:, None]
                R.check(o[s:s + 1, h].cpu(), want, spread, extra, torch.float16, 2.0 ** -11)


def test_dit_prefix_from_a_cache():
    """A DiT step on a prefix read from a 4-bit cache is the step on those values."""
    cfg = configs.DIT_PI
    inp = dit_inputs.make_dit_inputs(cfg, n_blocks=2)
    P, H, hd = cfg.prefix, cfg.n_heads, cfg.head_dim
    model = oq.DiT(cfg, inp, device="cuda:0")
    x0 = torch.from_numpy(inp["x0"].astype(np.float32)).to(DEV)
    plain = model.step(x0.clone(), 0)
    cache = oq.KV4Cache.empty(2 * -(-P // 64), H, hd, 64, rotate_k=True)
    values = []
    for l in range(2):
        slots = torch.arange(P, device=DEV) + l * -(-P // 64) * 64
        k, v = (torch.from_numpy(np.ascontiguousarray(inp[n][l], dtype=np.float16)).to(DEV).view(P, H, hd) for n in ("kp", "vp"))
        oq.kv4_append(cache, k, v, slots)
        model.load_prefix(l, cache, slots)
        values.append([t.float().cpu().numpy().reshape(1, P, H * hd) for t in oq.kv4_gather(cache, slots)])
    a = model.step(x0.clone(), 0)
    inp2 = dict(inp, kp=[v[0] for v in values], vp=[v[1] for v in values])
    other = oq.DiT(cfg, inp2, device="cuda:0")
    b = other.step(x0.clone(), 0)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and not torch.equal(a, plain)
    with pytest.raises(ValueError, match="heads"):
        model.load_prefix(0, oq.KV4Cache.empty(1, 1, hd), slots)
    model.close()
    other.close()
