"""Cases of a layer's linears in microscaled 4-bit floating point and of what
stands between two of them: quantization (with the values read back), the
product, the norms before and after a block with its gate and residual, and
the gated activation.

Each kind is computed here in its plain form (elementary torch operations in
32 bits, in 64 where a value is rounded to a 4-bit code) and, where `own` is
set, by the library's calls.  Inputs are seeded and synthetic, made on the GPU.

Format: blocks of 32 channels share a step 2^s, s = floor(log2 max|x|) - 2
clamped to [-127, 127], held as the byte s + 127 (255: a block with an infinity
or a NaN); a channel's code is x / 2^s rounded to the nearest of 0, 0.5, 1, 1.5,
2, 3, 4, 6 (ties to the even code, past 6: 6), its index in the low three bits
and the sign in the fourth.  Codes: uint8 [rows][K / 2], the even channel in the
low nibble.  Steps: uint8 [rows][16 ceil(K / 512)], the first K / 32 of a row in use.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LARGEST = 16384 * 4096          # elements of an activation


def listed():
    return [
        # One decoded token's hidden state on its way into a linear: latency.
        {"name": "quantize_token_2048", "kind": "quantize", "M": 1, "K": 2048, "had": 1, "dtype": "bf16"},
        # A prompt's MLP activations, rotated in blocks of 32.
        {"name": "quantize_prompt_816x16384", "kind": "quantize", "M": 816, "K": 16384, "had": 32, "dtype": "f16"},
        # A large batched prefill, rotated in blocks of 128.
        {"name": "quantize_16384x4096", "kind": "quantize", "M": 16384, "K": 4096, "had": 128, "dtype": "bf16"},
        # One decoded token through a backbone's q|k|v linear: latency.
        {"name": "linear_token_qkv", "kind": "linear", "M": 1, "N": 2560, "K": 2048, "out": "bf16", "bias": False},
        # 50 action tokens through an action head's down linear, with a bias.
        {"name": "linear_actions_50", "kind": "linear", "M": 50, "N": 1024, "K": 4096, "out": "f16", "bias": True},
        # The gate|up linear over one prompt of 816 image and text tokens.
        {"name": "linear_prompt_gate_up", "kind": "linear", "M": 816, "N": 32768, "K": 2048, "out": "f16", "bias": False},
        # A large batched prefill, rows and columns off the tile sizes.
        {"name": "linear_4000x8200x8192", "kind": "linear", "M": 4000, "N": 8200, "K": 8192, "out": "bf16", "bias": True},
        # One decoded token between two blocks, normed behind the first and
        # before the second: latency.
        {"name": "norm_token_2048", "kind": "norm", "M": 1, "D": 2048, "post": "rms", "pre": "rms", "mods": 0,
         "resid": "bf16", "dtype": "bf16", "mx4": True},
        # An action head's batch of 64 x 16 tokens with each sample's own gate,
        # scale and shift.
        {"name": "norm_actions_64x16", "kind": "norm", "M": 1024, "D": 1536, "post": "none", "pre": "layer", "mods": 64,
         "resid": "f32", "dtype": "f16", "mx4": False},
        # A large prefill, the second norm's output in codes.
        {"name": "norm_prefill_16384x4096", "kind": "norm", "M": 16384, "D": 4096, "post": "rms", "pre": "rms", "mods": 0,
         "resid": "f32", "dtype": "bf16", "mx4": True},
        # The MLP's activation over one prompt, in codes for the down linear.
        {"name": "act_prompt_816", "kind": "act", "M": 816, "F": 16384, "act": "gelu", "dtype": "f16", "mx4": True},
        # A ragged large batch through another width, in 16 bits.
        {"name": "act_4011x5632", "kind": "act", "M": 4011, "F": 5632, "act": "silu", "dtype": "bf16", "mx4": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "norm", "act"])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "linear":
        c = {"kind": kind, "M": _log(rng, 1, 16384), "N": _log(rng, 1, 32768), "K": 32 * _log(rng, 1, 512),
             "out": dtype, "bias": rng.random() < 0.5}
        while c["M"] * c["N"] * c["K"] > 4000 * 8200 * 8192:
            c["M"] = max(1, c["M"] // 2)
        return c
    if kind == "quantize":
        c = {"kind": kind, "M": _log(rng, 1, 16384), "K": 32 * _log(rng, 1, 512), "had": rng.choice([1, 32, 64, 128]),
             "dtype": dtype}
        while c["K"] % c["had"]:
            c["had"] //= 2
        while c["M"] * c["K"] > LARGEST:
            c["M"] //= 2
        return c
    mx4 = rng.random() < 0.5
    if kind == "norm":
        c = {"kind": kind, "M": _log(rng, 1, 16384), "D": 32 * _log(rng, 1, 512) if mx4 else 8 * _log(rng, 1, 2048),
             "post": rng.choice(["none", "rms", "layer"]), "pre": rng.choice(["rms", "layer"]),
             "mods": rng.choice([0, 1, 7, 64]), "resid": rng.choice([dtype, "f32"]), "dtype": dtype, "mx4": mx4}
        while c["M"] * c["D"] > LARGEST:
            c["M"] //= 2
        return c
    c = {"kind": kind, "M": _log(rng, 1, 16384), "F": 32 * _log(rng, 1, 512) if mx4 else 8 * _log(rng, 1, 2048),
         "act": rng.choice(["gelu", "silu"]), "dtype": dtype, "mx4": mx4}
    while c["M"] * c["F"] > LARGEST // 2:
        c["M"] //= 2
    return c


def work(case):
    kind = case["kind"]
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M + N) * K * 17 // 32 + 2 * M * N + (2 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    if kind == "quantize":
        # read X, write and read codes and steps, write their values
        n = case["M"] * case["K"]
        return {"bytes": n * (2 + 2) + 2 * n * 17 // 32, "flops": n * (4 + (int(math.log2(case["had"])) if case["had"] > 1 else 0))}
    out = 2 + 2 * 17 / 32 if case["mx4"] else 2
    if kind == "norm":
        n = case["M"] * case["D"]
        mods = 3 * 2 * case["mods"] * case["D"]
        return {"bytes": int(n * (2 + 2 * (4 if case["resid"] == "f32" else 2) + out)) + mods + 8 * case["D"], "flops": 16 * n}
    n = case["M"] * case["F"]
    return {"bytes": int(n * (4 + out)), "flops": 20 * n}


def _outliers(x, g):
    """0.5% of the channels of x [rows, K] times 30, as activations have them."""
    m = torch.rand(x.shape[-1:], generator=g, device=DEV) < 0.005
    return torch.where(m, 30.0 * x, x)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, M = case["kind"], case["M"]
    state = dict(case)
    rnd = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    if kind == "quantize":
        state["x"] = _outliers(rnd(M, case["K"]), g).to(DTYPE[case["dtype"]])
    elif kind == "linear":
        # Codes and steps as quantization leaves them; the bytes of a row of
        # steps that are not in use hold 255.
        for name, x in (("x", _outliers(rnd(M, case["K"]), g)), ("w", 0.02 * rnd(case["N"], case["K"]))):
            q, s = _plain_codes(x)
            steps = torch.full((x.shape[0], 16 * -(-case["K"] // 512)), 255, dtype=torch.uint8, device=DEV)
            steps[:, : s.shape[1]] = s
            state[name + "q"], state[name + "s"] = q, steps
        state["b"] = rnd(case["N"]).half() if case["bias"] else None
    elif kind == "norm":
        D, dt = case["D"], DTYPE[case["dtype"]]
        state.update(y=_outliers(rnd(M, D), g).to(dt), r=(4.0 * _outliers(rnd(M, D), g)).to(DTYPE[case["resid"]]),
                     g1=(1 + 0.1 * rnd(D)).to(dt), b1=(0.1 * rnd(D)).to(dt), g2=(1 + 0.1 * rnd(D)).to(dt), b2=(0.1 * rnd(D)).to(dt),
                     gate=None, scale=None, shift=None, row=None, alpha=0.75)
        n = case["mods"]
        if n:
            state.update(gate=(1 + 0.1 * rnd(n, D)).to(dt), scale=(0.1 * rnd(n, D)).to(dt), shift=(0.1 * rnd(n, D)).to(dt),
                         row=(torch.arange(M, device=DEV) * n // M).to(torch.int32))
    else:
        state["gu"] = (1.5 * rnd(M, 2 * case["F"])).to(DTYPE[case["dtype"]])
    return state


# -- plain forms --------------------------------------------------------------

def _pow2(e):
    """2^e as float64, exactly (e whole, -1022 .. 1023)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _plain_codes(x):
    """Codes uint8 [rows, K / 2] and steps uint8 [rows, K / 32] of finite x [rows, K]."""
    v = x.view(x.shape[0], -1, 32)
    _, e = torch.frexp(v.abs().amax(-1))           # max = m 2^e, 0.5 <= m < 1
    s = torch.where(e == 0, torch.where(v.abs().amax(-1) > 0, -3, -127), e - 3).clamp(-127, 127)
    a = v.abs() * _pow2(-s[..., None])
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    a = torch.clamp(torch.round(a / step) * step, max=6.0)
    index = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    index = (index | torch.where(v < 0, 8, 0).to(torch.uint8)).view(x.shape)
    return index[:, 0::2] | index[:, 1::2] << 4, (s + 127).to(torch.uint8)


def _values(q, s):
    """What codes [rows, K / 2] and steps [rows, >= K / 32] stand for, [rows, K]."""
    grid = torch.tensor(GRID + tuple(-x for x in GRID), device=q.device)
    both = torch.stack((q & 15, q >> 4), -1).flatten(-2).long()
    v = grid[both].view(q.shape[0], -1, 32)
    return (v * _pow2(s[:, : v.shape[1], None].to(torch.int64) - 127).float()).view(both.shape)


def _through_codes(x):
    return _values(*_plain_codes(x)).to(torch.bfloat16)


def _hadamard(n):
    h = torch.ones((1, 1), dtype=torch.float64, device=DEV)
    two = torch.tensor([[1.0, 1.0], [1.0, -1.0]], dtype=torch.float64, device=DEV)
    for _ in range(int(math.log2(n))):
        h = torch.kron(two, h)
    return h


def _plain_quantize(s):
    x, b = s["x"].double(), s["had"]
    if b > 1:
        x = ((x.view(-1, b) @ _hadamard(b)) / math.sqrt(b)).view(x.shape)
    return _through_codes(x)


def _plain_linear(s):
    y = _values(s["xq"], s["xs"]) @ _values(s["wq"], s["ws"]).T
    y = y if s["b"] is None else y + s["b"].float()
    return y.to(DTYPE[s["out"]])


def _plain_norm_of(x, kind, gain, bias):
    eps = 1e-6
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * gain
    return n + bias if kind == "layer" else n


def _plain_norm(s):
    wide = torch.float64 if s["mx4"] else torch.float32
    up = lambda t: t.to(wide)  # noqa: E731
    y = up(s["y"])
    if s["post"] != "none":
        y = _plain_norm_of(y, s["post"], up(s["g1"]), up(s["b1"]))
    rows = None if s["row"] is None else s["row"].long()
    if rows is not None:
        y = y * up(s["gate"])[rows]
    r = s["alpha"] * up(s["r"]) + y
    h = _plain_norm_of(r, s["pre"], up(s["g2"]), up(s["b2"]))
    if rows is not None:
        h = h * (1 + up(s["scale"])[rows]) + up(s["shift"])[rows]
    return {"r": r.to(s["r"].dtype), "h": _through_codes(h) if s["mx4"] else h.to(s["y"].dtype)}


def _plain_act(s):
    x = s["gu"].to(torch.float64 if s["mx4"] else torch.float32)
    g, u = x[:, : s["F"]], x[:, s["F"]:]
    t = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g) if s["act"] == "gelu" else g
    h = g / (1 + torch.exp(-t)) * u
    return _through_codes(h) if s["mx4"] else h.to(s["gu"].dtype)


# -- the library's calls ------------------------------------------------------

def _own_values(oq, codes):
    return oq.mx4_dequantize(*codes, out_dtype=oq.OUT_BF16)


def _own_quantize(oq, s):
    return _own_values(oq, oq.mx4_quantize(s["x"], had_block=s["had"]))


def _own_linear(oq, s):
    return oq.mx4_linear(s["xq"], s["xs"], s["wq"], s["ws"], s["b"], oq.OUT_F16 if s["out"] == "f16" else oq.OUT_BF16)


def _own_norm(oq, s):
    if "norms" not in s:  # the norms' parameters, held once by a program
        post = None if s["post"] == "none" else oq.Norm(s["post"], s["g1"], s["b1"] if s["post"] == "layer" else None, eps=1e-6)
        pre = oq.Norm(s["pre"], s["g2"], s["b2"] if s["pre"] == "layer" else None, eps=1e-6)
        s["norms"] = post, pre
    post, pre = s["norms"]
    r, h = oq.residual_norm(s["r"], s["y"], pre=pre, post=post, alpha=s["alpha"], gate=s["gate"], scale=s["scale"],
                            shift=s["shift"], mod_row=s["row"], mx4=s["mx4"])
    return {"r": r, "h": _own_values(oq, h) if s["mx4"] else h}


def _own_act(oq, s):
    h = oq.gated_activation(s["gu"], oq.ACT_GELU_TANH if s["act"] == "gelu" else oq.ACT_SILU, mx4=s["mx4"])
    return _own_values(oq, h) if s["mx4"] else h


def run(state):
    kind = state["kind"]
    if own:
        import paper_2605_28803_amd as oq
        return {"quantize": _own_quantize, "linear": _own_linear, "norm": _own_norm, "act": _own_act}[kind](oq, state)
    return {"quantize": _plain_quantize, "linear": _plain_linear, "norm": _plain_norm, "act": _plain_act}[kind](state)


# -- 64 bits ------------------------------------------------------------------

def _powers64():
    return torch.tensor([2.0 ** e for e in range(-300, 301)], dtype=torch.float64, device=DEV)


def _nearest64(x):
    """The value that the 4-bit code of each x (float64 [rows, K], finite) stands for."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().max(-1, keepdim=True).values
    e = torch.floor(torch.log2(top.clamp_min(2.0 ** -200)))
    p = _powers64()[(e + 300).long()]
    e = e + (top >= 2 * p).double() - (top < p).double()
    unit = _powers64()[((e - 2).clamp(-127, 127) + 300).long()]
    a = b.abs() / unit
    # Above a border, or on one of those whose upper neighbour has the even code.
    v = torch.zeros_like(a)
    for at, gap, tie_up in ((0.25, 0.5, False), (0.75, 0.5, True), (1.25, 0.5, False), (1.75, 0.5, True), (2.5, 1.0, False),
                            (3.5, 1.0, True), (5.0, 2.0, False)):
        v += gap * ((a >= at) if tie_up else (a > at))
    return (torch.sign(b) * v * unit).flatten(-2)


def _signs64(n):
    i = torch.arange(n, device=DEV)
    odd = torch.zeros((n, n), dtype=torch.int64, device=DEV)
    for s in range(8):
        odd ^= ((i[:, None] & i[None, :]) >> s) & 1
    return (1 - 2 * odd).double()


def _operand64(q, s, K):
    mag = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=DEV) / 2
    x = torch.empty((q.shape[0], K), dtype=torch.float64, device=DEV)
    for nibble, part in ((q % 16, x[:, ::2]), (q // 16, x[:, 1::2])):
        part.copy_(mag[(nibble % 8).long()] * (1 - 2 * (nibble // 8).double()))
    return x * _powers64()[s[:, : K // 32].long() + 173].repeat_interleave(32, dim=1)


def _normed64(x, kind, gain, bias):
    if kind == "rms":
        return x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * gain.double()
    var, mean = torch.var_mean(x, -1, keepdim=True, correction=0)
    return (x - mean) / torch.sqrt(var + 1e-6) * gain.double() + bias.double()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        out = []
        for x in s["x"].split(4096):
            x = x.double()
            if case["had"] > 1:
                x = torch.mm(x.reshape(-1, case["had"]), _signs64(case["had"])).mul_(case["had"] ** -0.5).view(x.shape)
            out.append(_nearest64(x))
        return torch.cat(out)
    if kind == "linear":
        w = _operand64(s["wq"], s["ws"], case["K"]).t()
        out = []
        for q, st in zip(s["xq"].split(4096), s["xs"].split(4096)):
            y = torch.mm(_operand64(q, st, case["K"]), w)
            out.append(y if s["b"] is None else y.add_(s["b"].double()))
        return torch.cat(out)
    if kind == "norm":
        rs, hs = [], []
        for at in range(0, case["M"], 4096):
            rows = slice(at, at + 4096)
            y = s["y"][rows].double()
            if case["post"] != "none":
                y = _normed64(y, case["post"], s["g1"], s["b1"])
            if s["row"] is not None:
                y = s["gate"].double().index_select(0, s["row"][rows]) * y
            r = torch.add(y, s["r"][rows].double(), alpha=s["alpha"])
            h = _normed64(r, case["pre"], s["g2"], s["b2"])
            if s["row"] is not None:
                h = torch.addcmul(s["shift"].double().index_select(0, s["row"][rows]), h,
                                  s["scale"].double().index_select(0, s["row"][rows]) + 1)
            rs.append(r)
            hs.append(_nearest64(h) if case["mx4"] else h)
        return {"r": torch.cat(rs), "h": torch.cat(hs)}
    out = []
    for x in s["gu"].split(2048):
        g, u = x.double().split(case["F"], dim=1)
        gate = torch.sigmoid(g if case["act"] == "silu" else (8 / math.pi) ** 0.5 * g * (1 + 0.044715 * g.square()))
        out.append(_nearest64(g * gate * u) if case["mx4"] else g * gate * u)
    return torch.cat(out)
