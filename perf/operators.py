"""Cases of the operators of a backbone layer at serving time: the 8-bit
integer product, attention over a packed prompt, and the 4-bit key/value cache
(append, read back, attention over its pages).

Each kind is computed here in its plain form (elementary torch operations in
32 bits) and, where `own` is set, by the library's calls.  Inputs are seeded
and synthetic, made on the GPU.

Cache layout (what KV4Cache holds): pages of `page` tokens per kv head, codes
two's-complement nibbles in [-7, 7].  k_codes [page][head][token][hd / 2]: byte
b holds channels 2 b (low nibble) and 2 b + 1 (high).  v_codes
[page][head][token / 16][hd / 2][16]: byte (b, t) holds channels 2 b and 2 b + 1
of token t of the 16.  k_scale, v_scale fp32 [page][head][token].  A cache with
rotated keys holds k H / sqrt(hd), H the Sylvester Hadamard matrix.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # One decoded token through a backbone's q|k|v linear (2048 channels,
        # 8 x 256 query and 256 + 256 key and value columns): latency.
        {"name": "w8a8_token_qkv", "kind": "w8a8", "M": 1, "N": 2560, "K": 2048, "out": "f16", "bias": False},
        # The gate|up linear over one prompt of 816 image and text tokens.
        {"name": "w8a8_prompt_gate_up", "kind": "w8a8", "M": 816, "N": 32768, "K": 2048, "out": "f16", "bias": False},
        # A large batched prefill, rows and columns off the tile sizes.
        {"name": "w8a8_4000x8200x8192", "kind": "w8a8", "M": 4000, "N": 8200, "K": 8192, "out": "bf16", "bias": True},
        # A vision-language prefix (every token sees its whole sequence): five
        # prompts of up to 816 tokens, 8 query heads on one kv head of 256.
        {"name": "prompt_prefix_5x816", "kind": "prompt", "seqs": 5, "longest": 816, "spread": 1.2, "hq": 8, "hk": 1,
         "hd": 256, "causal": False, "dtype": "bf16"},
        # Many short and ragged causal prompts packed together, one head of
        # keys for each head of queries.
        {"name": "prompt_ragged_48x600", "kind": "prompt", "seqs": 48, "longest": 600, "spread": 60.0, "hq": 16,
         "hk": 16, "hd": 64, "causal": True, "dtype": "f16"},
        # One long causal prompt with grouped heads.
        {"name": "prompt_long_8192", "kind": "prompt", "seqs": 1, "longest": 8192, "spread": 1.0, "hq": 32, "hk": 8,
         "hd": 128, "causal": True, "dtype": "bf16"},
        # The tokens of one decoding step of 64 sequences enter the cache (and
        # are read back as the values they now stand for).
        {"name": "append_step_64", "kind": "append", "tokens": 64, "hk": 8, "hd": 128, "page": 64, "rotate": False,
         "run": 1, "dtype": "f16"},
        # Prompts of 16000 tokens in all enter the cache with rotated keys.
        {"name": "append_prompts_16000", "kind": "append", "tokens": 16000, "hk": 8, "hd": 128, "page": 64,
         "rotate": True, "run": 800, "dtype": "bf16"},
        # One token of one sequence over a vision-language prefix: a single
        # kv head, where only the split over the length fills the card.
        {"name": "cache_token_1x866", "kind": "cache", "seqs": 1, "longest": 866, "spread": 1.0, "nq": 1, "hq": 8,
         "hk": 1, "hd": 256, "page": 64, "rotate": True, "causal": True, "dtype": "bf16"},
        # Four policies' 50 action tokens each over their 816 cached tokens and
        # themselves, all seeing all.
        {"name": "cache_actions_4x50", "kind": "cache", "seqs": 4, "longest": 866, "spread": 1.0, "nq": 50, "hq": 8,
         "hk": 8, "hd": 128, "page": 32, "rotate": False, "causal": False, "dtype": "f16"},
        # A decoding step of 64 ragged sequences with grouped heads.
        {"name": "cache_step_64x4096", "kind": "cache", "seqs": 64, "longest": 4096, "spread": 16.0, "nq": 1, "hq": 32,
         "hk": 8, "hd": 128, "page": 64, "rotate": False, "causal": True, "dtype": "bf16"},
        # One token over a long document.
        {"name": "cache_long_131000", "kind": "cache", "seqs": 1, "longest": 131000, "spread": 1.0, "nq": 1, "hq": 32,
         "hk": 8, "hd": 128, "page": 128, "rotate": False, "causal": True, "dtype": "f16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["w8a8", "w8a8", "prompt", "prompt", "append", "cache", "cache"])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "w8a8":
        c = {"kind": kind, "M": _log(rng, 1, 16384), "N": 8 * _log(rng, 8, 4096), "K": 64 * _log(rng, 1, 256),
             "out": dtype, "bias": rng.random() < 0.5}
        while c["M"] * c["N"] * c["K"] > 4000 * 8200 * 8192:
            c["M"] = max(1, c["M"] // 2)
        return c
    hd = rng.choice([64, 128, 256])
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 2, 4, 5, 8])
    if kind == "prompt":
        c = {"kind": kind, "seqs": _log(rng, 1, 64), "longest": _log(rng, 1, 8192), "spread": rng.choice([1.0, 4.0, 50.0]),
             "hq": hq, "hk": hk, "hd": hd, "causal": rng.random() < 0.7, "dtype": dtype}
        # (The plain form holds every pair of packed tokens.)
        while c["seqs"] * c["longest"] > 8192:
            c["seqs"], c["longest"] = max(1, c["seqs"] // 2), max(1, c["longest"] * 2 // 3)
        while c["hq"] * c["hd"] > 4096 or c["hq"] > 32:
            c["hq"], c["hk"] = c["hq"] // c["hk"], 1
        while sum(n * n for n in _lengths(c)) * c["hq"] * c["hd"] * (1 if c["causal"] else 2) > 8192 * 8192 * 32 * 128:
            c["longest"] = max(1, c["longest"] // 2)
        return c
    page = rng.choice([32, 64, 128, 256])
    if kind == "append":
        c = {"kind": kind, "tokens": _log(rng, 1, 16000), "hk": hk, "hd": hd, "page": page, "rotate": rng.random() < 0.5,
             "run": _log(rng, 1, 1000), "dtype": dtype}
        while c["tokens"] * hk * hd > 16000 * 8 * 128:
            c["tokens"] //= 2
        return c
    c = {"kind": kind, "seqs": _log(rng, 1, 128), "longest": _log(rng, 1, 131000), "spread": rng.choice([1.0, 4.0, 50.0]),
         "nq": rng.choice([1, 1, 1, 2, 5, 50]), "hq": hq, "hk": hk, "hd": hd, "page": page,
         "rotate": rng.random() < 0.5, "causal": rng.random() < 0.8, "dtype": dtype}
    while c["seqs"] * c["longest"] * hk * hd > 131000 * 8 * 128:
        c["seqs"], c["longest"] = max(1, c["seqs"] // 2), max(1, c["longest"] * 3 // 4)
    while c["nq"] > 1 and c["seqs"] * c["longest"] * c["hq"] * c["nq"] * hd > 131000 * 32 * 4 * 128:
        c["nq"] = max(1, c["nq"] // 5)
    c["longest"] = max(c["longest"], c["nq"])
    return c


def _lengths(case):
    """Lengths of the case's sequences: the longest first, the others spread
    over a factor `spread` below it (by their logarithm)."""
    r = random.Random(17 * case["longest"] + case["seqs"])
    least = case.get("nq", 1)
    more = [max(least, int(case["longest"] / math.exp(r.uniform(0, math.log(case["spread"])))))
            for _ in range(case["seqs"] - 1)]
    return [case["longest"]] + more


def _pairs(case):
    """Query-key pairs that the mask leaves, over all sequences."""
    n = 0
    for length in _lengths(case):
        q = case.get("nq", length)
        n += q * length - (q * (q - 1) // 2 if case["causal"] else 0)
    return n


def work(case):
    kind = case["kind"]
    if kind == "w8a8":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + 4 * (M + N) + 2 * M * N + (2 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    hk, hd = case["hk"], case["hd"]
    if kind == "append":
        n = case["tokens"] * hk
        # read K and V, write and read codes and scales, write the fp32 values
        return {"bytes": n * (4 * hd + 2 * (hd + 8) + 8 * hd) + 16 * case["tokens"],
                "flops": n * hd * (4 + (2 * int(math.log2(hd)) if case["rotate"] else 0))}
    flops = 4 * hd * case["hq"] * _pairs(case)
    if kind == "prompt":
        return {"bytes": 2 * sum(_lengths(case)) * (2 * case["hq"] + 2 * hk) * hd, "flops": flops}
    tokens = case["seqs"] * case["nq"]
    return {"bytes": sum(_lengths(case)) * hk * (hd + 8) + 4 * tokens * case["hq"] * hd, "flops": flops}


def _outliers(x, g):
    """1% of the channels of x ([..., hd]) times 8, as keys have them."""
    m = torch.rand(x.shape[-2:], generator=g, device=DEV) < 0.01
    return torch.where(m, 8.0 * x, x)


def _order(n, seed):
    return torch.randperm(n, generator=torch.Generator().manual_seed(seed))


def _fill(shape, page, pages, table, lens, g, rotate):
    """A cache that holds `lens` tokens of seeded keys and values behind each
    row of the page table; the rest of it is left as it came (NaN scales)."""
    hk, hd = shape
    state = {"k_codes": torch.randint(0, 256, (pages, hk, page, hd // 2), generator=g, device=DEV, dtype=torch.uint8),
             "v_codes": torch.randint(0, 256, (pages, hk, page // 16, hd // 2, 16), generator=g, device=DEV, dtype=torch.uint8),
             "k_scale": torch.full((pages, hk, page), float("nan"), device=DEV),
             "v_scale": torch.full((pages, hk, page), float("nan"), device=DEV)}
    for row, n in zip(table, lens):
        used = row[: -(-n // page)].long().to(DEV)
        t = used.numel() * page
        for name in ("k", "v"):
            x = torch.randn((t, hk, hd), generator=g, device=DEV)
            if name == "k":
                x = _outliers(x, g)
                x = x @ _hadamard(hd, torch.float32) / math.sqrt(hd) if rotate else x
            top = x.abs().amax(-1, keepdim=True)
            q = (torch.round(7 * x / top).to(torch.int32) & 15).to(torch.uint8)
            packed = (q[..., 0::2] | q[..., 1::2] << 4).view(-1, page, hk, hd // 2)
            scale = (top[..., 0] / 7).masked_fill((torch.arange(t, device=DEV) >= n)[:, None], float("nan"))
            state[name + "_scale"][used] = scale.view(-1, page, hk).transpose(1, 2)
            if name == "k":
                state["k_codes"][used] = packed.transpose(1, 2)
            else:
                state["v_codes"][used] = packed.view(-1, page // 16, 16, hk, hd // 2).permute(0, 3, 1, 4, 2)
    return state


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    state = dict(case)
    if case["kind"] == "w8a8":
        M, N, K = case["M"], case["N"], case["K"]
        code = lambda n: torch.clamp(torch.round(torch.randn((n, K), generator=g, device=DEV) * 32), -127, 127).to(torch.int8)  # noqa: E731
        state.update(Xq=code(M), Wq=code(N), xs=torch.rand((M,), generator=g, device=DEV) * 0.02 + 0.01,
                     ws=torch.rand((N,), generator=g, device=DEV) * 4e-4 + 2e-4,
                     b=torch.randn((N,), generator=g, device=DEV).half() if case["bias"] else None)
        return state
    hk, hd, dt = case["hk"], case["hd"], DTYPE[case["dtype"]]
    if case["kind"] == "prompt":
        lens = _lengths(case)
        hq, total = case["hq"], sum(lens)
        # q|k|v of a token side by side, as one linear writes them.
        qkv = torch.randn((total, hq + 2 * hk, hd), generator=g, device=DEV)
        qkv = _outliers(qkv, g).to(dt)
        state.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:],
                     cu=torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV))
        return state
    page = case["page"]
    if case["kind"] == "append":
        n, run = case["tokens"], min(case["run"], case["tokens"])
        # Runs of tokens, each from the place in a page where its sequence goes on.
        at = _order(64, seed)
        pages = -(-(run + 64) // page)
        first = torch.arange(-(-n // run)) * pages * page + at[torch.arange(-(-n // run)) % 64]
        slots = (first[:, None] + torch.arange(run)[None, :]).reshape(-1)[:n]
        total = pages * first.numel()
        table = _order(total, seed + 1)
        slots = table[slots // page] * page + slots % page
        state.update(_fill((hk, hd), page, total, [], [], g, case["rotate"]), slots=slots.to(DEV),
                     k=_outliers(torch.randn((n, hk, hd), generator=g, device=DEV), g).to(dt),
                     v=torch.randn((n, hk, hd), generator=g, device=DEV).to(dt))
        return state
    lens = _lengths(case)
    wide = -(-max(lens) // page)
    total = sum(-(-n // page) for n in lens) + 3
    order, table, at = _order(total, seed), torch.zeros((len(lens), wide), dtype=torch.int32), 0
    for i, n in enumerate(lens):
        m = -(-n // page)
        table[i, :m] = order[at:at + m]
        at += m
    nq = case["nq"]
    state.update(_fill((hk, hd), page, total, table, lens, g, case["rotate"]), table=table.to(DEV),
                 lens=torch.tensor(lens, dtype=torch.int32, device=DEV), longest=max(lens),
                 cu=torch.arange(len(lens) + 1, dtype=torch.int32, device=DEV) * nq,
                 q=torch.randn((len(lens) * nq, case["hq"], hd), generator=g, device=DEV).to(dt))
    return state


# -- plain forms --------------------------------------------------------------

def _hadamard(n, dtype):
    h = torch.ones((1, 1), dtype=dtype, device=DEV)
    two = torch.tensor([[1.0, 1.0], [1.0, -1.0]], dtype=dtype, device=DEV)
    for _ in range(int(math.log2(n))):
        h = torch.kron(two, h)
    return h


def _nibbles(p):
    """Packed codes [..., hd / 2] as signed values [..., hd]."""
    both = torch.stack((p & 15, p >> 4), -1).flatten(-2).float()
    return torch.where(both >= 8, both - 16, both)


def _softmax_rows(s, mask):
    """exp(s - max) over the last axis where `mask` holds, and its sum."""
    s = s.masked_fill(~mask, float("-inf"))
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(torch.isinf(top), 0.0, top))
    return e, e.sum(-1, keepdim=True)


def _plain_w8a8(s):
    acc = s["Xq"].float() @ s["Wq"].float().T
    y = acc * s["xs"][:, None] * s["ws"][None, :]
    y = y if s["b"] is None else y + s["b"].float()
    return y.to(DTYPE[s["out"]])


def _plain_prompt(s):
    q, k, v = (s[x].float().transpose(0, 1) for x in "qkv")           # [heads, T, hd]
    t, hk = q.shape[1], s["hk"]
    pos = torch.arange(t, device=DEV)
    seq = torch.bucketize(pos, s["cu"][1:].long(), right=True)
    mask = seq[:, None] == seq[None, :]
    mask = mask & (pos[None, :] <= pos[:, None]) if s["causal"] else mask
    q = q.reshape(hk, -1, t, s["hd"]) / math.sqrt(s["hd"])
    e, total = _softmax_rows(q @ k[:, None].transpose(-1, -2).contiguous(), mask)
    o = (e @ v[:, None]) / total
    return o.flatten(0, 1).transpose(0, 1).to(s["q"].dtype)


def _plain_codes(x, norm):
    """Codes and steps of the rows x / norm in 64 bits: a ratio next to a half
    integer goes one way or the other, so it is formed before norm (a root)."""
    top = x.abs().amax(-1, keepdim=True)
    q = torch.round(7 * x / torch.where(top > 0, top, 1.0))
    return q, (top[..., 0] / (7 * norm)).float()


def _plain_append(s):
    hd, page, slots = s["hd"], s["page"], s["slots"]
    k, v = s["k"].double(), s["v"].double()
    if s["rotate"]:
        k = k @ _hadamard(hd, torch.float64)
    at, t = slots // page, slots % page
    for name, x, norm in (("k", k, math.sqrt(hd) if s["rotate"] else 1.0), ("v", v, 1.0)):
        q, scale = _plain_codes(x, norm)
        q = (q.to(torch.int32) & 15).to(torch.uint8)
        packed = q[..., 0::2] | q[..., 1::2] << 4                         # [n, hk, hd / 2]
        s[name + "_scale"][at, :, t] = scale
        if name == "k":
            s["k_codes"][at, :, t] = packed
        else:
            s["v_codes"][at, :, t // 16, :, t % 16] = packed
    k = _nibbles(s["k_codes"][at, :, t]) * s["k_scale"][at, :, t][..., None]
    v = _nibbles(s["v_codes"][at, :, t // 16, :, t % 16]) * s["v_scale"][at, :, t][..., None]
    if s["rotate"]:
        k = (k @ _hadamard(hd, torch.float32)) / math.sqrt(hd)
    return {"k": k, "v": v}


def _plain_cache(s):
    hk, hd, page, nq, wide = s["hk"], s["hd"], s["page"], s["nq"], s["longest"]
    b = s["lens"].numel()
    q = s["q"].float()
    if s["rotate"]:
        q = (q @ _hadamard(hd, torch.float32)) / math.sqrt(hd)
    q = q.view(b, nq, hk, -1, hd).permute(0, 2, 3, 1, 4).flatten(2, 3) / math.sqrt(hd)   # [b, hk, rows, hd]
    table = s["table"].long()
    there = torch.arange(wide, device=DEV)[None, :] < s["lens"][:, None]
    ks, vs = (s[n][table].permute(0, 2, 1, 3).flatten(2)[:, :, :wide] for n in ("k_scale", "v_scale"))
    ks, vs = (torch.where(there[:, None], x, 0.0) for x in (ks, vs))
    k = _nibbles(s["k_codes"][table].permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :wide])
    sc = (q @ k.transpose(-1, -2).contiguous()) * ks[:, :, None]
    del k
    last = s["lens"].long()[:, None] - nq + torch.arange(nq, device=DEV)[None, :] if s["causal"] else \
        (s["lens"].long() - 1)[:, None].expand(b, nq)
    mask = torch.arange(wide, device=DEV)[None, None, :] <= last[:, :, None]              # [b, nq, wide]
    mask = mask[:, None, None].expand(b, 1, s["hq"] // hk, nq, wide).flatten(2, 3)
    e, total = _softmax_rows(sc, mask)
    del sc
    v = _nibbles(s["v_codes"][table].permute(0, 2, 1, 3, 5, 4).flatten(2, 4)[:, :, :wide])
    o = (e * vs[:, :, None]) @ v / total
    return o.view(b, hk, -1, nq, hd).permute(0, 3, 1, 2, 4).reshape(b * nq, s["hq"], hd).to(s["q"].dtype)


# -- the library's calls ------------------------------------------------------

def _own_cache(oq, s):
    if "cache" not in s:  # the holder of a cache's tensors, made once by a program
        s["cache"] = oq.KV4Cache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], rotate_k=s["rotate"])
    return s["cache"]


def _own_w8a8(oq, s):
    return oq.w8a8_linear(s["Xq"], s["xs"], s["Wq"], s["ws"], s["b"], oq.OUT_F16 if s["out"] == "f16" else oq.OUT_BF16)


def _own_prompt(oq, s):
    return oq.attention_prompt(s["q"], s["k"], s["v"], s["cu"], causal=s["causal"])


def _own_append(oq, s):
    cache = _own_cache(oq, s)
    oq.kv4_append(cache, s["k"], s["v"], s["slots"])
    k, v = oq.kv4_gather(cache, s["slots"], oq.OUT_F32)
    return {"k": k, "v": v}


def _own_cache_attention(oq, s):
    one = s["nq"] == 1
    return oq.attention_kv4(s["q"], _own_cache(oq, s), s["table"], s["lens"], None if one else s["cu"], max_q=s["nq"],
                            max_len=s["longest"], causal=s["causal"])


def run(state):
    kind = state["kind"]
    if own:
        import paper_2605_28803_amd as oq
        return {"w8a8": _own_w8a8, "prompt": _own_prompt, "append": _own_append, "cache": _own_cache_attention}[kind](oq, state)
    return {"w8a8": _plain_w8a8, "prompt": _plain_prompt, "append": _plain_append, "cache": _plain_cache}[kind](state)


# -- 64 bits ------------------------------------------------------------------

def _signs64(n):
    i = torch.arange(n, device=DEV)
    bits = i[:, None] & i[None, :]
    odd = torch.zeros_like(bits)
    for s in range(9):
        odd ^= (bits >> s) & 1
    return (1 - 2 * odd).double()


def _signed64(byte):
    lo, hi = (byte % 16).long(), (byte // 16).long()
    x = torch.empty(byte.shape[:-1] + (2 * byte.shape[-1],), dtype=torch.float64, device=byte.device)
    x[..., ::2] = (lo - 16 * (lo > 7)).double()
    x[..., 1::2] = (hi - 16 * (hi > 7)).double()
    return x


def _attend64(q, k, v, visible):
    """One head: rows q [n, hd], keys and values [L, hd], and how many keys each row sees."""
    s = q @ k.T / math.sqrt(q.shape[-1])
    s[torch.arange(k.shape[0], device=DEV)[None, :] >= visible[:, None]] = float("-inf")
    return torch.softmax(s, -1) @ v


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "w8a8":
        w = s["Wq"].double()
        rows = []
        for x, xs in zip(s["Xq"].split(2048), s["xs"].split(2048)):
            y = torch.mm(x.double(), w.t()).mul_(xs.double()[:, None]).mul_(s["ws"].double())
            rows.append(y if s["b"] is None else y.add_(s["b"].double()))
        return torch.cat(rows)
    hd, rep = case["hd"], case["hq"] // case["hk"] if "hq" in case else 1
    if kind == "append":
        h = _signs64(hd)  # (sums of signed inputs are exact; their root comes last)
        out = {}
        for name in ("k", "v"):
            x = s[name].double()
            if name == "k" and case["rotate"]:
                x = x @ h
            peak = x.abs().max(-1, keepdim=True).values
            y = torch.round(7 * x / peak.clamp_min(1e-300)) * (peak / 7)
            out[name] = y @ h / hd if name == "k" and case["rotate"] else y
        return out
    lens = _lengths(case)
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for i, n in enumerate(lens):
        nq = case.get("nq", n)
        rows = slice(at, at + nq)
        at += nq
        visible = torch.arange(n - nq + 1, n + 1, device=DEV) if case["causal"] else torch.full((nq,), n, device=DEV)
        for j in range(case["hk"]):
            if kind == "prompt":
                k, v = s["k"][rows, j].double(), s["v"][rows, j].double()
            else:
                pages = s["table"][i, : -(-n // case["page"])].long()
                k = _signed64(s["k_codes"][pages, j].reshape(-1, hd // 2)[:n])
                v = _signed64(s["v_codes"][pages, j].permute(0, 1, 3, 2).reshape(-1, hd // 2)[:n])
                k, v = (x * s[c][pages, j].reshape(-1)[:n, None].double() for x, c in ((k, "k_scale"), (v, "v_scale")))
            for r in range(rep):
                q = s["q"][rows, j * rep + r].double()
                out[rows, j * rep + r] = _attend64(q @ _signs64(hd) / math.sqrt(hd) if case.get("rotate") else q, k, v, visible)
    return out
