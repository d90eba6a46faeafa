"""The 4-bit key/value cache: append (codes and steps against float64, bit for
bit), gather, and attention over its pages, with ragged and empty sequences,
masked and unused places that hold NaN, bad pages, splits over the length,
strides, streams and captured graphs."""
import math

import pytest
import torch

import paper_2605_28803_amd as oq
from tests import serving_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _buffers(pages, hk, d, page, seed=0):
    """Buffers that hold arbitrary codes and NaN steps."""
    g = _gen(seed + 99)
    return [torch.randint(0, 256, (pages, hk, page, d // 2), generator=g, dtype=torch.uint8),
            torch.randint(0, 256, (pages, hk, page // 16, d // 2, 16), generator=g, dtype=torch.uint8),
            torch.full((pages, hk, page), math.nan), torch.full((pages, hk, page), math.nan)]


def _cache(bufs, rotate):
    return oq.KV4Cache(*(b.to(DEV) for b in bufs), rotate_k=rotate)


def _same(cache, bufs):
    for got, want in zip((cache.k_codes, cache.v_codes), bufs[:2]):
        assert torch.equal(got.cpu(), want)
    for got, want in zip((cache.k_scale, cache.v_scale), bufs[2:]):
        # fp32 of the float64 step: one rounding here, at most two there
        torch.testing.assert_close(got.cpu(), want, rtol=2.0 ** -22, atol=0, equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("d,hk,page", [(64, 3, 16), (64, 3, 32), (128, 2, 96), (256, 1, 64), (128, 8, 256)])
def test_append_and_gather(d, hk, page, rotate, dtype):
    g = _gen(d + hk)
    pages, n = 5, 2 * page + 13
    bufs = _buffers(pages, hk, d, page)
    cache = _cache(bufs, rotate)
    k = torch.randn((n, hk, d), generator=g)
    k[:, :, 3] *= 20
    v = torch.randn((n, hk, d), generator=g) * torch.logspace(-3, 3, n)[:, None, None]
    # Rows of zeros, of one spike, of equal magnitudes, of exact ties (7 x / max = k + 1/2).
    k[0], v[0] = 0, 0
    k[1], v[1] = 0, 0
    k[1, :, 5], v[1, :, d - 1] = -2.0, 3.0
    k[2], v[2] = 1.5, -0.25
    v[3] = (torch.arange(d) % 15 - 7).float()[None] * 0.5
    v[3, :, 0] = 7.0
    k[3] = v[3]
    k, v = k.to(dtype), v.to(dtype)
    slots = torch.randperm(pages * page, generator=g)[:n]
    slots[7], slots[11] = -1, pages * page  # skipped
    wide = torch.randn((n, 2 * hk, d), generator=g).to(dtype).to(DEV)  # strided rows
    wide[:, :hk] = k.to(DEV)
    oq.kv4_append(cache, wide[:, :hk], v.to(DEV), slots.to(DEV))
    torch.cuda.synchronize()
    R.put(bufs, slots, k, v, rotate)
    _same(cache, bufs)
    # Gather, in every type; slots out of range give zeros.
    for out, dt in ((oq.OUT_F32, torch.float32), (oq.OUT_F16, torch.float16), (oq.OUT_BF16, torch.bfloat16)):
        K = torch.full((n, 2 * hk, d), 9.0, dtype=dt, device=DEV)
        gk, gv = oq.kv4_gather(cache, slots.to(DEV), out, K=K[:, hk:])
        torch.cuda.synchronize()
        assert (K[:, :hk] == 9.0).all()
        bad = (slots < 0) | (slots >= pages * page)
        want_k, want_v = R.take(bufs, slots.clamp(0, pages * page - 1), d, rotate)
        want_k[bad], want_v[bad] = 0, 0
        size_k = want_k.abs()
        if rotate:
            # The sum of codes is exact: the step's rounding, its product with 1 / sqrt(d), the product.
            want_k = want_k @ R.hadamard(d) / math.sqrt(d)
            size_k = want_k.abs()
        u = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dt]
        tiny = 2.0 ** -25 if dt == torch.float16 else 0.0
        scale = 2.0 ** -24
        # (sums of up to d float64 products differ from the exact sum of codes)
        assert ((gk.cpu().double() - want_k).abs() <= (u + 5 * scale) * size_k + tiny + 1e-12 * want_k.abs().max()).all()
        if dt == torch.float16:
            want_v = want_v.clamp(-65504, 65504)
        assert ((gv.cpu().double() - want_v).abs() <= (u + 2 * scale) * want_v.abs() + tiny).all()


def test_append_one_token_leaves_its_neighbours():
    for t in (0, 1, 15, 16, 31):
        bufs = _buffers(2, 2, 128, 32, seed=t)
        cache = _cache(bufs, True)
        k, v = torch.randn((2, 1, 2, 128), generator=_gen(t)).half()
        s = torch.tensor([32 + t])
        oq.kv4_append(cache, k.to(DEV), v.to(DEV), s.to(DEV))
        torch.cuda.synchronize()
        R.put(bufs, s, k, v, True)
        _same(cache, bufs)


def test_append_extreme_magnitudes():
    # The largest and smallest finite values of both types.
    for dtype in (torch.float16, torch.bfloat16):
        f = torch.finfo(dtype)
        small = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -133
        v = torch.tensor([f.max, -f.max, f.max / 2, f.tiny, small, -small, 0.0, f.max / 3]).to(dtype).repeat(8)[None, None]
        w = torch.tensor([small, -small, 3 * small, 7 * small, 2 * small, 0, 4 * small, 5 * small]).to(dtype).repeat(8)[None, None]
        x = torch.cat((v, w))
        bufs = _buffers(1, 1, 64, 32)
        cache = _cache(bufs, False)
        s = torch.tensor([0, 1])
        oq.kv4_append(cache, x.to(DEV), x.to(DEV), s.to(DEV))
        torch.cuda.synchronize()
        R.put(bufs, s, x, x, False)
        assert torch.equal(cache.k_codes.cpu()[:, :, :2], bufs[0][:, :, :2])
        # (a step below fp32's normal numbers is off by at most its smallest one)
        assert ((cache.k_scale.cpu()[0, 0, :2].double() - bufs[2][0, 0, :2].double()).abs()
                <= 2.0 ** -22 * bufs[2][0, 0, :2].abs() + 2.0 ** -149).all()


def _attention(lens, nqs, hq, hk, d, page, rotate, causal, dtype, max_len=None, cu=True, bad=(), seed=0, vscale=None,
               lead=0, tail=0, scale=None, zero=()):
    """One call against float64.  nqs: query tokens of each sequence; bad: (sequence, page index, entry)."""
    g = _gen(seed + sum(lens) + d)
    n = len(lens)
    top = max(lens) if max_len is None else max_len
    width = max(1, -(-top // page)) + 1
    pages = sum(-(-x // page) for x in lens) + 2
    order = torch.randperm(pages, generator=g)
    table = torch.randint(-2 ** 31, 2 ** 31 - 1, (n, width), generator=g).to(torch.int32)  # unused entries hold anything
    bufs = _buffers(pages, hk, d, page, seed)
    at, there = 0, []
    for i, L in enumerate(lens):
        m = -(-L // page)
        table[i, :m] = order[at:at + m].to(torch.int32)
        at += m
        pos = torch.arange(L)
        slots = table[i, :m].long().repeat_interleave(page)[:L] * page + pos % page
        k = torch.randn((L, hk, d), generator=g).to(dtype)
        v = torch.randn((L, hk, d), generator=g)
        if vscale is not None:
            v = v * torch.exp(torch.empty((L, 1, 1)).uniform_(-vscale, vscale, generator=g))
        v = v.to(dtype)
        for z in zero:
            if z < L:
                v[z] = 0
        R.put(bufs, slots, k, v, rotate)
        there.append(slots)
    for i, j, e in bad:
        table[i, j] = e
    T = lead + sum(nqs) + tail
    q = torch.randn((T, hq + 1, d), generator=g).to(dtype)  # strided
    O = torch.full((T, hq, d), 3.0, dtype=dtype, device=DEV)
    cu_q = torch.tensor([lead] + [lead + sum(nqs[:i + 1]) for i in range(n)], dtype=torch.int32)
    cache = _cache(bufs, rotate)
    oq.attention_kv4(q.to(DEV)[:, :hq], cache, table.to(DEV), torch.tensor(lens, dtype=torch.int32).to(DEV),
                     cu_q.to(DEV) if cu else None, max_q=max(nqs) if cu else None, max_len=top, causal=causal, scale=scale, O=O)
    torch.cuda.synchronize()
    got = O.cpu()
    assert (got[:lead] == 3.0).all() and (tail == 0 or (got[T - tail:] == 3.0).all())
    s = d ** -0.5 if scale is None else scale
    at = lead
    for i, (L, nq) in enumerate(zip(lens, nqs)):
        k, v = R.take(bufs, there[i], d, rotate)
        ok = torch.ones(L, dtype=torch.bool)
        for bi, j, _ in bad:
            if bi == i:
                ok[j * page:(j + 1) * page] = False
        k, v = torch.where(ok[:, None, None], k, 0.0), torch.where(ok[:, None, None], v, 0.0)
        see = torch.arange(L)[None, :] <= (L - nq + torch.arange(nq) if causal else torch.full((nq,), L))[:, None]
        see = see & ok[None, :]
        for h in range(hq):
            qq = q[at:at + nq, h].double()
            if rotate:
                qq = qq @ R.hadamard(d) / math.sqrt(d)
            kk, vv = k[:, h // (hq // hk)], v[:, h // (hq // hk)]
            o, spread, p = R.attend(qq, kk, vv, s, see)
            extra = 2 * R.score_error(qq, kk, s)
            if L and nq:
                # The accumulator starts at 72 sum(q) in units of the step; a rotated query is
                # rounded in fp32 (log2 d sums) and to 22 bits, each against its row's sum.
                one = (qq.abs().sum(-1)).max().item() * s
                step = kk.abs().max().item() / 7 if kk.numel() else 0.0
                extra += 2 * one * step * (80 * (d + 8) * 2.0 ** -24 + 7 * 12 * 2.0 ** -22)
                # Probabilities below 2^-14 of the largest contribution lose up to 2^-25 of it each.
                spread = spread + L * 7 * 2.0 ** -25 / 2 ** -10 * 0.5 * (p[:, :, None] * vv.abs()[None]).amax((1, 2))[:, None]
            R.check(got[at:at + nq, h], o, spread, extra, dtype, 2.0 ** -11)
        at += nq


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("d,hq,hk,page", [(64, 4, 4, 16), (64, 12, 2, 48), (128, 8, 2, 64), (256, 8, 1, 96), (128, 15, 3, 128)])
def test_one_token_each(d, hq, hk, page, rotate, dtype):
    lens = [1, 0, 33, 127, 128, 129, 300, 2]
    _attention(lens, [1] * len(lens), hq, hk, d, page, rotate, True, dtype, cu=False)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,hq,hk", [(64, 3, 3), (128, 8, 2), (256, 5, 1)])
def test_several_tokens(d, hq, hk, causal):
    # ... among them more query tokens than cached ones: the first see nothing and give zeros.
    _attention([40, 200, 3, 0, 129], [5, 17, 8, 2, 0], hq, hk, d, 32, True, causal, torch.float16, lead=2, tail=3)


def test_many_rows():
    _attention([300, 70], [130, 70], 8, 1, 128, 64, False, True, torch.bfloat16)
    _attention([260], [50], 8, 8, 128, 32, False, False, torch.float16)


@pytest.mark.parametrize("n", [511, 512, 513, 1500, 6000])
def test_split_over_the_length(n):
    _attention([n], [1], 4, 1, 128, 64, False, True, torch.float16, cu=False)
    _attention([n, 5, 700], [2, 2, 2], 8, 2, 64, 128, True, True, torch.bfloat16, max_len=7000, tail=4)
    _attention([n], [1], 8, 1, 256, 64, True, True, torch.bfloat16, cu=False)


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("lens,nqs,hq,hk,d", [
    ([900, 20], [20, 2], 8, 2, 128),                       # 32 rows, shortest chunks
    ([3000, 500, 0, 1], [20, 20, 3, 1], 8, 2, 128),        # 32 rows, eight waves, splits of several steps
    ([3000, 700, 64], [40, 5, 64], 8, 4, 64),
    ([900, 1000, 513], [1, 1, 1], 16, 1, 64),              # whole sequences of several steps
    ([600 + 20 * i for i in range(17)], [1] * 17, 8, 8, 128),
    ([1500, 300, 90] * 9, [1] * 27, 10, 10, 64),           # splits that only the long ones have
])
def test_shapes_of_the_split(lens, nqs, hq, hk, d, rotate):
    _attention(lens, nqs, hq, hk, d, 64, rotate, True, torch.float16)


def test_bad_pages_are_masked():
    _attention([200, 150], [1, 1], 4, 2, 128, 32, False, True, torch.float16, cu=False,
               bad=[(0, 0, -1), (0, 3, 2 ** 31 - 1), (1, 4, 1000)])
    _attention([64], [2], 4, 2, 64, 32, False, True, torch.float16, bad=[(0, 0, -7), (0, 1, 99)])  # nothing is left


def test_steps_of_any_size():
    # Values whose steps span e^16, rows of zero values among them.
    _attention([700], [3], 4, 2, 128, 64, False, True, torch.bfloat16, vscale=8.0, zero=(0, 5, 600))
    _attention([100], [1], 2, 2, 64, 32, True, True, torch.float16, vscale=5.0, cu=False, zero=range(100))


def test_large_scores():
    _attention([500], [4], 4, 2, 128, 64, True, True, torch.float16, scale=1.0)


def test_sharp_maximum_in_a_small_value():
    # The most likely token has a tiny value: it counts in the sum, not in the product.
    bufs = _buffers(1, 1, 64, 64)
    k, v = torch.zeros((2, 64, 1, 64), dtype=torch.float16)
    k[:, 0, 0] = 1.0
    k[0, 0, 0] = 9.0
    v[:] = 2.0
    v[0] = 2.0 ** -20
    R.put(bufs, torch.arange(64), k, v, False)
    q = torch.zeros((1, 1, 64), dtype=torch.float16)
    q[0, 0, 0] = 8.0
    o = oq.attention_kv4(q.to(DEV), _cache(bufs, False), torch.zeros((1, 1), dtype=torch.int32, device=DEV),
                         torch.tensor([64], dtype=torch.int32, device=DEV), scale=0.125)
    kk, vv = R.take(bufs, torch.arange(64), 64, False)
    ref, spread, p = R.attend(q[:, 0].double(), kk[:, 0], vv[:, 0], 0.125, torch.ones((1, 64), dtype=torch.bool))
    R.check(o.cpu()[:, 0], ref, spread, 2.0 ** -18, torch.float16, 2.0 ** -11)


def _tail(L, below, dtype):
    """One token with a value in one channel only, the others below it by `below`
    in the exponent, with values in every channel: in all channels but one the
    output is the small probabilities' alone."""
    bufs = _buffers(L // 64, 1, 64, 64)
    k, v = torch.zeros((2, L, 1, 64), dtype=dtype)
    k[5, 0, 0] = 7.0
    v[:] = 7.0
    v[5], v[5, 0, 0] = 0.0, 7.0
    order = torch.arange(L)
    R.put(bufs, order, k, v, False)
    q = torch.zeros((1, 1, 64), dtype=dtype)
    q[0, 0, 0] = 1.0
    scale = below / 7.0
    o = oq.attention_kv4(q.to(DEV), _cache(bufs, False), torch.arange(L // 64, dtype=torch.int32, device=DEV)[None],
                         torch.tensor([L], dtype=torch.int32, device=DEV), scale=scale)
    kk, vv = R.take(bufs, order, 64, False)
    ref, spread, _ = R.attend(q[:, 0].double(), kk[:, 0], vv[:, 0], scale, torch.ones((1, L), dtype=torch.bool))
    # (the scores are below 32, so their fp32 errors, of a few steps of 2^-19, are below 2^-16)
    R.check(o.cpu()[:, 0], ref, spread, 2.0 ** -15, dtype, 2.0 ** -11)


@pytest.mark.parametrize("L,below", [(4096, 10.0), (65536, 17.7), (131072, 18.5)])
def test_many_small_probabilities(L, below):
    # e^-10, e^-17.7 and e^-18.5: below fp16's normal numbers, and below half its smallest one.
    _tail(L, below, torch.float16)
    _tail(L, below, torch.bfloat16)


def _small(seed=0, n=3000):
    g = torch.Generator(device=DEV).manual_seed(seed)
    cache = oq.KV4Cache.empty(n // 64 + 1, 2, 128, 64)
    k, v = torch.randn((2, n, 2, 128), device=DEV, generator=g).half()
    slots = torch.arange(n, device=DEV)
    oq.kv4_append(cache, k, v, slots)
    table = torch.arange(n // 64 + 1, dtype=torch.int32, device=DEV)[None]
    return cache, table, torch.tensor([n], dtype=torch.int32, device=DEV), torch.randn((1, 8, 128), device=DEV, generator=g).half()


def test_streams_and_repeats():
    cache, table, lens, q = _small()
    want = oq.attention_kv4(q, cache, table, lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = oq.attention_kv4(q, cache, table, lens)
    b = oq.attention_kv4(q, cache, table, lens)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)


def test_workspace_belongs_to_the_call_s_stream():
    """A workspace made inside a call on another stream is not handed out again
    on the current one while that call still waits."""
    cache, table, lens, q = _small()
    want = oq.attention_kv4(q, cache, table, lens)
    nbytes = oq.attention_kv4_workspace_bytes(cache, 1, 8, 1, 1, table.shape[1] * 64)
    assert nbytes > 0
    O = torch.empty_like(q)
    a = torch.randn((4096, 4096), device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(20):
            a = (a @ a).clamp(-1, 1)  # (the stream is busy for some time)
    oq.attention_kv4(q, cache, table, lens, O=O, stream=s)
    x = [torch.full((nbytes,), 7, dtype=torch.uint8, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(O, want)
    assert all((t == 7).all() for t in x)


def test_captured_step():
    """A decoding step (append, attend) captured once and replayed while the
    sequence grows; two graphs may share a workspace when they do not overlap."""
    cache, table, lens, q = _small()
    eager, _, _, _ = _small()
    k, v = torch.randn((2, 1, 2, 128), device=DEV).half()
    slot = lens.long()
    cap = table.shape[1] * 64
    work = torch.empty((max(16, oq.attention_kv4_workspace_bytes(cache, 1, 8, 1, 1, cap)),), dtype=torch.uint8, device=DEV)
    O = [torch.empty_like(q), torch.empty_like(q)]

    def step(c, o):
        oq.kv4_append(c, k, v, slot)
        oq.attention_kv4(q, c, table, lens, O=o, work=work, max_len=cap)

    step(cache, O[0])
    torch.cuda.synchronize()
    graphs = []
    for o in O:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(cache, o)
        graphs.append(gr)
    for i in range(4):
        g = torch.Generator(device=DEV).manual_seed(50 + i)
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, device=DEV, generator=g))
        slot.fill_(3000 + i)
        lens.fill_(3001 + i)
        oq.kv4_append(eager, k, v, slot)
        want = oq.attention_kv4(q, eager, table, lens, max_len=cap)
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(O[0], want) and torch.equal(O[1], want)


def test_lengths_past_max_len_are_clamped():
    cache, table, lens, q = _small()
    a = oq.attention_kv4(q, cache, table, lens, max_len=1000)
    b = oq.attention_kv4(q, cache, table, torch.full_like(lens, 1000))
    torch.cuda.synchronize()
    # The same keys; other splits may sum in another order.
    assert torch.isfinite(a).all()
    torch.testing.assert_close(a, b, rtol=2.0 ** -10, atol=2.0 ** -12)
    c = oq.attention_kv4(q, cache, table, torch.full_like(lens, -4))
    assert (c == 0).all()


def test_query_tokens_past_max_q_are_left():
    """max_q below a sequence's query tokens: the first max_q are what they are without it."""
    for n in (900, 3000):
        cache, table, lens, _ = _small(n=n)
        q = torch.randn((9, 8, 128), device=DEV, generator=torch.Generator(device=DEV).manual_seed(7)).half()
        cu = torch.tensor([1, 8], dtype=torch.int32, device=DEV)
        full = oq.attention_kv4(q, cache, table, lens, cu, max_q=7, max_len=n)
        O = torch.full_like(q, 3.0)
        oq.attention_kv4(q, cache, table, lens, cu, max_q=4, max_len=n, O=O)
        torch.cuda.synchronize()
        torch.testing.assert_close(O[1:5], full[1:5], rtol=2.0 ** -9, atol=2.0 ** -11)  # (other splits)
        assert (O[5:] == 3.0).all() and (O[0] == 3.0).all()


def test_empty_cache_and_no_table():
    cache = oq.KV4Cache.empty(1, 2, 64, 16)
    q = torch.randn((3, 4, 64), device=DEV).half()
    o = oq.attention_kv4(q, cache, torch.zeros((3, 0), dtype=torch.int32, device=DEV), torch.tensor([0, 5, -1], dtype=torch.int32, device=DEV))
    assert (o == 0).all()


def test_nothing_to_do():
    cache, table, lens, q = _small()
    e = q[:0]
    assert oq.attention_kv4(e, cache, table[:0], lens[:0]).shape == (0, 8, 128)
    oq.kv4_append(cache, q[:0, :2], q[:0, :2], torch.zeros(0, dtype=torch.int64, device=DEV))
    k, v = oq.kv4_gather(cache, torch.zeros(0, dtype=torch.int64, device=DEV))
    assert k.shape == (0, 2, 128)
