"""Refusals of the serving operators, without a GPU: the C entry points before
they touch the device, the binding's checks of shapes, types and devices, and
the plain references that the GPU tests use."""
import ctypes as C
import math

import pytest
import torch

import paper_2605_28803_amd as oq
from paper_2605_28803_amd import _lib
from tests import serving_ref as R

OK, NULL, SHAPE, ALIGN, DEVICE, HIP, WORKSPACE, ARG = 0, -1, -2, -3, -4, -5, -6, -7
P16, P4, P2 = C.c_void_p(0x10000), C.c_void_p(0x10004), C.c_void_p(0x10002)  # never dereferenced on error paths


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def _c(**kw):
    f = dict(k_codes=0x10000, v_codes=0x10000, k_scale=0x10000, v_scale=0x10000, n_pages=4, page_tokens=64, n_kv_heads=2,
             head_dim=128, rotate_k=1)
    f.update(kw)
    return C.byref(_lib.oq_kv4_cache(**f))


BAD_CACHES = [(dict(k_codes=None), NULL), (dict(v_scale=None), NULL), (dict(head_dim=96), SHAPE), (dict(head_dim=0), SHAPE),
              (dict(n_pages=0), SHAPE), (dict(n_pages=2 ** 31), SHAPE), (dict(page_tokens=8), SHAPE), (dict(page_tokens=56), SHAPE),
              (dict(page_tokens=65552), SHAPE), (dict(n_pages=2 ** 30, page_tokens=65536), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_kv_heads=65536), SHAPE),
              (dict(k_codes=0x10004), ALIGN), (dict(k_scale=0x10008), ALIGN), (dict(rotate_k=2), ARG)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_bad_caches(lib, change, status):
    c = _c(**change)
    assert lib.oq_kv4_append(c, P16, P16, 4, 256, 256, 0, P16, None) == status
    assert lib.oq_kv4_gather(c, P16, 4, P16, P16, 256, 256, 0, None) == status
    assert lib.oq_attention_kv4(c, P16, 4, 1024, 8, 0, None, 1, P16, 8, P16, 4, 100, 1, 0.1, P16, 1024, P16, 1 << 30,
                                None) == status


def test_no_cache(lib):
    assert lib.oq_kv4_append(None, P16, P16, 4, 256, 256, 0, P16, None) == NULL
    assert lib.oq_attention_kv4_workspace_bytes(None, 1, 8, 1, 1, 100) == 0


def test_append_and_gather_refusals(lib):
    def both(n, ldk, ldv, dtype, K, V, slots):
        return (lib.oq_kv4_append(_c(), K, V, n, ldk, ldv, dtype, slots, None),
                lib.oq_kv4_gather(_c(), slots, n, K, V, ldk, ldv, dtype, None))
    assert both(-1, 256, 256, 0, P16, P16, P16) == (SHAPE, SHAPE)
    assert both(4, 248, 256, 0, P16, P16, P16) == (SHAPE, SHAPE)
    assert both(4, 256, 255, 0, P16, P16, P16) == (SHAPE, SHAPE)
    assert both(4, 260, 256, 0, P16, P16, P16) == (ALIGN, ALIGN)
    assert both(4, 256, 256, 5, P16, P16, P16) == (ARG, ARG)
    assert both(4, 256, 256, 0, None, P16, P16) == (NULL, NULL)
    assert both(4, 256, 256, 0, P16, None, P16) == (NULL, NULL)
    assert both(4, 256, 256, 0, P16, P16, None) == (NULL, NULL)
    assert both(4, 256, 256, 0, P4, P16, P16) == (ALIGN, ALIGN)
    assert both(4, 256, 256, 0, P16, P16, P4) == (ALIGN, ALIGN)
    assert both(0, 256, 256, 0, None, None, None) == (OK, OK)
    assert lib.oq_kv4_append(_c(), P16, P16, 4, 256, 256, 2, P16, None) == ARG  # fp32 is for gather only


def _attend(lib, cache=None, Q=P16, tokens=4, ldq=1024, heads=8, dtype=0, cu=None, max_q=1, table=P16, table_ld=8, lens=P16, n=4,
            max_len=100, causal=1, scale=0.1, O=P16, ldo=1024, work=P16, nbytes=1 << 30):
    return lib.oq_attention_kv4(cache or _c(), Q, tokens, ldq, heads, dtype, cu, max_q, table, table_ld, lens, n, max_len, causal,
                                scale, O, ldo, work, nbytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(Q=None), NULL), (dict(O=None), NULL), (dict(lens=None), NULL), (dict(table=None), NULL),
    (dict(Q=P4), ALIGN), (dict(O=P4), ALIGN), (dict(work=P4), ALIGN), (dict(lens=P2), ALIGN), (dict(table=P2), ALIGN),
    (dict(cu=P2), ALIGN), (dict(ldq=1028), ALIGN), (dict(ldo=1028), ALIGN),
    (dict(tokens=-1), SHAPE), (dict(tokens=5), SHAPE), (dict(max_q=2), SHAPE), (dict(max_q=0), SHAPE), (dict(max_q=65536, cu=P16), SHAPE), (dict(heads=7), SHAPE),
    (dict(heads=0), SHAPE), (dict(n=-1), SHAPE), (dict(n=40000, tokens=40000), SHAPE), (dict(max_len=-1), SHAPE),
    (dict(max_len=513), SHAPE), (dict(max_len=2 ** 30 + 1, table_ld=2 ** 40), SHAPE), (dict(table_ld=-1), SHAPE), (dict(ldq=1016), SHAPE), (dict(ldo=8), SHAPE),
    (dict(dtype=2), ARG), (dict(dtype=-1), ARG), (dict(causal=2), ARG), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG),
    (dict(scale=math.inf), ARG), (dict(scale=math.nan), ARG),
    (dict(cu=P16, tokens=2 ** 31), SHAPE), (dict(heads=65536, ldq=2 ** 23, ldo=2 ** 23), SHAPE),
    (dict(cu=P16, max_q=65535, heads=2050, ldq=2 ** 20, ldo=2 ** 20), SHAPE), (dict(scale=3e38), ARG),
])
def test_attention_kv4_refusals(lib, change, status):
    assert _attend(lib, **change) == status


def test_attention_kv4_workspace(lib):
    c = _c(n_pages=4096)
    need = lib.oq_attention_kv4_workspace_bytes(c, 1, 8, 1, 1, 100000)
    assert need > 0
    big = dict(cache=c, tokens=1, n=1, max_len=100000, table_ld=2000)
    assert _attend(lib, **big, work=None, nbytes=0) == WORKSPACE
    assert _attend(lib, **big, nbytes=need - 1) == WORKSPACE
    # one split needs none
    assert lib.oq_attention_kv4_workspace_bytes(c, 1, 8, 1, 1, 64) == 0
    assert lib.oq_attention_kv4_workspace_bytes(c, 1, 7, 1, 1, 100000) == 0  # (a shape that the call refuses)


def test_nothing_to_attend(lib):
    assert _attend(lib, n=0, tokens=0, Q=None, O=None, lens=None) == OK


def _prompt(lib, Q=P16, K=P16, V=P16, tokens=4, ldq=1024, ldk=256, ldv=256, dtype=0, cu=P16, n=1, hq=8, hk=2, d=128, causal=1,
            scale=0.1, O=P16, ldo=1024):
    return lib.oq_attention_prompt(Q, K, V, tokens, ldq, ldk, ldv, dtype, cu, n, hq, hk, d, causal, scale, O, ldo, None)


@pytest.mark.parametrize("change,status", [
    (dict(Q=None), NULL), (dict(K=None), NULL), (dict(V=None), NULL), (dict(O=None), NULL), (dict(cu=None), NULL),
    (dict(Q=P4), ALIGN), (dict(K=P4), ALIGN), (dict(V=P4), ALIGN), (dict(O=P4), ALIGN), (dict(cu=P2), ALIGN),
    (dict(ldq=1028), ALIGN), (dict(ldk=260), ALIGN), (dict(ldv=260), ALIGN), (dict(ldo=1028), ALIGN),
    (dict(ldq=1016), SHAPE), (dict(ldk=248), SHAPE), (dict(ldv=248), SHAPE), (dict(ldo=1016), SHAPE), (dict(ldk=2 ** 25), SHAPE),
    (dict(tokens=-1), SHAPE), (dict(tokens=2 ** 31), SHAPE), (dict(n=-1), SHAPE), (dict(d=48), SHAPE), (dict(hq=7), SHAPE),
    (dict(hk=0), SHAPE), (dict(hq=0), SHAPE), (dict(dtype=2), ARG), (dict(causal=-1), ARG), (dict(scale=0.0), ARG),
    (dict(scale=math.nan), ARG), (dict(scale=3e38), ARG), (dict(tokens=0, Q=None), OK), (dict(n=0, cu=None), OK),
])
def test_attention_prompt_refusals(lib, change, status):
    assert _prompt(lib, **change) == status


def test_w8a8_refusals(lib):
    g = lib.oq_w8a8_linear
    assert g(None, P16, 4, P16, P16, None, 64, 64, P16, 64, 0, None) == NULL
    assert g(P16, None, 4, P16, P16, None, 64, 64, P16, 64, 0, None) == NULL
    assert g(P16, P16, 4, P16, None, None, 64, 64, P16, 64, 0, None) == NULL
    assert g(P16, P16, 4, P16, P16, None, 64, 96, P16, 64, 0, None) == SHAPE
    assert g(P16, P16, 4, P16, P16, None, 64, 16448, P16, 64, 0, None) == SHAPE
    assert g(P16, P16, 4, P16, P16, None, 64, 64, P16, 32, 0, None) == SHAPE
    assert g(P4, P16, 4, P16, P16, None, 64, 64, P16, 64, 0, None) == ALIGN
    assert g(P16, P16, 4, P4, P16, None, 64, 64, P16, 64, 0, None) == ALIGN
    assert g(P16, P16, 4, P16, P16, None, 64, 64, P16, 68, 0, None) == ALIGN
    assert g(P16, P16, 4, P16, P16, None, 64, 64, P16, 64, 2, None) == ARG
    assert g(None, None, 0, None, None, None, 64, 64, None, 64, 0, None) == OK
    h = lib.oq_w8a8_gemm_i32
    assert h(P16, 4, None, 64, 64, P16, 64, None) == NULL
    assert h(P16, 4, P16, 64, 64, P16, 66, None) == ALIGN
    assert lib.oq_quantize_weights_i8(None, 4, 64, 64, 64, P16, P16, None) == NULL
    assert lib.oq_quantize_weights_i8(P16, 4, 96, 96, 64, P16, P16, None) == SHAPE


def test_binding_refusals():
    h = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    cu = torch.zeros(2, dtype=torch.int32)
    q, k = h(4, 8, 128), h(4, 2, 128)
    with pytest.raises(ValueError, match="one GPU"):
        oq.attention_prompt(q, k, k, cu)
    with pytest.raises(ValueError, match="side by side"):
        oq.attention_prompt(h(4, 128, 8).transpose(1, 2), k, k, cu)
    with pytest.raises(ValueError, match="heads, head_dim"):
        oq.attention_prompt(q, h(4, 2, 64), k, cu)
    c = oq.KV4Cache.empty(2, 2, 128, device="cpu")
    with pytest.raises(ValueError, match="one GPU"):
        oq.kv4_append(c, k, k, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="one GPU"):
        oq.kv4_gather(c, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="one GPU"):
        oq.attention_kv4(q, c, torch.zeros((4, 1), dtype=torch.int32), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="v_codes"):
        oq.KV4Cache(c.k_codes, c.k_codes, c.k_scale, c.v_scale)
    with pytest.raises(ValueError, match="k_scale"):
        oq.KV4Cache(c.k_codes, c.v_codes, c.k_scale.double(), c.v_scale)
    i8 = torch.zeros((4, 64), dtype=torch.int8)
    with pytest.raises(ValueError, match="int8"):
        oq.w8a8_linear(i8, torch.ones(4), torch.zeros((8, 32), dtype=torch.uint8), torch.ones(8))
    w8 = torch.zeros((8, 64), dtype=torch.int8)
    for bad, what in (((i8.t().contiguous().t(), torch.ones(4), w8, torch.ones(8)), "int8"),
                      ((i8, torch.ones(3), w8, torch.ones(8)), "x_scale"), ((i8, torch.ones(4), w8, torch.ones(9)), "w_scale"),
                      ((i8, torch.ones(4).half(), w8, torch.ones(8)), "x_scale"),
                      ((i8, torch.ones(4), w8, torch.ones(8), torch.zeros(8)), "bias"),
                      ((i8, torch.ones(4), w8, torch.ones(8), None, oq.OUT_F16, torch.zeros((4, 8))), "Y")):
        with pytest.raises(ValueError, match=what):
            oq.w8a8_linear(*bad)
    for bad, what in (((i8, torch.ones(8)[::2], w8, torch.ones(8)), "x_scale"),
                      ((i8, torch.ones(4), w8, torch.ones(8), torch.zeros(16).half()[::2]), "bias"),
                      ((i8, torch.ones(4), w8, torch.ones(8)), "one GPU")):
        with pytest.raises(ValueError, match=what):
            oq.w8a8_linear(*bad)
    with pytest.raises(ValueError, match="one GPU"):
        oq.w8a8_gemm_i32(i8, w8)
    for bad, what in (((h(8, 64).float(), 64), "W_u"), ((h(64, 8).t(), 64), "W_u"), ((h(8, 64), 64, w8[:4]), "Wq8"),
                      ((h(8, 64), 64, w8, torch.ones(4)), "w_scale"), ((h(8, 64), 64, w8, torch.ones(8)), "one GPU")):
        with pytest.raises(ValueError, match=what):
            oq.quantize_weights_i8(*bad)
    with pytest.raises(ValueError, match="acc"):
        oq.w8a8_gemm_i32(i8, w8, torch.zeros((4, 9), dtype=torch.int32))


@pytest.mark.parametrize("cache", [dict(n_kv_heads=1, head_dim=64), dict(n_kv_heads=8, head_dim=128), dict(n_kv_heads=2, head_dim=256)])
def test_workspace_holds_every_split(lib, cache):
    """At most 64 splits of at least 256 tokens, for any plan of the sizes allowed."""
    c = _c(n_pages=2 ** 20, **cache)
    hk = cache["n_kv_heads"]
    for n_seqs in (1, 7, 65535 // hk):
        for max_q in (1, 50, 65535):
            for max_len in (1, 512, 513, 131000, 2 ** 30):
                row = 8 * hk * (cache["head_dim"] + 4) * 4
                size = lib.oq_attention_kv4_workspace_bytes(c, 3, 8 * hk, n_seqs, max_q, max_len)
                assert size % (3 * row) == 0 and size // (3 * row) <= min(65, -(-max_len // 256))


def test_plain_cache_by_hand():
    """The reference's layout and codes on numbers worked by hand."""
    x = torch.tensor([[7.0, -3.5, 0.5, 1.5] + [0.0] * 60])      # 7 x / 7: 7, -3.5 -> -4, 0.5 -> 0, 1.5 -> 2
    q, step = R.codes(x.double(), False)
    assert q[0, :5].tolist() == [7, -4, 0, 2, 0] and step.item() == 1.0
    p = R.pack(q)
    assert p[0, :3].tolist() == [7 | 12 << 4, 0 | 2 << 4, 0]
    assert torch.equal(R.unpack(p), q)
    bufs = [torch.zeros((2, 1, 32, 32), dtype=torch.uint8), torch.zeros((2, 1, 2, 32, 16), dtype=torch.uint8),
            torch.zeros((2, 1, 32)), torch.zeros((2, 1, 32))]
    R.put(bufs, torch.tensor([32 + 17]), x[:, None], x[:, None], False)
    assert bufs[0][1, 0, 17, 0] == 7 | 12 << 4 and bufs[1][1, 0, 1, 1, 1] == 2 << 4 and bufs[3][1, 0, 17] == 1.0
    # Rotation: H_64 of one spike has equal magnitudes.
    q, step = R.codes(torch.eye(64, dtype=torch.float64)[:1] * 8, True)
    assert (q.abs() == 7).all() and abs(step.item() - 1 / 7) < 1e-15
    # Attention of one query over two keys: weights 1/4 and 3/4.
    o, spread, w = R.attend(torch.tensor([[math.log(3.0)]], dtype=torch.float64), torch.tensor([[0.0], [1.0]]).double(),
                            torch.tensor([[4.0], [-8.0]]).double(), 1.0, torch.ones((1, 2), dtype=torch.bool))
    assert abs(o.item() + 5) < 1e-12 and abs(spread.item() - 7) < 1e-12 and abs(w[0, 0].item() - 0.25) < 1e-12
