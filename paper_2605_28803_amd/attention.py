"""Attention over packed prompts and the 4-bit key/value cache (binding of
oq_attention_prompt, oq_kv4_* and oq_attention_kv4 in include/oq.h).

Marshalling only.  Shapes, types and devices are checked here, because the C
entry points see pointers alone.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import _check, _current_device, _empty, _lib, _on, _ptr  # (the package has these before it imports this module)

_DTYPE = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_TORCH = {0: torch.float16, 1: torch.bfloat16, 2: torch.float32}


def _want(ok, what):
    if not ok:
        raise ValueError(what)


# The host's time bounds the smallest calls, so the checks below ask a tensor as little as they can.

def _heads(t, name, head_dim):
    """Token stride of a [tokens, heads, head_dim] tensor whose heads of a token
    lie side by side."""
    if t.dim() == 3:
        n, h, d = t.shape
        s0, s1, s2 = t.stride()
        if d == head_dim:
            if s2 == 1 and (s1 == d or h <= 1):
                return s0 if n > 1 else h * d
            raise ValueError(f"{name}: the heads of a token must lie side by side")
    raise ValueError(f"{name}: [tokens, heads, head_dim] expected")


def _ints(t, name, dtype, n, dev):
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name}: contiguous {dtype} of {n} elements on cuda:{dev} expected")


def _device(t, u, v):
    """Index of the tensors' device, which has to be the current one (the library
    launches there)."""
    dev = t.get_device()
    if dev < 0 or u.get_device() != dev or v.get_device() != dev:
        raise ValueError("the tensors must be on one GPU")
    if dev != _current_device():
        raise ValueError(f"cuda:{dev} is not the current device")
    return dev


def attention_prompt(Q, K, V, cu_seqlens, causal=True, scale=None, O=None, stream=None):
    """O [T, Hq, d] = softmax(scale Q K^T) V within each packed sequence.
    Q [T, Hq, d], K, V [T, Hkv, d] fp16 or bf16 (views of a q|k|v output serve),
    cu_seqlens int32 [n + 1] on the device; scale defaults to d ** -0.5.  Rows of
    no sequence are left as they were in O (unspecified when O is made here)."""
    _want(Q.dim() == 3, "Q: [tokens, heads, head_dim] expected")
    T, hq, d = Q.shape
    ldq, ldk, ldv = _heads(Q, "Q", d), _heads(K, "K", d), _heads(V, "V", d)
    dev = _device(Q, K, V)
    _want(K.shape[0] == T and V.shape == K.shape, "K and V need Q's tokens and equal shapes")
    _want(Q.dtype in _DTYPE and K.dtype == Q.dtype and V.dtype == Q.dtype, "Q, K and V need one type")
    n_cu = cu_seqlens.numel()
    _want(n_cu >= 1, "cu_seqlens: at least one element expected")
    _ints(cu_seqlens, "cu_seqlens", torch.int32, n_cu, dev)
    if O is None:
        O, ldo = _empty(Q, (T, hq, d), Q.dtype, stream), hq * d
    else:
        _want(O.shape == Q.shape and O.dtype == Q.dtype and O.get_device() == dev, "O: Q's shape, type and device expected")
        ldo = _heads(O, "O", d)
    _check(_lib.load().oq_attention_prompt(_ptr(Q), _ptr(K), _ptr(V), T, ldq, ldk, ldv, _DTYPE[Q.dtype], _ptr(cu_seqlens),
                                           n_cu - 1, hq, K.shape[1], d, int(causal),
                                           d ** -0.5 if scale is None else scale, _ptr(O), ldo, _on(stream, dev)),
           "oq_attention_prompt")
    return O


class KV4Cache:
    """The tensors of a paged 4-bit key/value cache (oq_kv4_cache): k_codes
    uint8 [pages, heads, page_tokens, d / 2], v_codes uint8 [pages, heads,
    page_tokens / 16, d / 2, 16], k_scale, v_scale fp32 [pages, heads,
    page_tokens].  KV4Cache.empty makes them."""

    def __init__(self, k_codes, v_codes, k_scale, v_scale, rotate_k=False):
        _want(k_codes.dim() == 4, "k_codes: [pages, heads, page_tokens, d / 2] expected")
        p, h, t, half = k_codes.shape
        dev = k_codes.device
        for x, name, dtype, shape in ((k_codes, "k_codes", torch.uint8, (p, h, t, half)),
                                      (v_codes, "v_codes", torch.uint8, (p, h, t // 16, half, 16)),
                                      (k_scale, "k_scale", torch.float32, (p, h, t)),
                                      (v_scale, "v_scale", torch.float32, (p, h, t))):
            _want(x.dtype == dtype and x.shape == shape and x.is_contiguous() and x.device == dev,
                  f"{name}: contiguous {dtype} {list(shape)} on {dev} expected")
        self.k_codes, self.v_codes, self.k_scale, self.v_scale = k_codes, v_codes, k_scale, v_scale
        self.n_pages, self.n_kv_heads, self.page_tokens, self.head_dim = p, h, t, 2 * half
        self.rotate_k, self.device = bool(rotate_k), dev
        self._c = _lib.oq_kv4_cache(k_codes.data_ptr(), v_codes.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), p, t, h,
                                    2 * half, int(self.rotate_k))
        self.ref = C.byref(self._c)
        self._work_bytes = {}  # workspace sizes asked for (of this cache's heads)

    @classmethod
    def empty(cls, n_pages, n_kv_heads, head_dim, page_tokens=64, rotate_k=True, device="cuda:0"):
        """A cache of n_pages pages, cleared."""
        z = lambda dt, *shape: torch.zeros(shape, dtype=dt, device=device)  # noqa: E731
        return cls(z(torch.uint8, n_pages, n_kv_heads, page_tokens, head_dim // 2),
                   z(torch.uint8, n_pages, n_kv_heads, page_tokens // 16, head_dim // 2, 16),
                   z(torch.float32, n_pages, n_kv_heads, page_tokens), z(torch.float32, n_pages, n_kv_heads, page_tokens),
                   rotate_k)


def kv4_append(cache, K, V, slots, stream=None):
    """Quantize K, V (fp16 or bf16 [n, Hkv, d]) into the cache's slots (int64
    [n] = page * page_tokens + place; out of range: skipped)."""
    n = K.shape[0]
    ldk, ldv = _heads(K, "K", cache.head_dim), _heads(V, "V", cache.head_dim)
    dev = _device(K, V, cache.k_codes)
    _want(K.shape[1] == cache.n_kv_heads and V.shape == K.shape, "K and V: [n, the cache's heads, head_dim] expected")
    _want(K.dtype in _DTYPE and V.dtype == K.dtype, "K and V need one type")
    _ints(slots, "slots", torch.int64, n, dev)
    _check(_lib.load().oq_kv4_append(cache.ref, _ptr(K), _ptr(V), n, ldk, ldv, _DTYPE[K.dtype], _ptr(slots), _on(stream, dev)),
           "oq_kv4_append")


def kv4_gather(cache, slots, out_dtype=0, K=None, V=None, stream=None):
    """(K, V) [n, Hkv, d]: the values that the slots hold (fp16, bf16 or fp32 by
    out_dtype: OUT_F16, OUT_BF16, OUT_F32)."""
    n = slots.numel()
    dev = _device(slots, slots, cache.k_codes)
    _ints(slots, "slots", torch.int64, n, dev)
    dt = _TORCH.get(out_dtype)
    _want(dt is not None, "out_dtype: OUT_F16, OUT_BF16 or OUT_F32 expected")
    shape = (n, cache.n_kv_heads, cache.head_dim)
    ld = []
    for t, name in ((K, "K"), (V, "V")):
        if t is None:
            ld.append(shape[1] * shape[2])
        else:
            _want(t.shape == shape and t.dtype == dt and t.get_device() == dev, f"{name}: {list(shape)} of {dt} on cuda:{dev} expected")
            ld.append(_heads(t, name, shape[2]))
    K = _empty(slots, shape, dt, stream) if K is None else K
    V = _empty(slots, shape, dt, stream) if V is None else V
    _check(_lib.load().oq_kv4_gather(cache.ref, _ptr(slots), n, _ptr(K), _ptr(V), ld[0], ld[1], out_dtype,
                                     _on(stream, dev)), "oq_kv4_gather")
    return K, V


def attention_kv4_workspace_bytes(cache, tokens, n_heads, n_seqs, max_q, max_len) -> int:
    key = (tokens, n_heads, n_seqs, max_q, max_len)
    size = cache._work_bytes.get(key)
    if size is None:
        if len(cache._work_bytes) >= 256:  # (max_len may grow with every step)
            cache._work_bytes.clear()
        size = cache._work_bytes[key] = int(_lib.load().oq_attention_kv4_workspace_bytes(cache.ref, *key))
    return size


def attention_kv4(Q, cache, block_table, seq_lens, cu_q=None, max_q=None, max_len=None, causal=True, scale=None, O=None,
                  work=None, stream=None):
    """Attention of query tokens over the cache.  Q fp16 or bf16 [T, Hq, d];
    block_table int32 [n, width] (pages of each sequence), seq_lens int32 [n].
    cu_q None: one query token per sequence (T == n); else int32 [n + 1], and
    max_q (the most query tokens of a sequence) is needed.  max_len (default:
    what the table's width holds) bounds seq_lens; scale defaults to d ** -0.5.
    A sequence's query tokens are its last ones (causal).  Rows of no sequence
    are left as they were in O (unspecified when O is made here)."""
    ldq = _heads(Q, "Q", cache.head_dim)
    T, hq, d = Q.shape
    dev = _device(Q, Q, cache.k_codes)
    n = seq_lens.numel()
    _want(Q.dtype in _DTYPE, "Q: fp16 or bf16 expected")
    _want(block_table.dim() == 2 and block_table.shape[0] == n, "block_table: [sequences, width] expected")
    width = block_table.shape[1]
    _ints(block_table, "block_table", torch.int32, n * width, dev)
    _ints(seq_lens, "seq_lens", torch.int32, n, dev)
    if cu_q is None:
        _want(T == n, "without cu_q there is one query token per sequence")
        _want(max_q in (None, 1), "without cu_q, max_q is 1")
        max_q = 1
    else:
        _want(max_q is not None, "cu_q needs max_q")
        _ints(cu_q, "cu_q", torch.int32, n + 1, dev)
    if max_len is None:
        max_len = min(width * cache.page_tokens, 2 ** 30)
    if O is None:
        O, ldo = _empty(Q, (T, hq, d), Q.dtype, stream), hq * d
    else:
        _want(O.shape == Q.shape and O.dtype == Q.dtype and O.get_device() == dev, "O: Q's shape, type and device expected")
        ldo = _heads(O, "O", d)
    if work is None:
        nbytes = attention_kv4_workspace_bytes(cache, T, hq, n, max_q, max_len)
        work = _empty(Q, (nbytes,), torch.uint8, stream) if nbytes else None
    else:
        _want(work.get_device() == dev and work.is_contiguous() and work.element_size() == 1, "work: contiguous bytes on Q's device expected")
    _check(_lib.load().oq_attention_kv4(cache.ref, _ptr(Q), T, ldq, hq, _DTYPE[Q.dtype], _ptr(cu_q), max_q, _ptr(block_table),
                                        width, _ptr(seq_lens), n, max_len, int(causal), d ** -0.5 if scale is None else scale,
                                        _ptr(O), ldo, _ptr(work), 0 if work is None else work.numel(),
                                        _on(stream, dev)), "oq_attention_kv4")
    return O
