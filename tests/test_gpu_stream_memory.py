"""Memory that a call on a given stream makes (outputs, workspaces) is of that
stream: not a block that the current stream may still read, and not one that is
handed out on the current stream while the call still writes it."""
import pytest
import torch

import paper_2605_28803_amd as oq

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _h(*shape):
    return torch.randn(shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(len(shape))).half()


def _calls():
    M, N, K = 96, 320, 1024
    X, W = _h(M, K), _h(N, K)
    Xq, xs = oq.rotate_quantize_act(X, K)
    Xt, _ = oq.rotate_quantize_act_tiled(X, K)
    Xq8, xs8 = oq.rotate_quantize_act_i8(X, K)
    Wq, ws = oq.quantize_weights(W, K)
    Wq8, ws8 = oq.quantize_weights_i8(W, K)
    delta = torch.full((K,), 0.5, device=DEV)
    Y = oq.rotate_act_f32(X, K)
    perm, Rt, _, _ = oq.prepare_weights_composite(W)
    energy = oq.channel_energy(W)
    U, _ = oq.block_svd(W, perm)
    qkv = _h(M, 10, 64)
    cu = torch.tensor([0, M], dtype=torch.int32, device=DEV)
    cache = oq.KV4Cache.empty(80, 1, 64)
    slots = torch.arange(5000, device=DEV)
    oq.kv4_append(cache, _h(5000, 1, 64), _h(5000, 1, 64), slots)
    table = torch.arange(80, dtype=torch.int32, device=DEV)[None]
    lens = torch.tensor([5000], dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    return {
        "rotate_quantize_act": lambda s: oq.rotate_quantize_act(X, K, stream=s),
        "rotate_quantize_act_tiled": lambda s: oq.rotate_quantize_act_tiled(X, K, stream=s),
        "codes_to_tiled": lambda s: oq.codes_to_tiled(Xq, stream=s),
        "rotate_quantize_act_composite": lambda s: oq.rotate_quantize_act_composite(X, perm, Rt, stream=s),
        "rotate_debug_f32": lambda s: oq.rotate_debug_f32(X, K, stream=s),
        "w4a4_linear": lambda s: oq.w4a4_linear(Xq, xs, Wq, ws, stream=s),
        "w4a4_gemm_i32": lambda s: oq.w4a4_gemm_i32(Xq, Wq, stream=s),
        "w4a4_linear_tiled": lambda s: oq.w4a4_linear_tiled(Xt, xs, Wq, ws, stream=s),
        "w4a4_gemm_i32_tiled": lambda s: oq.w4a4_gemm_i32_tiled(Xt, M, Wq, stream=s),
        "quantize_weights": lambda s: oq.quantize_weights(W, K, stream=s),
        "rotate_quantize_act_i8": lambda s: oq.rotate_quantize_act_i8(X, K, stream=s),
        "w4a8_linear": lambda s: oq.w4a8_linear(Xq8, xs8, Wq, ws, stream=s),
        "w4a8_gemm_i32": lambda s: oq.w4a8_gemm_i32(Xq8, Wq, stream=s),
        "quantize_weights_i8": lambda s: oq.quantize_weights_i8(W, K, stream=s),
        "w8a8_linear": lambda s: oq.w8a8_linear(Xq8, xs8, Wq8, ws8, stream=s),
        "w8a8_gemm_i32": lambda s: oq.w8a8_gemm_i32(Xq8, Wq8, stream=s),
        "channel_energy": lambda s: oq.channel_energy(W, stream=s),
        "zigzag_permutation": lambda s: oq.zigzag_permutation(energy, stream=s),
        "block_svd": lambda s: oq.block_svd(W, perm, stream=s),
        "block_rotations": lambda s: oq.block_rotations(U, stream=s),
        "prepare_weights_composite": lambda s: oq.prepare_weights_composite(W, stream=s),
        "rotate_act_f32": lambda s: oq.rotate_act_f32(X, K, stream=s),
        "calibrate_step_scales": lambda s: oq.calibrate_step_scales(Y, stream=s),
        "calibrate_step_scales_noalloc": lambda s: oq.calibrate_step_scales_noalloc(Y, stream=s),
        "rotate_quantize_act_static": lambda s: oq.rotate_quantize_act_static(X, K, delta, stream=s),
        "rotate_quantize_act_static_tiled": lambda s: oq.rotate_quantize_act_static_tiled(X, K, delta, stream=s),
        "quantize_weights_step": lambda s: oq.quantize_weights_step(W, K, delta, stream=s),
        "attention_prompt": lambda s: oq.attention_prompt(qkv[:, :8], qkv[:, 8:9], qkv[:, 9:], cu, stream=s),
        "kv4_gather": lambda s: oq.kv4_gather(cache, slots, stream=s),
        "attention_kv4": lambda s: oq.attention_kv4(qkv[:1, :8], cache, table, lens, stream=s),
    }


def test_outputs_belong_to_the_call_s_stream():
    """Blocks just freed on the current stream are not what a call on another one
    writes, and what it made does not come back on the current one; values as ever."""
    s = torch.cuda.Stream()
    for name, call in _calls().items():
        want = call(None)
        torch.cuda.synchronize()
        tensors = (want,) if torch.is_tensor(want) else want
        freed = [torch.empty_like(t) for t in tensors]
        at = {t.data_ptr() for t in freed}
        del freed
        got = call(s)
        torch.cuda.synchronize()
        got = (got,) if torch.is_tensor(got) else got
        for a, b in zip(got, tensors):
            assert torch.equal(a, b), name
        assert not at & {t.data_ptr() for t in got}, name
        like, at = [(t.shape, t.dtype) for t in got], {t.data_ptr() for t in got}
        del got, a
        again = [torch.empty(n, dtype=dt, device=DEV) for n, dt in like for _ in range(4)]
        assert not at & {t.data_ptr() for t in again}, name
        del again


@pytest.mark.parametrize("name", ["attention_prompt", "attention_kv4", "kv4_gather", "w8a8_linear", "w8a8_gemm_i32", "quantize_weights_i8"])
def test_what_the_current_stream_still_reads(name):
    """The current stream is busy and will copy a block that its owner has
    dropped: a call on an idle stream leaves it alone."""
    call = _calls()[name]
    out = call(None)
    out = (out,) if torch.is_tensor(out) else out
    s = torch.cuda.Stream()
    call(s)  # (the other stream's memory is there)
    a = torch.randn((4096, 4096), device=DEV)
    torch.cuda.synchronize()
    for _ in range(10):
        a = (a @ a).clamp(-1, 1)
    blocks = [torch.full_like(t, 7) for t in out]
    for _ in range(10):
        a = (a @ a).clamp(-1, 1)
    copies = [b.clone() for b in blocks]
    del blocks
    got = call(s)
    torch.cuda.synchronize()
    assert all((c == 7).all() for c in copies)
    assert all(torch.equal(x, y) for x, y in zip((got,) if torch.is_tensor(got) else got, out))
