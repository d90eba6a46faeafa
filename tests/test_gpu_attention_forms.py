"""Every form of the attention kernels: head widths, rows of a kv head from one
to more than 16, short and long sequences (one or several splits, four or eight
waves), rotated or not, both types."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import serving_ref as R
from tests.test_gpu_attention_prompt import _run

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("nq,group", [(1, 1), (2, 2), (1, 7), (2, 4), (3, 4), (16, 1), (5, 5), (40, 1)])
def test_cache_attention(nq, group, d, rotate, dtype):
    hk = 2
    for lens in ([300, 0, 37], [3000, nq, 1100], [900] * 70 if d == 128 and nq == 1 else [513]):
        g = torch.Generator().manual_seed(d + nq)
        n, page = len(lens), 48
        wide = -(-max(lens) // page)
        cache = oq.KV4Cache.empty(n * wide, hk, d, page, rotate_k=rotate)
        table = torch.randperm(n * wide, generator=g).to(torch.int32).view(n, wide)
        pos = torch.cat([torch.arange(L) for L in lens])
        seq = torch.arange(n).repeat_interleave(torch.tensor(lens))
        slots = table[seq, pos // page].long() * page + pos % page
        k, v = torch.randn((2, pos.numel(), hk, d), generator=g).to(dtype)
        oq.kv4_append(cache, k.to(DEV), v.to(DEV), slots.to(DEV))
        q = torch.randn((n * nq, group * hk, d), generator=g).to(dtype)
        cu = torch.arange(n + 1, dtype=torch.int32) * nq
        o = oq.attention_kv4(q.to(DEV), cache, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                             None if nq == 1 else cu.to(DEV), max_q=nq, max_len=max(lens)).cpu()
        bufs = [t.cpu() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)]
        s = d ** -0.5
        for i in range(n) if n < 10 else (0, 33, 69):
            L = lens[i]
            kk, vv = R.take(bufs, slots[seq == i], d, rotate)
            see = torch.arange(L)[None, :] <= (L - nq + torch.arange(nq))[:, None]
            for h in range(group * hk):
                qq, ka, va = q[i * nq:(i + 1) * nq, h].double(), kk[:, h // group], vv[:, h // group]
                qq = qq @ R.hadamard(d) / d ** 0.5 if rotate else qq
                ref, spread, p = R.attend(qq, ka, va, s, see)
                extra = 2 * R.score_error(qq, ka, s)
                if L:
                    # The accumulator starts at 72 sum(q) in units of the step (max / 7); a rotated query is
                    # rounded in fp32 (log2 d sums) and to 22 bits, each against its row's sum.
                    one = qq.abs().sum(-1).max().item() * s
                    extra += 2 * one * ka.abs().max().item() / 7 * (80 * (d + 8) * 2.0 ** -24 + (7 * 12 * 2.0 ** -22 if rotate else 0))
                    # A probability times a step is rounded to 2^-11 of itself down to 2^-29 of the largest,
                    # below that to half of 2^-39 of it (spread is taken times 2^-10).
                    spread = spread + L * 7 * 2.0 ** -40 * 2.0 ** 10 * (p[:, :, None] * va.abs()[None]).amax((1, 2))[:, None]
                R.check(o[i * nq:(i + 1) * nq, h], ref, spread, extra, dtype, 2.0 ** -11)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,hq,hk", [(64, 130, 5), (128, 52, 4), (256, 52, 4)])
def test_prompt_attention_of_one_key_group(d, hq, hk, causal):
    """Enough workgroups that no keys are dealt to groups, over several steps."""
    _run([700], hq, hk, d, causal, torch.bfloat16)
