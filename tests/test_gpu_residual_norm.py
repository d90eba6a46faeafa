"""The norms around a block with its gate and residual, and the gated activation,
on the GPU: 16-bit outputs within float bounds of the 64-bit values, codes exactly
those of the 64-bit values."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import mx4_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
H, B, F32 = torch.float16, torch.bfloat16, torch.float32


def strided(x, pad):
    """x on the GPU in rows `pad` elements longer (NaN behind)."""
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype)
    wide[:, : x.shape[1]] = x
    return wide.to(DEV)[:, : x.shape[1]]


def make(M, D, dtype, rt, seed, mods=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    out = torch.where(torch.rand((D,), generator=g) < 0.02, 30.0, 1.0)
    t = dict(R=(3 * rnd(M, D) * out).to(rt), Y=(rnd(M, D) * out + 0.3).to(dtype))
    for n in ("g1", "g2", "b1", "b2"):
        t[n] = (0.2 * rnd(D) + (1 if n[0] == "g" else 0)).to(dtype)
    for n in ("gate", "scale", "shift"):
        t[n] = (0.3 * rnd(mods, D) + (1 if n == "gate" else 0)).to(dtype) if mods else None
    t["row"] = torch.randint(0, max(mods, 1), (M,), generator=g).to(torch.int32) if mods else None
    return t


def norms(t, pre, post, offset=0.0, eps=1e-6):
    """(binding's norms, reference's) of kinds, with gain and bias."""
    def one(kind, g, b):
        if kind is None:
            return None, None
        b = b if kind == "layer" else None
        return oq.Norm(kind, g.to(DEV), None if b is None else b.to(DEV), eps, offset), (kind, g, b, offset, eps)
    (a, ra), (b, rb) = one(pre, t["g2"], t["b2"]), one(post, t["g1"], t["b1"])
    return a, b, ra, rb


def pick(t, n):
    return None if t[n] is None else t[n][t["row"].long()]


SIZES = [(1, 8), (1, 2048), (3, 40), (4, 96), (5, 520), (70, 1024), (9, 1536), (2, 4096), (3, 8192), (2, 9216), (2, 16384),
         (600, 1000), (530, 1536), (520, 2048), (515, 2560), (513, 6144), (516, 12288)]
FORMS = [("rms", None, H, H, 0), ("rms", "rms", B, F32, 0), ("layer", None, H, F32, 3), ("layer", "layer", B, B, 1), ("rms", "layer", H, F32, 64)]


@pytest.mark.parametrize("M,D", SIZES)
@pytest.mark.parametrize("pre,post,dtype,rt,mods", FORMS)
def test_16_bits(M, D, pre, post, dtype, rt, mods):
    t = make(M, D, dtype, rt, M + D, mods)
    p, q, rp, rq = norms(t, pre, post, 1.0 if mods == 64 else 0.0)
    if mods == 64:
        t["g1"], t["g2"] = t["g1"] - 1, t["g2"] - 1
        p, q, rp, rq = norms(t, pre, post, 1.0)
    dev = lambda n: None if t[n] is None else t[n].to(DEV)  # noqa: E731
    r, h = oq.residual_norm(strided(t["R"], 8), strided(t["Y"], 16), p, q, 0.75, dev("gate"), dev("scale"), dev("shift"), dev("row"))
    wr, er, wh, eh = R.residual_norm(t["R"], t["Y"], rp, rq, 0.75, pick(t, "gate"), pick(t, "scale"), pick(t, "shift"))
    R.check(r, wr, er, rt)
    R.check(h, wh, eh, dtype)


@pytest.mark.parametrize("M,D", [s for s in SIZES if s[1] % 32 == 0])
@pytest.mark.parametrize("pre,post,dtype,rt,mods", FORMS)
def test_codes(M, D, pre, post, dtype, rt, mods):
    t = make(M, D, dtype, rt, M + D + 1, mods)
    p, q, rp, rq = norms(t, pre, post)
    dev = lambda n: None if t[n] is None else t[n].to(DEV)  # noqa: E731
    r, h = oq.residual_norm(strided(t["R"], 8), strided(t["Y"], 16), p, q, 0.75, dev("gate"), dev("scale"), dev("shift"), dev("row"),
                            mx4=True)
    wr, er, wh, _ = R.residual_norm(t["R"], t["Y"], rp, rq, 0.75, pick(t, "gate"), pick(t, "scale"), pick(t, "shift"))
    R.check(r, wr, er, rt)
    R.check_codes(h, wh)


@pytest.mark.parametrize("mx4", [False, True])
def test_parts_that_are_left_out(mx4):
    M, D = 37, 1024
    t = make(M, D, H, H, 3, 1)
    t["row"] = None
    p, q, rp, rq = norms(t, "rms", "layer")
    x, y = t["R"].to(DEV), t["Y"].to(DEV)
    one = lambda n: t[n].expand(M, -1)  # noqa: E731

    def check(got, want):
        R.check(got[0], want[0], want[1], got[0].dtype)
        if want[2] is None:
            assert got[1] is None
        elif mx4:
            R.check_codes(got[1], want[2])
        else:
            R.check(got[1], want[2], want[3], H)

    # A norm alone; a residual alone; no residual; a gate without the others; rows of [D].
    check(oq.residual_norm(x, None, p, mx4=mx4), R.residual_norm(t["R"], None, rp, None, 1.0, None, None, None))
    check(oq.residual_norm(None, y, p, q, mx4=mx4), R.residual_norm(None, t["Y"], rp, rq, 1.0, None, None, None))
    check(oq.residual_norm(x, y, p, mx4=mx4, gate=t["gate"][0].to(DEV)), R.residual_norm(t["R"], t["Y"], rp, None, 1.0, one("gate"), None, None))
    check(oq.residual_norm(x, y, p, mx4=mx4, shift=t["shift"].to(DEV)), R.residual_norm(t["R"], t["Y"], rp, None, 1.0, None, None, one("shift")))
    check(oq.residual_norm(x, y, None, q, alpha=-2.0), R.residual_norm(t["R"], t["Y"], None, rq, -2.0, None, None, None))
    bare = oq.Norm("rms", eps=0.5)
    check(oq.residual_norm(x, y, bare, bare, mx4=mx4),
          R.residual_norm(t["R"], t["Y"], ("rms", None, None, 0.0, 0.5), ("rms", None, None, 0.0, 0.5), 1.0, None, None, None))
    # fp32 residual without a block's output.
    check(oq.residual_norm(t["R"].float().to(DEV), None, p, mx4=mx4, dtype=H), R.residual_norm(t["R"], None, rp, None, 1.0, None, None, None))


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("M,D", [(6, 256), (5, 2048), (600, 1024)])
def test_rows_without_a_modulation(mx4, M, D):
    """Tokens whose index is out of range are left as they were; one modulation
    tensor holds the three parts side by side."""
    t = make(M, D, B, F32, 9, 4)
    p, _, rp, _ = norms(t, "layer", None)
    t["row"][0], t["row"][M - 1], t["row"][M // 2] = -1, 4, 2 ** 31 - 1
    mod = torch.cat([t["gate"], t["scale"], t["shift"]], 1).to(DEV)
    gate, scale, shift = mod.split(D, 1)
    out = torch.full((M, D), 5.0, device=DEV)
    h = (torch.full((M, D // 2), 0xA5, dtype=torch.uint8, device=DEV), torch.full((M, oq.mx4_step_bytes(D)), 0xA5, dtype=torch.uint8, device=DEV)) \
        if mx4 else torch.full((M, D), 6.0, dtype=B, device=DEV)
    oq.residual_norm(t["R"].to(DEV), t["Y"].to(DEV), p, None, 1.0, gate, scale, shift, t["row"].to(DEV), mx4, out, h)
    keep = (t["row"] >= 0) & (t["row"] < 4)
    t["row"] = t["row"].clamp(0, 3)
    want = R.residual_norm(t["R"], t["Y"], rp, None, 1.0, pick(t, "gate"), pick(t, "scale"), pick(t, "shift"))
    R.check(out.cpu()[keep], want[0][keep], want[1][keep], F32)
    assert bool((out.cpu()[~keep] == 5).all())
    if mx4:
        R.check_codes([x.cpu()[keep] for x in h], want[2][keep])
        assert all(bool((x.cpu()[~keep] == 0xA5).all()) for x in h)
    else:
        R.check(h.cpu()[keep], want[2][keep], want[3][keep], B)
        assert bool((h.cpu()[~keep] == 6).all())


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("M,D,rt", [(17000, 32, B), (9000, 64, F32), (4500, 1024, F32), (4500, 1024, B), (4200, 2048, B), (2100, 4096, F32), (1100, 8192, F32),
                                    (1100, 16384, B), (1100, 16384, F32)])
def test_more_rows_than_the_chip_holds(mx4, M, D, rt):
    """A workgroup's second and third row are worked on as its first, also behind one
    that is skipped."""
    t = make(M, D, B, rt, D, 3)
    p, q, rp, rq = norms(t, "layer", "rms")
    t["row"][::5] = -1
    keep = t["row"] >= 0
    out = torch.full((M, D), 5.0, dtype=rt, device=DEV)
    r, h = oq.residual_norm(t["R"].to(DEV), t["Y"].to(DEV), p, q, 1.5, t["gate"].to(DEV), t["scale"].to(DEV), t["shift"].to(DEV), t["row"].to(DEV), mx4, out)
    assert bool((r[~keep.to(DEV)] == 5).all())
    for n in ("R", "Y", "row"):
        t[n] = t[n][keep]
    wr, er, wh, eh = R.residual_norm(t["R"], t["Y"], rp, rq, 1.5, pick(t, "gate"), pick(t, "scale"), pick(t, "shift"))
    R.check(r.cpu()[keep], wr, er, rt)
    if mx4:
        R.check_codes([c.cpu()[keep] for c in h], wh)
    else:
        R.check(h.cpu()[keep], wh, eh, B)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("M,D,holds", [(5120, 1536, 1024), (2560, 8192, 512)])
def test_skipped_rows_between_others(mx4, M, D, holds):
    """One exchange a row, and every other row of a workgroup left: the rows on either
    side do not share its memory."""
    t = make(M, D, B, B, D, 2)
    t["row"] = torch.where(torch.arange(M) // holds % 2 == 1, -1, 0).to(torch.int32)
    keep = t["row"] >= 0
    p, _, rp, _ = norms(t, "rms", None)
    _, h = oq.residual_norm(t["R"].to(DEV), t["Y"].to(DEV), p, None, 1.5, t["gate"].to(DEV), None, None, t["row"].to(DEV), mx4)
    _, _, wh, eh = R.residual_norm(t["R"][keep], t["Y"][keep], rp, None, 1.5, t["gate"][:1].double().expand(int(keep.sum()), D), None, None)
    if mx4:
        R.check_codes([c.cpu()[keep] for c in h], wh)
    else:
        R.check(h.cpu()[keep], wh, eh, B)


@pytest.mark.parametrize("M,D", [(4, 512), (3, 4096), (700, 2048)])
def test_in_place_is_the_same(M, D):
    t = make(M, D, H, H, 4)
    p, q, _, _ = norms(t, "rms", "rms")
    x, y = t["R"].to(DEV), t["Y"].to(DEV)
    r, h = oq.residual_norm(x, y, p, q)
    oq.residual_norm(x, y, p, q, R_out=x, H=y)
    assert torch.equal(x, r) and torch.equal(y, h)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("D", [64, 2048])
def test_special_rows(mx4, D):
    """Rows of zeros, of one value, of large and of tiny numbers; a NaN and an
    infinity stay in their rows."""
    t = make(8, D, B, F32, 5)
    t["Y"][0] = 0
    t["R"][0] = 0
    t["Y"][1], t["R"][1] = 3.0, 1.0
    t["Y"][2], t["R"][2] = t["Y"][2] * 1e15, t["R"][2] * 1e15
    t["Y"][3], t["R"][3] = t["Y"][3] * 1e-20, t["R"][3] * 1e-20
    for kind in ("rms", "layer"):
        p, q, rp, rq = norms(t, kind, kind)
        x, y = t["R"].clone(), t["Y"].clone()
        x[6, 3], y[7, D - 1] = float("nan"), float("inf")
        r, h = oq.residual_norm(x.to(DEV), y.to(DEV), p, q, mx4=mx4)
        want = [w[:6] for w in R.residual_norm(t["R"], t["Y"], rp, rq, 1.0, None, None, None)]
        R.check(r[:6], want[0], want[1], F32)
        if mx4:
            index, byte = R.unpack(*h)
            assert bool((byte[6:] == 255).all()) and not bool((byte[:6] == 255).any())
            rest = [0, 2, 3, 4, 5]  # (LayerNorm of one value is 0 by 0 up to the mean's rounding)
            R.check_codes([c[rest] for c in h], want[2][rest])
        else:
            R.check(h[:6], want[2], want[3], B)
            assert bool(torch.isnan(h[6:]).all())


@pytest.mark.parametrize("dtype", [H, B])
@pytest.mark.parametrize("act", [oq.ACT_GELU_TANH, oq.ACT_SILU])
@pytest.mark.parametrize("M,F", [(1, 8), (1, 16384), (3, 40), (7, 96), (50, 4096), (300, 1056), (2, 65536)])
def test_activation(dtype, act, M, F):
    g = torch.Generator().manual_seed(F + act)
    x = torch.randn((M, 2 * F), generator=g) * torch.tensor([0.1, 1.5, 8.0])[torch.randint(0, 3, (M, 1), generator=g)]
    x[:, ::7] *= 4
    x = x.to(dtype)
    gu = strided(x, 8)
    want, bound = R.activation(x, act)
    R.check(oq.gated_activation(gu, act), want, bound, dtype)
    if F % 32 == 0:
        R.check_codes(oq.gated_activation(gu, act, mx4=True), want)


@pytest.mark.parametrize("act", [oq.ACT_GELU_TANH, oq.ACT_SILU])
def test_activation_far_out(act):
    """Every bf16 gate with ups from tiny to huge: what e^-t does in float at its
    ends does not show in the codes; zeros, NaN and infinities."""
    gates = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(B)
    gates = gates[torch.isfinite(gates)]
    gates = gates[gates.double().abs() < 1e36]  # (g^3 within a double of the reference)
    gates = torch.cat([gates, gates[: -gates.numel() % 32]])
    rows = []
    for up in (1.0, 1e-30, -3e30, 0.0):
        rows.append(torch.cat([gates, torch.full_like(gates, up)]))
    x = torch.stack(rows).view(4, 2, -1, 32).transpose(1, 2).reshape(-1, 64)     # one block a row
    want, _ = R.activation(x, act)
    R.check_codes(oq.gated_activation(x.to(DEV), act, mx4=True), want)
    x = x[:4].clone()
    x[0, 3], x[1, 40], x[2, 5], x[2, 37] = float("nan"), float("inf"), float("inf"), 1.0
    _, byte = R.unpack(*oq.gated_activation(x.to(DEV), act, mx4=True))
    assert byte[:3].flatten().tolist() == [255, 255, 255] and byte[3].item() != 255


def test_no_rows():
    z = torch.empty((0, 64), dtype=H, device=DEV)
    r, h = oq.residual_norm(z, z, oq.Norm("rms"))
    assert r.shape == h.shape == (0, 64) and oq.gated_activation(z).shape == (0, 32)
