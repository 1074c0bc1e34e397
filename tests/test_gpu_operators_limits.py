"""What include/streamkl.h says of values at the limits: how far a non-finite one reaches, and how large logits may be."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def make(B, H, HK, NQ, NK, d, dv, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()   # noqa: E731
    args = [mk(B, H, NQ, d), mk(B, HK, NK, d), mk(B, H, NQ, d), mk(B, HK, NK, d), mk(B, HK, NK, dv)]
    return [*args, 0.2 + 0.6 * torch.rand(H, generator=gen, device="cuda")], mk(B, H, NQ, dv)


def run(sk, args, do, splits=1):
    saved = sk.diff_fwd(*args, None, True, splits=splits, save=True)
    return saved, sk.diff_bwd(*args, do, *saved, None, True)


# 64 packed rows a wave (64/64, 64/128), 32 (128/128), 16 or 32 in the backward; offsets that are no multiples of the tile
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("H,HK", [(2, 2), (6, 2)])
@pytest.mark.parametrize("d,dv,NQ,NK", [(64, 64, 300, 300), (64, 128, 257, 290), (128, 128, 300, 301), (32, 32, 290, 257)])
def test_reach_of_a_non_finite_value(gpu_lib, d, dv, NQ, NK, H, HK, value, splits):
    args, do = make(1, H, HK, NQ, NK, d, dv)
    off = NK - NQ
    clean, g = run(gpu_lib, args, do, splits)
    group = slice(0, H // HK)   # the heads of key head 0
    for j in (200, 223, 224, NK - 1):   # the ends of tiles among them
        far = max(0, j - 94 - off)   # rows before this one are out of reach
        for which in (4, 1, 3):
            bad = [a.clone() for a in args]
            bad[which][0, 0, j, 3] = value
            dirty, h = run(gpu_lib, bad, do, splits)
            for a, b in ((clean[0], dirty[0]), (clean[1], dirty[1]), (g[0], h[0]), (g[2], h[2])):
                assert torch.equal(a[:, :, :far], b[:, :, :far])
                assert torch.equal(a[:, group.stop:], b[:, group.stop:])
            if which == 4:
                assert not torch.isfinite(dirty[0][0, group, j - off:, 3]).any()
            else:   # hidden keys leave the rows before them, not only far ones, as they are in the forward pass
                assert torch.equal(clean[0][:, :, :j - off], dirty[0][:, :, :j - off])
    i = 40 - min(off, 0)
    near = off + i + 62   # keys behind this one are out of reach
    for which in (0, 2, 6):
        bad = [a.clone() for a in (*args, do)]
        bad[which][0, 1, i, 5] = value
        dirty, h = run(gpu_lib, bad[:6], bad[6], splits)
        keep = torch.ones(1, H, NQ, dtype=torch.bool, device="cuda")
        keep[0, 1, i] = False
        for a, b in ((clean[0], dirty[0]), (g[0], h[0]), (g[2], h[2])):
            assert torch.equal(a[keep], b[keep])
        for n in (1, 3, 4):
            assert torch.equal(g[n][:, :, near + 1:], h[n][:, :, near + 1:])


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128)])
def test_logits_up_to_2_28(gpu_lib, d, dv, sign, splits):
    """All logits +-2^27.9: flat maps, the mean of the values; a key of half the size makes no difference above 0."""
    args, _ = make(1, 2, 1, 5, 200, d, dv)
    top = 2.0 ** 27.9
    for i, fill in ((0, 1024.0), (1, sign), (2, 1024.0), (3, sign)):
        args[i] = torch.full_like(args[i], fill)
    if sign > 0:
        args[1][0, 0, 100:] = 0.5   # map 1 has the first half of the keys
    out, out2, lse1, lse2 = gpu_lib.diff_fwd(*args, top / (1024 * d), False, splits=splits, save=True)
    v = args[4][0, 0].double()
    m1, m2 = (v[:100] if sign > 0 else v).mean(0), v.mean(0)
    lam = args[5].double()[None, :, None, None]
    # probabilities are equal, so that only the one rounding of each output is left; float32 sums of 200 terms
    small = 2.0 ** -16 * v.abs().mean()
    assert ((out2.double() - m2).abs() <= 2.0 ** -8 * m2.abs() + small).all()
    ref = m1 - lam * m2
    assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2 * small).all()
    for lse, n in ((lse1, 100 if sign > 0 else 200), (lse2, 200)):
        assert ((lse.double() - (sign * top + math.log(n))).abs() <= 2.0 ** -22 * top).all()


@pytest.mark.parametrize("splits", [1, 3])
def test_values_up_to_2_40_above_a_reference_that_stays(gpu_lib, splits):
    """Logits that rise by just under 64 doublings after the first tile, which does not move the reference."""
    args, _ = make(1, 2, 1, 40, 400, 64, 64)
    q1, k1, q2, k2, v, _ = args
    rise = 63.0 * math.log(2)
    for q, k in ((q1, k1), (q2, k2)):
        q.fill_(1.0)
        k.fill_(0.0)
        k[:, :, 32:].fill_(rise / 64)
    v.mul_(2.0 ** 38)
    out, out2, lse1, _ = gpu_lib.diff_fwd(*args, 1.0, False, splits=splits, save=True)
    top = float(k1[0, 0, 32].double().sum())
    w = torch.ones(400, dtype=torch.float64, device="cuda")
    w[:32] = math.exp(-top)
    mean = (w[:, None] * v[0, 0].double()).sum(0) / w.sum()
    # equal probabilities above the first tile, whose rounding to bf16 is one factor, at most 2^-8; float32 sums
    small = 2.0 ** -16 * v.double().abs().mean()
    assert ((out2.double() - mean).abs() <= 2.0 ** -7 * mean.abs() + small).all()
    assert ((lse1.double() - (top + math.log(float(w.sum())))).abs() <= 2.0 ** -18).all()


@pytest.mark.parametrize("splits,NQ", [(1, 70), (3, 70), (3, 2100)])
def test_log_sum_exp_of_a_row_that_is_not_a_number(gpu_lib, splits, NQ):
    """NaN, not the -inf of a row that sees no key."""
    args, _ = make(1, 1, 1, NQ, 200, 64, 64)
    kv_len = torch.tensor([150], dtype=torch.int32, device="cuda")
    args[0][0, 0, 40] = float("nan")
    args[2][0, 0, 41] = float("nan")
    q_len = torch.tensor([45], dtype=torch.int32, device="cuda")
    _, _, lse1, lse2 = gpu_lib.diff_fwd(*args, None, False, q_len, kv_len, splits=splits, save=True)
    for lse, i in ((lse1, 40), (lse2, 41)):
        assert torch.isnan(lse[0, 0, i]) and torch.isneginf(lse[0, 0, 45:]).all()
        assert int(torch.isfinite(lse).sum()) == 44
    q_len.fill_(NQ)
    kv_len.fill_(0)
    assert all(torch.isneginf(x).all() for x in gpu_lib.diff_fwd(*args, None, False, q_len, kv_len, splits=splits, save=True)[2:])
