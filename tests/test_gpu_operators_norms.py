"""Differential attention on the GPU against the plain fp64 form, in norm: roundings of many elements that are independent
of each other average, which elementwise bounds (sums of worst cases) cannot see."""
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo

pytestmark = pytest.mark.gpu

NAMES = ("dq1", "dk1", "dq2", "dk2", "dv", "dlam")


def n64(t):
    return t.detach().double().cpu().numpy()


def make(B, H, HK, NQ, NK, d, dv, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()   # noqa: E731
    args = (mk(B, H, NQ, d), mk(B, HK, NK, d), mk(B, H, NQ, d), mk(B, HK, NK, d), mk(B, HK, NK, dv))
    return (*args, 0.2 + 0.6 * torch.rand(H, generator=gen, device="cuda")), mk(B, H, NQ, dv)


def dlam_terms(args, do, causal):
    """dlam and the root of the sum of the squares of its terms P_2 dP, per head, in 64 bits."""
    q, k, v = (args[i].double() for i in (2, 3, 4))
    B, H, NQ, d = q.shape
    HK, NK = k.shape[1:3]
    hidden = torch.ones(NQ, NK, dtype=torch.bool, device="cuda").triu(NK - NQ + 1) if causal else None
    value, size = np.zeros(H), np.zeros(H)
    for b in range(B):
        for h in range(H):
            j = h // (H // HK)
            z = q[b, h] @ k[b, j].t().contiguous() / math.sqrt(d)
            if causal:
                z = z.masked_fill(hidden, -math.inf)
            t = torch.softmax(z, 1) * (do[b, h].double() @ v[b, j].t().contiguous())
            value[h] -= float(t.sum())
            size[h] += float((t * t).sum())
    return value, np.sqrt(size)


# Relative to the root of the sum of the squared terms, to which errors that are independent from term to term add up.
# A term is off by the rounding of its exponent (half a step, 2^-22 below 8, 2^-21 below 16, times ln 2), the exponential
# (2^-23), its logit and dP (d products in a few float32 sums: 2^-22 each): in norm, a rounding of at most r having the
# norm r / sqrt(3), 2^-22 with 256 keys and 2^-21 with 8192 (2^13 keys: exponents to 16).
@pytest.mark.parametrize("B,H,HK,NQ,NK,d,dv,causal,seeds,bound", [
    (1, 1, 1, 256, 256, 64, 64, False, 24, 2.0 ** -22),    # one head, where the sum cancels
    (1, 16, 16, 64, 8192, 64, 64, False, 1, 2.0 ** -21),   # long sums; 32 rows a wave
    (1, 8, 2, 300, 8192, 128, 128, False, 1, 2.0 ** -21),  # 16 rows a wave, the key axis in ranges
    (2, 4, 2, 200, 4096, 64, 192, True, 2, 2.0 ** -21),
    (1, 2, 2, 6007, 6007, 128, 128, False, 1, 2.0 ** -21),  # many rows: what their errors have in common adds up
    (1, 2, 1, 4001, 4001, 64, 128, True, 1, 2.0 ** -21)])
def test_dlam_is_as_exact_as_its_terms(gpu_lib, B, H, HK, NQ, NK, d, dv, causal, seeds, bound):
    rel = []
    for seed in range(seeds):
        args, do = make(B, H, HK, NQ, NK, d, dv, seed)
        saved = gpu_lib.diff_fwd(*args, None, causal, save=True)
        got = gpu_lib.diff_bwd(*args, do, *saved, None, causal, want=("dlam",))[5]
        value, size = dlam_terms(args, do, causal)
        rel.append((n64(got) - value) / size)
    rms = float(np.sqrt(np.mean(np.concatenate(rel) ** 2)))
    print(f"dlam {rms:.2e}, bound {bound:.2e}", flush=True)
    assert rms <= bound


# The saved value is rounded once: 2^-24 of it, at most 2^-21 below 16, in norm 2^-21 / sqrt(3) = 2.8e-7. The sum over the
# keys of a half-wave has 256 additions in a chunk and 256 chunks here, each addition off by 2^-24 of a sum that grows:
# sqrt(256) 2^-24 / 3 in norm, over the two half-waves 2.2e-7. Exponentials (2^-23 each) and the factor of the logits (two
# roundings of 2^-25, times a mean logit of about 1) are small next to that. Together 3.6e-7.
@pytest.mark.parametrize("splits", [1, 5, "auto"])
@pytest.mark.parametrize("d,dv,NQ", [(64, 64, 80), (128, 128, 8)])
def test_log_sum_exp_does_not_drift(gpu_lib, d, dv, NQ, splits):
    """Over 131072 keys, in one pass and joined from ranges."""
    (q1, k1, q2, k2, v, lam), _ = make(1, 2, 1, NQ, 131072, d, dv, seed=d)
    saved = gpu_lib.diff_fwd(q1, k1, q2, k2, v, lam, splits=splits, save=True)
    for lse, q, k in ((saved[2], q1, k1), (saved[3], q2, k2)):
        ref = torch.logsumexp(q[0].double().flatten(0, 1) @ k[0, 0].double().t().contiguous() / math.sqrt(d), 1)
        rms = float((lse.flatten().double() - ref).pow(2).mean().sqrt())
        print(f"lse {rms:.2e}", flush=True)
        assert rms <= 2.0 ** -21


def partial_floats(sk, B, H, HK, NQ, NK, d, dv, causal):
    """Floats of partial gradients in the backward's workspace; the sums for dlam at most added."""
    return sk.diff_bwd_workspace_bytes(B, H, HK, NQ, NK, d, dv, causal) // 4 - B * H * -(-NQ // 32) * 128


def check(sk, args, do, causal, q_len=None, kv_len=None):
    """Outputs and gradients element by element, and in norm. Each is a sum of products of which one operand is rounded to
    bf16 (2^-8 / sqrt(3) in norm), with the outputs' own rounding, or that of the outputs in D: three such, 2^-8."""
    lens = [None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda") for x in (q_len, kv_len)]
    saved = sk.diff_fwd(*args, None, causal, *lens, save=True)
    got = sk.diff_bwd(*args, do, *saved, None, causal, *lens)
    torch.cuda.synchronize()
    plain = [n64(a) for a in args]
    scale = plain[0].shape[-1] ** -0.5
    ref, tol = oo.diff(*plain, scale, causal, q_len, kv_len)
    grads, gtol = oo.diff_backward(*plain, scale, causal, n64(do), q_len, kv_len)
    pairs = [("out", saved[0], ref["out"], tol["out"]), ("out2", saved[1], ref["out2"], tol["out2"])]
    pairs += [(n, t, grads[n], gtol[n]) for n, t in zip(NAMES, got)]
    for n, t, r, bound in pairs:
        e = np.abs(n64(t) - r)
        assert (e <= bound + 1e-30).all(), f"{n}: worst {np.nanmax(e / (bound + 1e-30)):.2f} bounds"
        if n != "dlam":
            norm = float(np.sqrt((e * e).sum()) / np.sqrt((r * r).sum()))
            print(f"{n} {norm:.2e}", flush=True)
            assert norm <= 2.0 ** -8, n


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,dv", [(64, 64), (64, 128), (96, 160), (128, 128), (64, 192), (128, 256)])
@pytest.mark.parametrize("NK,kv_len", [(1000, None), (2011, [2011, 1203])])
def test_query_gradients_from_ranges_of_keys(gpu_lib, d, dv, NK, kv_len, causal):
    """Few rows against many keys; partials that are larger than the key-owned kernel's would be."""
    B, H, HK, NQ = (1 if kv_len is None else 2), 4, 2, 100
    floats = partial_floats(gpu_lib, B, H, HK, NQ, NK, d, dv, causal)
    assert floats >= 2 * (2 * B * H * NQ * d) and floats < 2 * (B * HK * NK * (2 * d + dv))
    args, do = make(B, H, HK, NQ, NK, d, dv, seed=d + dv)
    check(gpu_lib, args, do, causal, None, kv_len)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,dv", [(32, 64), (64, 128), (96, 160), (128, 128), (96, 256), (128, 192), (128, 256)])
@pytest.mark.parametrize("G,NQ,q_len", [(8, 300, None), (2, 1100, [1100, 770])])
def test_key_gradients_from_ranges_of_rows(gpu_lib, d, dv, G, NQ, q_len, causal):
    """Many rows, of several heads, against few keys: the key-owned kernel has several ranges, the other one (seven key
    tiles)."""
    B, NK = (1 if q_len is None else 2), 201
    assert partial_floats(gpu_lib, B, G, 1, NQ, NK, d, dv, causal) >= 2 * (B * NK * (2 * d + dv))
    args, do = make(B, G, 1, NQ, NK, d, dv, seed=d + dv)
    check(gpu_lib, args, do, causal, q_len, None)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128)])
def test_square_maps_in_norm(gpu_lib, d, dv, causal):
    args, do = make(1, 2, 2, 256, 256, d, dv, seed=d)
    check(gpu_lib, args, do, causal)


# Terms g x r are off by a few roundings of 2^-24, r in common to a row; a lane adds up to about a hundred of them, 2048
# partial rows follow in runs of 32 and 64. Independent roundings, relative to the root of the sum of the squares: below
# sqrt(4 + 100 / 3) 2^-24 / sqrt(3) = 2.1e-7.
@pytest.mark.parametrize("B,N,H,HK,d,rot,dtype", [(1, 4096, 32, 8, 128, 128, torch.bfloat16), (4, 1021, 12, 12, 96, 64, torch.float32),
                                                  (1, 1, 1, 1, 64, 64, torch.float32), (2, 700, 3, 1, 256, 0, torch.float16)])
def test_norm_weight_gradients_are_as_exact_as_their_terms(gpu_lib, B, N, H, HK, d, rot, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda")   # noqa: E731
    q, k, w = mk(B, N, H, d).to(dtype), mk(B, N, HK, d).to(dtype), 1 + 0.2 * mk(2, d)
    table = gpu_lib.rope_table(N, rot) if rot else None
    dy = mk(B, H, N, d).bfloat16(), mk(B, HK, N, d).bfloat16()
    got = gpu_lib.qk_norm_rope_bwd(q, k, *dy, w[0], w[1], table)
    for x, g, dw in ((q, dy[0], got[2]), (k, dy[1], got[3])):
        x, g = x.double(), g.double().transpose(1, 2)
        if rot:
            c, s = (t[None, :, None] for t in table.double().split(rot // 2, 1))
            a, b = g[..., :rot // 2], g[..., rot // 2:rot]
            g = torch.cat((a * c + b * s, b * c - a * s, g[..., rot:]), -1)
        t = (g * x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)).flatten(0, 2)
        rel = (dw.double() - t.sum(0)) / t.square().sum(0).sqrt()
        rms = float(rel.square().mean().sqrt())
        print(f"dw {rms:.2e}", flush=True)
        assert rms <= 2.0 ** -22
