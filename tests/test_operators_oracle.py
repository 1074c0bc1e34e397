"""The plain fp64 forms of norm-and-rotation and differential attention against independent ones (CPU only): torch
fp64 autograd, central differences, closed forms."""
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo


def rng(seed):
    return np.random.default_rng(seed)


def table(n, rot, base=10000.0):
    a = np.arange(n)[:, None] * base ** (-np.arange(0, rot, 2) / rot)
    return np.concatenate([np.cos(a), np.sin(a)], 1)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 32])
@pytest.mark.parametrize("copies", [1, 3])
def test_norm_rope_against_complex_products(interleaved, rot, copies):
    r = rng(1)
    B, N, H, d, eps = 2, 5, 3, 32, 1e-5
    x, w, tab, pos = r.normal(size=(B, N, H, d)), r.normal(size=d), table(40, rot) if rot else None, r.integers(0, 40, (B, N))
    y, _ = oo.norm_rope(x, w, tab, pos, eps, interleaved, copies)
    dy = r.normal(size=y.shape)
    tx, tw = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    z = tx / torch.sqrt((tx ** 2).mean(-1, keepdim=True) + eps) * tw
    if rot:
        t = torch.tensor(tab[pos])[:, :, None]
        turn = torch.complex(t[..., :rot // 2], t[..., rot // 2:])
        u = torch.complex(z[..., 0:rot:2], z[..., 1:rot:2]) if interleaved else \
            torch.complex(z[..., :rot // 2], z[..., rot // 2:rot])
        u = u * turn
        head = torch.stack((u.real, u.imag), -1).flatten(-2) if interleaved else torch.cat((u.real, u.imag), -1)
        z = torch.cat((head, z[..., rot:]), -1)
    ref = z.permute(0, 2, 1, 3).repeat_interleave(copies, 1)
    np.testing.assert_allclose(y, ref.detach().numpy(), rtol=1e-12, atol=1e-13)
    dx, _, dw, _ = oo.norm_rope_backward(x, w, tab, pos, eps, dy, interleaved, copies)
    gx, gw = torch.autograd.grad(ref, (tx, tw), torch.tensor(dy))
    np.testing.assert_allclose(dx, gx.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(dw, gw.numpy(), rtol=1e-10, atol=1e-12)


def test_norm_rope_gradient_against_differences():
    r = rng(2)
    x, w, tab, pos = r.normal(size=(1, 3, 2, 32)), r.normal(size=32), table(9, 16), np.array([0, 4, 8])
    dy = r.normal(size=(1, 2, 3, 32))
    dx, _, dw, _ = oo.norm_rope_backward(x, w, tab, pos, 1e-3, dy)
    f = lambda a, b: (oo.norm_rope(a, b, tab, pos, 1e-3)[0] * dy).sum()   # noqa: E731
    h = 1e-6
    for idx in ((0, 0, 0, 0), (0, 1, 1, 9), (0, 2, 0, 31)):
        e = np.zeros_like(x)
        e[idx] = h
        assert math.isclose((f(x + e, w) - f(x - e, w)) / (2 * h), dx[idx], rel_tol=1e-6, abs_tol=1e-8)
    for j in (0, 7, 20):
        e = np.zeros_like(w)
        e[j] = h
        assert math.isclose((f(x, w + e) - f(x, w - e)) / (2 * h), dw[j], rel_tol=1e-6, abs_tol=1e-8)


def test_rotation_keeps_relative_positions():
    """q . k after the rotation depends on the distance of their positions alone."""
    r = rng(3)
    x, z, tab = r.normal(size=(1, 1, 1, 32)), r.normal(size=(1, 1, 1, 32)), table(64, 32)
    dots = [(oo.norm_rope(x, None, tab, [p + 7], 1e-6)[0] * oo.norm_rope(z, None, tab, [p], 1e-6)[0]).sum()
            for p in (0, 13, 50)]
    np.testing.assert_allclose(dots, dots[0], rtol=1e-10)


CASES = [(2, 4, 2, 7, 9, True, None, None), (1, 3, 1, 9, 7, True, None, None), (2, 2, 2, 6, 6, False, [4, 0], [5, 3]),
         (2, 2, 1, 8, 8, True, [8, 3], [8, 3]), (1, 1, 1, 1, 1, True, None, None)]


def diff_inputs(case, d=32, dv=32, seed=4):
    B, H, HK, nq, nk, causal, ql, kl = case
    r = rng(seed)
    q1, q2 = r.normal(size=(2, B, H, nq, d))
    k1, k2 = r.normal(size=(2, B, HK, nk, d))
    return (q1, k1, q2, k2, r.normal(size=(B, HK, nk, dv)), r.uniform(-1, 1, H)), r.normal(size=(B, H, nq, dv)), causal, ql, kl


@pytest.mark.parametrize("case", CASES)
def test_diff_against_torch_autograd(case):
    args, do, causal, ql, kl = diff_inputs(case)
    B, H, HK, nq, nk = case[:5]
    scale = 0.3
    res, _ = oo.diff(*args, scale, causal, ql, kl)
    g, _ = oo.diff_backward(*args, scale, causal, do, ql, kl)
    t = [torch.tensor(x, requires_grad=True) for x in args]
    q1, k1, q2, k2, v, lam = t
    ex = lambda x: x.repeat_interleave(H // HK, 1)   # noqa: E731
    ok = torch.tensor(np.stack([oo.visible(nq, nk, nq if ql is None else ql[b], nk if kl is None else kl[b], causal)
                                for b in range(B)]))[:, None]

    def attend(q, k):
        z = (scale * q @ ex(k).transpose(2, 3)).masked_fill(~ok, -1e30)
        return torch.softmax(z, -1) * ok

    out = (attend(q1, k1) - lam[None, :, None, None] * attend(q2, k2)) @ ex(v)
    np.testing.assert_allclose(res["out"], out.detach().numpy(), rtol=1e-10, atol=1e-12)
    for n, r in zip(("dq1", "dk1", "dq2", "dk2", "dv", "dlam"), torch.autograd.grad(out, t, torch.tensor(do))):
        np.testing.assert_allclose(g[n], r.numpy(), rtol=1e-9, atol=1e-11, err_msg=n)


def test_diff_gradients_against_differences():
    args, do, causal, ql, kl = diff_inputs((1, 2, 1, 5, 6, True, [4], [5]))
    g, _ = oo.diff_backward(*args, 0.4, causal, do, ql, kl)
    f = lambda a: (oo.diff(*a, 0.4, causal, ql, kl)[0]["out"] * do).sum()   # noqa: E731
    h = 1e-6
    for n, i, idx in (("dq1", 0, (0, 1, 3, 5)), ("dk1", 1, (0, 0, 2, 8)), ("dq2", 2, (0, 0, 2, 0)),
                      ("dk2", 3, (0, 0, 4, 31)), ("dv", 4, (0, 0, 1, 3)), ("dlam", 5, (1,))):
        up, down = [list(x.copy() for x in args) for _ in range(2)]
        up[i][idx] += h
        down[i][idx] -= h
        assert math.isclose((f(up) - f(down)) / (2 * h), g[n][idx], rel_tol=1e-6, abs_tol=1e-8), n


def test_diff_closed_forms():
    """Equal maps and lam = 1 cancel; lam = 0 is plain attention; zero queries average the values."""
    (q1, k1, _, _, v, _), _, _, _, _ = diff_inputs((1, 2, 1, 4, 5, False, None, None))
    same, _ = oo.diff(q1, k1, q1, k1, v, np.ones(2), 0.5, False)
    np.testing.assert_allclose(same["out"], 0.0, atol=1e-15)
    flat, _ = oo.diff(0 * q1, k1, q1, k1, v, np.zeros(2), 0.5, False)
    np.testing.assert_allclose(flat["out"], np.broadcast_to(v.mean(2)[:, :, None], flat["out"].shape), rtol=1e-12)
    np.testing.assert_allclose(flat["lse1"], math.log(5), rtol=1e-12)


def test_empty_rows():
    args, do, _, _, _ = diff_inputs((2, 2, 1, 6, 3, True, None, None))
    res, _ = oo.diff(*args, 0.4, True, None, [0, 3])
    g, _ = oo.diff_backward(*args, 0.4, True, do, None, [0, 3])
    assert not res["out"][0].any() and np.isneginf(res["lse1"][0]).all()
    assert not res["out"][1, :, :3].any() and res["out"][1, :, 3:].any()
    assert not any(g[n][0].any() for n in ("dq1", "dk1", "dq2", "dk2", "dv"))
