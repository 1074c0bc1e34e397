"""The oracle of the operators on rows of logits against torch float64 autograd and closed forms (CPU only)."""
import numpy as np
import pytest
import torch

from oracle import logits_oracle as lo


def rows(R, V, seed=0, spread=2.0):
    return np.random.default_rng(seed).normal(size=(R, V)) * spread


@pytest.mark.parametrize("scale", [1.0, 0.5, 1.7])
def test_token_logprobs_against_torch(scale):
    x = rows(5, 37)
    tokens = np.array([0, 36, -1, 5, -100])
    up = [np.random.default_rng(i).normal(size=5) for i in (1, 2, 3)]
    t = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(t * scale, -1)
    ent = -(lp.exp() * lp).sum(-1)
    lse = torch.logsumexp(t * scale, -1)
    kept = torch.tensor(tokens) >= 0
    logp = torch.where(kept, lp.gather(-1, torch.tensor(tokens).clamp_min(0)[:, None])[:, 0], 0.0)
    out = lo.token_logprobs(x, tokens, scale, 4)
    for name, ref in (("logp", logp), ("entropy", ent), ("lse", lse)):
        np.testing.assert_allclose(out[name][0], ref.detach().numpy(), rtol=1e-12, atol=1e-12)
    top = torch.topk(lp, 4)
    assert (out["top_ids"] == top.indices.numpy()).all()
    np.testing.assert_allclose(out["top_logp"][0], top.values.detach().numpy(), rtol=1e-12)
    sum((torch.tensor(u) * y).sum() for u, y in zip(up, (logp, ent, lse))).backward()
    dx, _ = lo.token_logprobs_grad(x, tokens, scale, *up)
    np.testing.assert_allclose(dx, t.grad.numpy(), rtol=1e-10, atol=1e-12)


def test_token_logprobs_closed_forms():
    """Uniform rows, one certain token, an empty row, equal logits by index."""
    V = 8
    x = np.zeros((4, V))
    x[1] = -np.inf
    x[1, 3] = 2.0
    x[2] = -np.inf
    x[3] = [1, 3, 2, 3, 0, 3, 1, 2]
    out = lo.token_logprobs(x, np.array([1, 3, 0, 9]), 1.0, 4)
    assert out["entropy"][0][0] == pytest.approx(np.log(V)) and out["entropy"][0][1] == 0 and out["entropy"][0][2] == 0
    assert out["logp"][0][1] == 0 and np.isneginf(out["logp"][0][2]) and np.isnan(out["logp"][0][3])
    assert np.isneginf(out["lse"][0][2])
    assert out["top_ids"][3].tolist() == [1, 3, 5, 2] and out["top_ids"][0].tolist() == [0, 1, 2, 3]
    dx, _ = lo.token_logprobs_grad(x, np.array([1, 3, 0, -1]), 1.0, np.ones(4), np.ones(4), np.ones(4))
    assert not dx[2].any() and np.isfinite(dx).all()


@pytest.mark.parametrize("rest,reverse", [(True, False), (True, True), (False, False)])
@pytest.mark.parametrize("twice", [False, True])
def test_distill_against_torch(rest, reverse, twice):
    R, V, K = 4, 23, 5
    rng = np.random.default_rng(4)
    x = rows(R, V, 3)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(R)])
    ids[1, 3:] = -1
    ids[2] = -1
    if twice:
        ids[0, 4] = ids[0, 1]
    t = np.log(rng.dirichlet(np.ones(K + 1), size=R)[:, :K])
    s1, s2 = (1.0, 0.7) if rest else (0.5, 0.7)
    g = rng.normal(size=R)
    xt = torch.tensor(x, requires_grad=True)
    lq = torch.log_softmax(xt * s2, -1)
    total = 0.0
    for r in range(R):
        k = ids[r] >= 0
        if not k.any():
            continue
        i, v = torch.tensor(ids[r][k]), torch.tensor(t[r][k])
        a, b = (v, lq[r][i]) if rest else (torch.log_softmax(s1 * v, -1), lq[r][i])
        if rest:
            out = torch.ones(V, dtype=torch.bool)
            out[i] = False
            a = torch.cat((a, torch.log(torch.clamp(1 - v.exp().sum(), min=lo.LEAST_REST))[None]))
            b = torch.cat((b, torch.logsumexp(lq[r][out], 0)[None]))
        if reverse:
            a, b = b, a
        total = total + g[r] * (a.exp() * (a - b)).sum()
    total.backward()
    loss, _, dx, _ = lo.distill(x, ids, t, s1, s2, rest, reverse, g)
    assert (g * loss).sum() == pytest.approx(float(total.detach()), rel=1e-10)
    np.testing.assert_allclose(dx, xt.grad.numpy(), rtol=1e-9, atol=1e-12)


def test_distill_closed_forms():
    """A student that agrees has no loss and no gradient; a list of the whole vocabulary leaves no rest; the full list
    without a rest is the plain divergence."""
    rng = np.random.default_rng(5)
    V, K = 12, 4
    x = rows(1, V, 6)
    lp = x - np.log(np.exp(x).sum())
    ids = np.argsort(-x, -1)[:, :K]
    for reverse in (False, True):
        loss, _, dx, _ = lo.distill(x, ids, np.take_along_axis(lp, ids, -1), 1.0, 1.0, True, reverse)
        assert abs(loss[0]) < 1e-12 and np.abs(dx).max() < 1e-12
    t = np.log(rng.dirichlet(np.ones(V)))[None]
    every = np.arange(V)[None]
    plain = (np.exp(t) * (t - lp)).sum()
    for rest in (True, False):
        loss, _, dx, _ = lo.distill(x, every, t, 1.0, 1.0, rest, False)
        assert loss[0] == pytest.approx(plain, rel=1e-9)
        np.testing.assert_allclose(dx, np.exp(lp) - np.exp(t), atol=1e-12)


def test_distill_gradient_against_differences():
    rng = np.random.default_rng(7)
    V, K, h = 9, 3, 1e-6
    x = rows(1, V, 8)
    ids = rng.permutation(V)[:K][None]
    t = np.log(rng.dirichlet(np.ones(K + 1)))[None, :K]
    for rest, reverse in ((True, False), (True, True), (False, False)):
        _, _, dx, _ = lo.distill(x, ids, t, 1.0, 0.8, rest, reverse)
        for j in range(V):
            up, dn = x.copy(), x.copy()
            up[0, j] += h
            dn[0, j] -= h
            d = (lo.distill(up, ids, t, 1.0, 0.8, rest, reverse)[0] - lo.distill(dn, ids, t, 1.0, 0.8, rest, reverse)[0])
            assert dx[0, j] == pytest.approx(d[0] / (2 * h), abs=1e-7)
