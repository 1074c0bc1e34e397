"""Rows of logits at the ends of what the operators take: values far from zero, tokens outside the vocabulary, NaN in lists,
outputs that are edited in place, how exact long sums are."""
import numpy as np
import pytest
import torch

from oracle import logits_oracle as lo
from test_gpu_token_logprobs import HALF, TINY, check_fwd, logits, near, np64

pytestmark = pytest.mark.gpu


def f32(v):
    """A scale as the kernels hold it."""
    return float(np.float32(v))


def far_rows(V, dtype, seed=0):
    """Nine rows: of the type's lowest and largest value, of equal values far from zero, of noise around such values (which
    the type rounds to a few of its numbers), half of the lowest value, and noise."""
    top = torch.finfo(dtype).max
    far = (-60000.0, -30000.0, 2.0 ** 14, 2.0 ** 12) if dtype is torch.float16 else (-1e30, -1e12, 2.0 ** 60, 2.0 ** 26)
    noise = logits(9, V, torch.float32, seed=seed)
    x = noise.clone()
    x[0], x[1], x[2], x[3] = -top, top, far[0], far[1]
    x[4] = far[2]
    x[4, ::3] = far[2] / 2
    x[5] += far[3]
    x[6] -= min(2.0 ** 24, top / 4)
    x[7, ::2] = -top
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("scale", [1.0, 0.9, 2.0 / 3.0, 0.6, 0.3])
@pytest.mark.parametrize("V", [5, 1000, 70001])
def test_gradients_of_rows_far_from_zero(gpu_lib, V, scale, dtype):
    """The log-sum-exp of such a row does not hold what its probabilities are, nor does any number added to it."""
    x, scale = far_rows(V, dtype), f32(scale)
    tokens = torch.tensor([0, 1, V - 1, 2, 0, 3, 4, 2, -1], device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(V)
    up = [torch.randn(9, generator=gen, device="cuda") for _ in range(3)]
    xg = x.clone().requires_grad_(True)
    y = gpu_lib.token_logprobs(xg, tokens, scale=scale)
    dx, = torch.autograd.grad((y.logp, y.entropy, y.lse), xg, up)
    ref, bound = lo.token_logprobs_grad(np64(x), tokens.cpu().numpy(), scale, *(np64(u) for u in up))
    near(dx, (ref, bound + HALF[dtype] * np.abs(ref) + TINY[dtype]), "dx")
    z, err = gpu_lib.token_logprobs_fwd(x, tokens, scale, save=True)
    same = gpu_lib.token_logprobs_bwd(x, tokens, z.lse, err, z.entropy, *up, scale=scale, out=x)   # in place
    assert same is x and torch.equal(x, dx)


@pytest.mark.parametrize("teacher", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("s1", [1.0, 0.7, 0.3])
@pytest.mark.parametrize("R", [5, 600])
def test_teacher_logits_far_from_zero(gpu_lib, R, s1, teacher):
    """Lists of the type's lowest value are uniform, as rows of it are; lists around a value far from zero."""
    V, K, s1 = 3001, 7, f32(s1)
    gen = torch.Generator(device="cuda").manual_seed(R)
    x = logits(R, V, torch.float32, seed=R)
    ids = torch.stack([torch.randperm(V, generator=gen, device="cuda")[:K] for _ in range(R)])
    t = torch.randn(R, K, generator=gen, device="cuda").to(teacher)
    low = torch.finfo(teacher).min
    t[0] = low
    t[1, 2:] = low
    t[2] = low
    t[2, 3] = low / 2
    t[3] = low / 4
    ids[3, 5:] = -1
    g = torch.ones(R, device="cuda")
    xg = x.requires_grad_(True)
    y = gpu_lib.topk_distill(xg, ids, t, s1=s1, rest=False)
    dx, = torch.autograd.grad(y, xg, g)
    loss, lb, ref, db = lo.distill(np64(x), ids.cpu().numpy(), np64(t), s1, 1.0, False, False)
    near(y, (loss, lb), "loss")
    near(dx, (ref, db + HALF[torch.float32] * np.abs(ref)), "dx")
    for bad in (-torch.inf, torch.inf, torch.nan):
        t[0] = bad   # a list of nothing, or of no numbers, is no distribution
        y = gpu_lib.topk_distill(x.detach(), ids, t, s1=s1, rest=False)
        assert torch.isnan(y[0]) and torch.isfinite(y[1:]).all()


@pytest.mark.parametrize("which", ["entropy", "lse", "dlogp 0"])
def test_a_token_outside_the_vocabulary_spoils_its_log_probability_only(gpu_lib, which):
    """Entropies and log-sum-exps do not depend on the token, nor do their gradients."""
    V, R = 3001, 6
    x = logits(R, V, torch.float32, seed=5).requires_grad_(True)
    tokens = torch.tensor([1, V, V + 7, -1, 1 << 40, 3], device="cuda")
    out = (1, 2, 4)
    y = gpu_lib.token_logprobs(x, tokens)
    one, zero = torch.ones(R, device="cuda"), torch.zeros(R, device="cuda")
    outputs, up = {"entropy": ((y.entropy,), (one,)), "lse": ((y.lse,), (one,)),
                   "dlogp 0": ((y.logp, y.entropy), (torch.where(tokens < V, 1.0, 0.0), one))}[which]
    dx, = torch.autograd.grad(outputs, x, up, retain_graph=True)
    g = np64(up[0]) if which == "dlogp 0" else None
    h, e = (None, np.ones(R)) if which == "lse" else (np.ones(R), None)
    ref, bound = lo.token_logprobs_grad(np64(x), np.where(np64(tokens) < V, np64(tokens), -1).astype(np.int64), 1.0, g, h, e)
    near(dx, (ref, bound + HALF[torch.float32] * np.abs(ref)), "dx")
    dx, = torch.autograd.grad((y.logp, y.entropy), x, (one, zero))   # and its own gradient with it
    bad = torch.isnan(dx).all(-1)
    assert bad[list(out)].all() and torch.isfinite(dx[[0, 3, 5]]).all()


def test_a_finished_gradient_is_not_in_the_place_of_the_logits(gpu_lib):
    """An in-place step and then a loss scale: the logits that the second pass would read are gone."""
    x = logits(4, 300, torch.float32, seed=3)
    ids = torch.arange(6, dtype=torch.int32, device="cuda").expand(4, 6).contiguous()
    t = torch.full((4, 6), -2.0, device="cuda")
    logit = x.clone()
    loss, stats, dx = gpu_lib.topk_distill_step(logit, ids, t, out=logit)
    three = torch.full((1,), 3.0, device="cuda")
    keep = dx.clone()
    with pytest.raises(ValueError):
        gpu_lib.topk_distill_bwd(logit, ids, t, stats, dfactor=three, done_if_one=True, out=logit)
    assert torch.equal(logit, keep)
    gpu_lib.topk_distill_bwd(x, ids, t, stats, dfactor=three, done_if_one=True, out=logit)   # from the logits it does
    near(logit, (3.0 * np64(keep), 2.0 ** -20 * np.abs(3.0 * np64(keep))), "dx")


@pytest.mark.parametrize("N", [3, 700])
def test_outputs_are_edited_in_place(gpu_lib, N):
    """Outputs of one call are tensors of their own: editing one neither needs nor touches the others."""
    x = logits(N, 1000, torch.float32, seed=6).requires_grad_(True)
    tokens = torch.arange(N, device="cuda") % 1000
    ref = gpu_lib.token_logprobs(x.detach(), tokens)
    keep = tokens % 2 == 0
    y = gpu_lib.token_logprobs(x, tokens)
    y.logp.masked_fill_(~keep, 0.0)
    y.logp.mul_(2.0)
    assert torch.equal(y.logp, torch.where(keep, 2.0 * ref.logp, 0.0))
    assert torch.equal(y.entropy, ref.entropy) and torch.equal(y.lse, ref.lse)
    dx, = torch.autograd.grad(y.logp.sum() + y.entropy.sum(), x)
    z = gpu_lib.token_logprobs(x, tokens)
    same, = torch.autograd.grad((2.0 * z.logp[keep]).sum() + z.entropy.sum(), x)
    assert torch.equal(dx, same)
    with torch.no_grad():
        z = gpu_lib.token_logprobs(x, tokens)
        z.logp.zero_()
        assert torch.equal(z.lse, ref.lse)
    w = torch.ones(N, device="cuda", requires_grad=True)
    z = gpu_lib.token_logprobs(x.detach(), tokens)
    z.logp.mul_(w)   # weights that are trained, on scores that are not
    assert torch.equal(torch.autograd.grad(z.logp.sum(), w)[0], ref.logp)


@pytest.mark.parametrize("rest,direction", [(True, "fwd"), (True, "rev"), (False, "fwd")])
@pytest.mark.parametrize("R", [3, 600])
def test_an_id_outside_the_vocabulary_spoils_an_empty_row_too(gpu_lib, R, rest, direction):
    """Loss and gradient alike; without it the row has no loss."""
    V, K = 2003, 4
    x = logits(R, V, torch.float32, seed=7)
    x[:2] = -torch.inf
    ids = torch.arange(K, device="cuda").expand(R, K).contiguous()
    ids[1, 2] = V
    t = torch.full((R, K), -2.0, device="cuda")
    opts = dict(rest=rest, direction=direction)
    loss, stats, dx = gpu_lib.topk_distill_step(x, ids, t, **opts)
    back = gpu_lib.topk_distill_bwd(x, ids, t, stats, **opts)
    for g in (dx, back):
        assert loss[0] == 0 and not g[0].any()
        assert torch.isnan(loss[1]) and torch.isnan(g[1]).all()
        assert torch.isfinite(loss[2:]).all() and torch.isfinite(g[2:]).all()


@pytest.mark.parametrize("direction", ["fwd", "rev"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("R,V", [(4, 1), (4, 2003), (600, 2003)])
def test_a_listed_logit_that_is_none_beside_nothing(gpu_lib, R, V, value, direction):
    """A row of -inf but for a NaN or +inf in its list is spoilt, not empty, whatever its teacher's value."""
    x = torch.full((R, V), -torch.inf, device="cuda")
    x[1:, V // 2] = 2.0
    x[0, V // 2] = value
    ids = torch.full((R, 2), -1, dtype=torch.int32, device="cuda")
    ids[:, 1] = V // 2
    t = torch.full((R, 2), -0.5, device="cuda")
    for w, v in ((1.0, -0.5), (0.0, -0.5), (1.0, -torch.inf), (0.0, -torch.inf)):
        g = torch.ones(R, device="cuda")
        g[0], t[0] = w, v
        loss, stats, dx = gpu_lib.topk_distill_step(x, ids, t, g, direction=direction)
        back = gpu_lib.topk_distill_bwd(x, ids, t, stats, g, direction=direction)
        assert torch.isnan(loss[0]) and torch.isfinite(loss[1:]).all()
        for d in (dx, back):
            assert (torch.isnan(d[0]).all() if w else not d[0].any()) and torch.isfinite(d[1:]).all()


def model_rows(R, V, dtype, seed):
    """Rows as a language model has them: a broad floor, and 32 tokens that hold most of the mass."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")   # noqa: E731
    x = normal(R, V) * 2.5
    ids = (torch.randint(0, V, (R, 1), generator=gen, device="cuda") + 3001 * torch.arange(32, device="cuda")) % V
    score = -1.2 * torch.log(torch.arange(1, 33, device="cuda")) + 0.3 * normal(R, 32)
    x.scatter_(1, ids, torch.log_softmax(score, -1) + float(np.log(V) + 0.5 * 2.5 ** 2 + np.log(5.0)) + 0.4 * normal(R, 32))
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,V", [(96, 100003), (520, 128000)])
def test_how_exact_long_sums_are(gpu_lib, R, V, dtype):
    """Errors in norm over rows of a model, in parts and whole. A result is rounded to 24 bits, 0.3 U of it in norm (U =
    2^-24). What holds most of a row's mass passes some 25 roundings of 0.3 U each, in all directions, in both sums of an
    entropy, l and a, where that of a counts with the 3 nats that the reference may be off: 0.3 U sqrt(25) sqrt(2) 3 = 6 U,
    of entropies near 4: 1.6 U. Three times that has to hold. One chain of all terms of a lane with references up to 24
    doublings off comes to 13 to 17 U in the long rows."""
    n, K, U = 96, 32, 2.0 ** -24
    x = model_rows(R, V, dtype, V)
    tokens = torch.arange(R, device="cuda") * 97 % V
    y = gpu_lib.token_logprobs(x, tokens)
    ref = lo.token_logprobs(np64(x[:n]), tokens[:n].cpu().numpy(), 1.0, 0)
    for name in ("logp", "entropy", "lse"):
        value = ref[name][0]
        assert np.linalg.norm(np64(getattr(y, name)[:n]) - value) <= 5 * U * np.linalg.norm(value), name
    best = gpu_lib.token_logprobs(model_rows(R, V, torch.float32, V + 1), top=K)
    for rest, direction in ((True, "fwd"), (True, "rev"), (False, "fwd")):
        loss = gpu_lib.topk_distill(x, best.top_ids, best.top_logp, rest=rest, direction=direction)[:n]
        value = lo.distill(np64(x[:n]), best.top_ids[:n].cpu().numpy(), np64(best.top_logp[:n]), 1.0, 1.0, rest,
                           direction == "rev")[0]
        assert np.linalg.norm(np64(loss) - value) <= 5 * U * np.linalg.norm(value), (rest, direction)


def test_the_gradient_of_the_loss_passes_saved_tensor_hooks(gpu_lib):
    """What topk_distill_loss keeps of the logits' size goes through save_for_backward: an offloading hook sees it, and a
    checkpointed loss keeps none of it."""
    R, V, K = 300, 5003, 8
    x = logits(R, V, torch.float32, seed=8).requires_grad_(True)
    best = gpu_lib.token_logprobs(logits(R, V, torch.float32, seed=9), top=K)
    w = torch.rand(R, device="cuda")
    args = (best.top_ids, best.top_logp, w)
    ref, = torch.autograd.grad(gpu_lib.topk_distill_loss(x, *args), x)
    seen = []

    def pack(t):
        seen.append(t.shape)
        return t.cpu()

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        y = gpu_lib.topk_distill_loss(x, *args)
    assert seen.count((R, V)) == 2   # logits and gradient
    for up in (1.0, 3.0):   # handed over, and formed anew
        dx, = torch.autograd.grad(y, x, torch.tensor(up, device="cuda"), retain_graph=True)
        near(dx, (up * np64(ref), 2.0 ** -20 * np.abs(up * np64(ref))), "dx")
    before = torch.cuda.memory_allocated()
    y = torch.utils.checkpoint.checkpoint(gpu_lib.topk_distill_loss, x, *args, use_reentrant=False)
    assert torch.cuda.memory_allocated() - before < x.numel() * 4 // 2
    dx, = torch.autograd.grad(y, x)
    assert torch.equal(dx, ref)


def test_a_gradient_that_was_handed_over_is_the_callers(gpu_lib):
    """Editing it leaves a retained graph alone, and accumulating into a leaf makes no copy of it."""
    R, V, K = 300, 5003, 8
    x = logits(R, V, torch.float32, seed=8).requires_grad_(True)
    best = gpu_lib.token_logprobs(logits(R, V, torch.float32, seed=9), top=K)
    y = gpu_lib.topk_distill_loss(x, best.top_ids, best.top_logp)
    before = torch.cuda.memory_allocated()
    y.backward(retain_graph=True)
    assert torch.cuda.memory_allocated() - before < x.numel() * 4 // 2   # the gradient was there
    first = x.grad.clone()
    x.grad.zero_()
    y.backward()
    near(x.grad, (np64(first), 2.0 ** -20 * np.abs(np64(first))), "dx")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("scale", [0.9, 0.6, 0.3])
@pytest.mark.parametrize("V", [150, 1000, 70001])
def test_values_of_rows_far_from_zero(gpu_lib, V, scale, dtype):
    """Log probabilities, entropies, best tokens; losses on them and their gradients in both directions."""
    x, scale = far_rows(V, dtype), f32(scale)
    tokens = torch.tensor([0, 1, V - 1, 2, 0, 3, 4, 2, -1], device="cuda")
    check_fwd(gpu_lib, x, tokens, scale, 9)
    gen = torch.Generator(device="cuda").manual_seed(V)
    ids = torch.stack([torch.randperm(V, generator=gen, device="cuda")[:6] for _ in range(9)])
    t = torch.log_softmax(torch.randn(9, 8, generator=gen, device="cuda"), -1)[:, :6].contiguous()
    for rest, direction in ((True, "fwd"), (True, "rev"), (False, "fwd")):
        opts = dict(s2=scale, rest=rest, direction=direction)
        loss, stats, dx = gpu_lib.topk_distill_step(x, ids, t, **opts)
        back = gpu_lib.topk_distill_bwd(x, ids, t, stats, **opts)
        value, lb, ref, db = lo.distill(np64(x), ids.cpu().numpy(), np64(t), 1.0, scale, rest, direction == "rev")
        near(loss, (value, lb), "loss")
        for g in (dx, back):
            near(g, (ref, db + HALF[dtype] * np.abs(ref) + TINY[dtype]), "dx")
