"""topk_distill and topk_distill_loss against the 64-bit oracle: losses, gradients, lists, layouts, what autograd asks."""
import math

import numpy as np
import pytest
import torch
from torch.autograd import forward_ad as fw

from oracle import logits_oracle as lo

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
MODES = [(True, "fwd"), (True, "rev"), (False, "fwd")]


def np64(t):
    return t.detach().double().cpu().numpy()


def near(got, value, bound, name):
    got = np64(got)
    bad = ~((np.abs(got - value) <= bound) | (got == value) | (np.isnan(got) & np.isnan(value)))
    assert not bad.any(), (name, got[bad][:4], value[bad][:4], np.broadcast_to(bound, got.shape)[bad][:4])


def make(R, V, K, dtype=torch.bfloat16, seed=0, teacher=torch.float32, ragged=False, ids_type=torch.int32):
    """Logits near a teacher's distribution over K distinct tokens and a rest."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(R, V)) * 2.0
    ids = np.stack([rng.permutation(V)[:K] for _ in range(R)])
    share = rng.dirichlet(np.ones(K + 1) * 0.7, size=R) + 1e-6
    share /= share.sum(-1, keepdims=True)
    t = np.log(share[:, :K])
    base = math.log(V) + 2.0 - np.log(share[:, K:])
    np.put_along_axis(x, ids, t + base + 0.5 * rng.normal(size=(R, K)), -1)
    if ragged:
        for r in range(R):
            ids[r, rng.integers(0, K + 1):] = -1 - r
    return (torch.tensor(x, device="cuda").to(dtype), torch.tensor(ids, device="cuda").to(ids_type),
            torch.tensor(t, device="cuda").to(teacher))


def check(sk, x, ids, t, s1, s2, rest, direction, g):
    """Rows [R, V]: losses and gradients of topk_distill, of its step, and of the loss."""
    opts = dict(s1=s1, s2=s2, rest=rest, direction=direction)
    loss, lb, dx, db = lo.distill(np64(x), ids.cpu().numpy(), np64(t), s1, s2, rest, direction == "rev", np64(g))
    db = db + HALF[x.dtype] * np.abs(dx) + TINY[x.dtype]
    xg = x.detach().requires_grad_(True)
    y = sk.topk_distill(xg, ids, t, **opts)
    near(y, loss, lb, "loss")
    got, = torch.autograd.grad(y, xg, g)
    near(got, dx, db, "dx")
    total = sk.topk_distill_loss(xg, ids, t, g, **opts)
    live = np64(g) != 0
    near(total, (loss * np64(g))[live].sum(), (lb * np.abs(np64(g)))[live].sum() + 2.0 ** -23 * abs((loss * np64(g))[live].sum()),
         "total")
    got, = torch.autograd.grad(total, xg)
    near(got, dx, db, "dx of the loss")
    return y


@pytest.mark.parametrize("rest,direction", MODES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("V,K,R", [(2, 1, 3), (5, 4, 4), (9, 8, 5), (100, 64, 3), (1000, 1, 40), (1003, 128, 7),
                                   (4099, 17, 600), (50257, 20, 5), (131072, 64, 3), (262144, 32, 2), (300001, 100, 3)])
def test_values_and_gradients(gpu_lib, V, K, R, dtype, rest, direction):
    x, ids, t = make(R, V, K, dtype, seed=V + K, ragged=K > 4)
    g = torch.randn(R, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    check(gpu_lib, x, ids, t, 1.0 if rest else 0.7, 0.9, rest, direction, g)


@pytest.mark.parametrize("rest,direction", MODES)
@pytest.mark.parametrize("teacher", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ids_type", [torch.int32, torch.int64])
def test_types_of_lists(gpu_lib, ids_type, teacher, rest, direction):
    x, ids, t = make(9, 777, 12, seed=3, teacher=teacher, ids_type=ids_type)
    check(gpu_lib, x, ids, t, 1.0, 1.0, rest, direction, torch.ones(9, device="cuda"))


@pytest.mark.parametrize("rest,direction", MODES)
@pytest.mark.parametrize("R", [4, 700])
def test_the_same_token_twice(gpu_lib, R, rest, direction):
    x, ids, t = make(R, 3001, 9, torch.float32, seed=5)
    ids[:, 4] = ids[:, 1]
    ids[0] = ids[0, 0]
    t = t - math.log(2)
    check(gpu_lib, x, ids, t, 1.0, 1.0, rest, direction, torch.ones(R, device="cuda"))


@pytest.mark.parametrize("rest,direction", MODES)
def test_lists_of_the_whole_vocabulary_and_of_nothing(gpu_lib, rest, direction):
    V = 37
    x = torch.randn(6, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    ids = torch.arange(V, device="cuda").expand(6, V).contiguous()
    t = torch.log_softmax(torch.randn(6, V, device="cuda"), -1)
    ids[4] = -1
    ids[5, 1:] = -7
    y = check(gpu_lib, x, ids, t, 1.0, 1.0, rest, direction, torch.ones(6, device="cuda"))
    assert y[4] == 0


@pytest.mark.parametrize("direction", ["fwd", "rev"])
@pytest.mark.parametrize("R", [3, 600])
def test_a_student_that_is_sure_keeps_its_rest(gpu_lib, R, direction):
    """The mass outside the list is far below the rounding of 1."""
    x, ids, t = make(R, 5000, 8, torch.float32, seed=6)
    x.scatter_(1, ids.long(), (40.0 + torch.arange(8, device="cuda") / 8).expand(R, 8))
    y = check(gpu_lib, x, ids, t, 1.0, 1.0, True, direction, torch.ones(R, device="cuda"))
    assert torch.isfinite(y).all() and (y > 0).all()   # a divergence of unequal distributions


@pytest.mark.parametrize("rest,direction", MODES)
def test_a_student_that_agrees_has_no_loss(gpu_lib, rest, direction):
    x = torch.randn(5, 2000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) * 3
    best = gpu_lib.token_logprobs(x, top=50)
    check(gpu_lib, x, best.top_ids, best.top_logp, 1.0, 1.0, rest, direction, torch.ones(5, device="cuda"))
    y = gpu_lib.topk_distill(x, best.top_ids, best.top_logp, rest=True, direction=direction)
    assert y.abs().max() < 1e-6   # a few roundings of log probabilities near 5, second order in the loss


@pytest.mark.parametrize("rest,direction", MODES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R", [6, 600])
def test_masked_logits(gpu_lib, R, dtype, rest, direction):
    """-inf outside the list, everywhere outside it, the type's lowest value, rows of -inf."""
    V, K = 2003, 6
    x, ids, t = make(R, V, K, dtype, seed=8)
    low = torch.finfo(dtype).min
    x[0, :500] = -torch.inf
    x[0].scatter_(0, ids[0].long(), 1.0)
    kept = x[1].gather(0, ids[1].long())
    x[1] = -torch.inf
    x[1].scatter_(0, ids[1].long(), kept)
    x[2] = -torch.inf
    x[3, 100:1500] = low
    x[3].scatter_(0, ids[3].long(), 2.0)
    x[4] = low
    y = check(gpu_lib, x, ids, t, 1.0, 1.0, rest, direction, torch.ones(R, device="cuda"))
    assert torch.isfinite(y).all() and y[2] == 0


def test_a_listed_token_of_probability_0(gpu_lib):
    x, ids, t = make(3, 500, 4, torch.float32, seed=9)
    x[1, ids[1, 2]] = -torch.inf
    for rest in (True, False):
        y = gpu_lib.topk_distill(x, ids, t, rest=rest)
        assert torch.isinf(y[1]) and y[1] > 0 and torch.isfinite(y[[0, 2]]).all()
    y = gpu_lib.topk_distill(x, ids, t, direction="rev")
    assert torch.isfinite(y).all()
    t[0, 1] = -torch.inf   # the teacher rules it out
    y = gpu_lib.topk_distill(x, ids, t)
    assert torch.isfinite(y[0])
    assert torch.isinf(gpu_lib.topk_distill(x, ids, t, direction="rev")[0])


@pytest.mark.parametrize("rest,direction", MODES)
@pytest.mark.parametrize("R", [3, 600])
def test_what_spoils_a_row_spoils_no_other(gpu_lib, R, rest, direction):
    x, ids, t = make(R, 9001, 8, seed=10)
    opts = dict(rest=rest, direction=direction)
    g = torch.ones(R, device="cuda")
    clean, stats, dx = gpu_lib.topk_distill_step(x, ids, t, g, **opts)
    keep = torch.arange(R, device="cuda") != 1
    for k in range(3):
        x2, ids2, t2 = x.clone(), ids.clone(), t.clone()
        if k == 0:
            x2[1, 55] = float("nan")
        elif k == 1:
            ids2[1, 3] = 9001
        else:
            t2[1, 3] = float("nan")
        for w in (1.0, 0.0):
            g[1] = w
            loss, _, bad = gpu_lib.topk_distill_step(x2, ids2, t2, g, **opts)
            assert torch.equal(loss[keep], clean[keep]) and torch.equal(bad[keep], dx[keep])
            if w:
                assert torch.isnan(loss[1]) and torch.isnan(bad[1]).all()
            else:   # padding: left out of the sum, no gradient
                assert not bad[1].any()
                xg = x2.requires_grad_(True)
                total = gpu_lib.topk_distill_loss(xg, ids2, t2, g, **opts)
                assert torch.isfinite(total) and not torch.autograd.grad(total, xg)[0][1].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layouts(gpu_lib, dtype):
    V, K = 1003, 10
    pad = torch.full((3, 8, V + 21), float("nan"), dtype=dtype, device="cuda")
    x, ids, t = make(21, V, K, dtype, seed=11)
    g = torch.randn(3, 7, device="cuda")
    ref = [a.view(3, 7, *a.shape[1:]) for a in gpu_lib.topk_distill_step(x, ids, t, g.view(-1))]
    for first in range(0, 21, 5):
        pad.fill_(float("nan"))
        view = pad[:, :-1, first:first + V]
        view.copy_(x.view(3, 7, V))
        loss, _, dx = gpu_lib.topk_distill_step(view, ids.view(3, 7, K), t.view(3, 7, K), g)
        assert loss.shape == (3, 7) and dx.shape == (3, 7, V) and dx.is_contiguous()
        # the same sums in another order
        near(loss, np64(ref[0]), 2.0 ** -18 * (1 + np.abs(np64(ref[0]))), "loss")
        near(dx, np64(ref[2]), (2 * HALF[dtype] + 2.0 ** -16) * np.abs(np64(ref[2])) + 1e-9, "dx")


def test_gradients_in_place_and_beside_other_data(gpu_lib):
    for dtype in (torch.bfloat16, torch.float32):
        for rest, direction in MODES:
            for R in (3, 600):
                V = 9003
                x, ids, t = make(R, V, 20, dtype, seed=12)
                g = torch.randn(R, device="cuda")
                opts = dict(rest=rest, direction=direction)
                loss, stats, ref = gpu_lib.topk_distill_step(x, ids, t, g, **opts)
                wide = torch.full((R, V + 9), 7.0, dtype=dtype, device="cuda")
                out = gpu_lib.topk_distill_bwd(x, ids, t, stats, g, **opts, out=wide[:, 3:V + 3])
                near(out, np64(ref), 2 * HALF[dtype] * np.abs(np64(ref)) + 2.0 ** -20 * np.abs(np64(ref)), "dx")
                assert (wide[:, :3] == 7).all() and (wide[:, V + 3:] == 7).all()
                wide.fill_(7.0)
                gpu_lib.topk_distill_step(x, ids, t, g, **opts, out=wide[:, 3:V + 3])
                assert torch.equal(wide[:, 3:V + 3], ref) and (wide[:, :3] == 7).all() and (wide[:, V + 3:] == 7).all()
                same = x.clone()
                gpu_lib.topk_distill_bwd(same, ids, t, stats, g, **opts, out=same)
                assert torch.equal(same, out)
                same = x.clone()
                l2, _, _ = gpu_lib.topk_distill_step(same, ids, t, g, **opts, out=same)
                assert torch.equal(same, ref) and torch.equal(l2, loss)


@pytest.mark.parametrize("R", [4, 600])
def test_upstream_of_the_loss_and_retained_graphs(gpu_lib, R):
    x, ids, t = make(R, 3001, 16, seed=13)
    w = torch.rand(R, device="cuda")
    xg = x.requires_grad_(True)
    g1, = torch.autograd.grad(gpu_lib.topk_distill_loss(xg, ids, t, w), xg)
    loss, stats, step = gpu_lib.topk_distill_step(x.detach(), ids, t, w)
    assert torch.equal(g1, step)
    y = gpu_lib.topk_distill_loss(xg, ids, t, w)
    scaled, = torch.autograd.grad(y * 3.0, xg, retain_graph=True)
    assert torch.equal(scaled, gpu_lib.topk_distill_bwd(x.detach(), ids, t, stats, w, factor=3.0))
    keep = scaled.clone()
    again, = torch.autograd.grad(y, xg, retain_graph=True)   # formed anew, and the first one is left alone
    assert torch.equal(scaled, keep)
    assert torch.equal(again, gpu_lib.topk_distill_bwd(x.detach(), ids, t, stats, w))
    mean, = torch.autograd.grad(gpu_lib.topk_distill_loss(xg, ids, t), xg)
    near(mean, np64(gpu_lib.topk_distill_bwd(x.detach(), ids, t, stats, factor=1.0 / R)), 2.0 ** -7 * np.abs(np64(mean)),
         "mean")
    assert gpu_lib.topk_distill_loss(x.detach(), ids, t).requires_grad is False
    near(gpu_lib.topk_distill_loss(x.detach(), ids, t), np64(loss).mean(), 2.0 ** -22, "mean loss")


def test_tangents_and_gradients_of_the_teacher_are_refused(gpu_lib):
    x, ids, t = make(3, 100, 4, torch.float32)
    w = torch.ones(3, device="cuda")
    for call, args in ((gpu_lib.topk_distill, (x, ids, t)), (gpu_lib.topk_distill_loss, (x, ids, t, w)),
                       (gpu_lib.token_logprobs, (x, ids[:, 0].contiguous()))):
        plain = call(*args)
        with fw.dual_level():
            for i, a in enumerate(args):
                if a.is_floating_point():
                    dual = list(args)
                    dual[i] = fw.make_dual(a, torch.ones_like(a))
                    with pytest.raises(RuntimeError):
                        call(*dual)
            same = call(*args)
        for a, b in zip(*((p if isinstance(p, tuple) else (p,)) for p in (plain, same))):
            assert a is b is None or torch.equal(a, b)
    for args in ((x, ids, t.clone().requires_grad_(True), w), (x, ids, t, w.clone().requires_grad_(True))):
        with pytest.raises(ValueError):
            gpu_lib.topk_distill_loss(*args)
        with torch.no_grad():
            gpu_lib.topk_distill_loss(*args)


def test_no_rows(gpu_lib):
    for shape in ((0, 10), (2, 0, 10)):
        x = torch.zeros(shape, dtype=torch.bfloat16, device="cuda", requires_grad=True)
        ids = torch.zeros((*shape[:-1], 3), dtype=torch.int32, device="cuda")
        t = torch.zeros((*shape[:-1], 3), device="cuda")
        y = gpu_lib.topk_distill_loss(x, ids, t)
        assert y == 0 and torch.autograd.grad(y, x)[0].shape == shape
        assert gpu_lib.topk_distill(x, ids, t).shape == shape[:-1]


def test_refusals(gpu_lib):
    x, ids, t = make(4, 300, 6)
    call = gpu_lib.topk_distill
    wide = torch.zeros(4, 129, dtype=torch.int32, device="cuda")
    for bad in (lambda: call(x.cpu(), ids, t), lambda: call(x, ids.float(), t), lambda: call(x, ids[:3], t),
                lambda: call(x, ids, t[:, :5]), lambda: call(x, ids, t.double()), lambda: call(x, ids.t(), t.t()),
                lambda: call(x, ids[:, ::2], t[:, ::2]), lambda: call(x, ids, t, s1=0.5),
                lambda: call(x, ids, t, rest=False, direction="rev"), lambda: call(x, ids, t, direction="up"),
                lambda: call(x, ids, t, s2=0.0), lambda: call(x, ids, t, rest=False, s1=float("inf")),
                lambda: call(x, wide, wide.float()), lambda: call(x, ids[:, :0].contiguous(), t[:, :0].contiguous()),
                lambda: gpu_lib.topk_distill_loss(x, ids, t, torch.ones(3, device="cuda")),
                lambda: gpu_lib.topk_distill_loss(x, ids, t, torch.ones(4, device="cuda").double()),
                lambda: gpu_lib.topk_distill_loss(x.clone().requires_grad_(True), ids, t, torch.ones(4))):
        with pytest.raises((ValueError, gpu_lib.StreamKLError)):
            bad()
    loss, stats = gpu_lib.topk_distill_fwd(x, ids, t)
    for bad in (lambda: gpu_lib.topk_distill_bwd(x, ids, t, loss), lambda: gpu_lib.topk_distill_bwd(x, ids, t, stats[:3]),
                lambda: gpu_lib.topk_distill_bwd(x, ids, t, stats, out=x[:, :299]),
                lambda: gpu_lib.topk_distill_bwd(x, ids, t, stats, out=x[:1].expand(4, 300)),
                lambda: gpu_lib.topk_distill_bwd(x, ids, t, stats, done_if_one=True)):
        with pytest.raises((ValueError, gpu_lib.StreamKLError)):
            bad()


def test_offsets_past_32_bits(gpu_lib):
    V, R, K = 200003, 11000, 5
    x = torch.zeros((R, V), dtype=torch.bfloat16, device="cuda")
    last, ids1, t1 = make(2, V, K, seed=14)
    x[-2:] = last
    ids, t = ids1[:1].expand(R, K).contiguous(), t1[:1].expand(R, K).contiguous()
    ids[-2:], t[-2:] = ids1, t1
    loss, _, dx = gpu_lib.topk_distill_step(x, ids, t)
    ref, lb, rdx, db = lo.distill(np64(last), ids1.cpu().numpy(), np64(t1), 1.0, 1.0, True, False)
    near(loss[-2:], ref, lb, "loss")
    near(dx[-2:], rdx, db + 2.0 ** -8 * np.abs(rdx), "dx")
    assert torch.equal(dx[0], dx[R - 3])
