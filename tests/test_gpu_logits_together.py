"""The operators on rows of logits together, as a distillation step uses them: eager, captured, on other streams."""
import numpy as np
import pytest
import torch

from oracle import logits_oracle as lo

pytestmark = pytest.mark.gpu


def normal(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def np64(t):
    return t.detach().double().cpu().numpy()


def program(sk, teacher, student, tokens, top=16):
    """A teacher's best tokens, the student's loss on them with its gradient, and its scores."""
    best = sk.token_logprobs(teacher, top=top, entropy=False)
    loss, stats, grad = sk.topk_distill_step(student, best.top_ids, best.top_logp, factor=0.5)
    again = sk.topk_distill_bwd(student, best.top_ids, best.top_logp, stats, factor=0.25)
    scores, err = sk.token_logprobs_fwd(student, tokens, top=3, save=True)
    back = sk.token_logprobs_bwd(student, tokens, scores.lse, err, scores.entropy, loss, loss)
    return [best.top_ids, best.top_logp, loss, grad, again, *scores, back]


@pytest.mark.parametrize("direction", ["fwd", "rev"])
@pytest.mark.parametrize("B,N,V", [(1, 1, 30001), (2, 5, 4099), (3, 70, 1000)])
def test_teacher_to_student(gpu_lib, B, N, V, direction):
    """Through autograd from weights of a head, against the same in 64 bits."""
    h, D, K = normal(B, N, 32, seed=1), 32, 12
    wt, ws = normal(V, D, seed=2) * 0.4, (normal(V, D, seed=2) * 0.4 + normal(V, D, seed=3) * 0.05).requires_grad_(True)
    best = gpu_lib.token_logprobs(h @ wt.t(), top=K)
    student = h @ ws.t()
    student.retain_grad()
    loss = gpu_lib.topk_distill_loss(student, best.top_ids, best.top_logp, direction=direction)
    loss.backward()
    flat = np64(student).reshape(-1, V)
    ref = lo.token_logprobs(np64(h @ wt.t()).reshape(-1, V), None, 1.0, K)
    assert (best.top_ids.cpu().numpy().reshape(-1, K) == ref["top_ids"]).all()
    rows = B * N
    value, bound, dx, db = lo.distill(flat, best.top_ids.cpu().numpy().reshape(-1, K), np64(best.top_logp).reshape(-1, K),
                                      1.0, 1.0, True, direction == "rev", np.full(rows, 1.0 / rows))
    assert abs(float(loss.detach()) - value.mean()) <= bound.mean() + 2.0 ** -23 * abs(value.mean())
    got = np64(student.grad).reshape(-1, V)
    assert (np.abs(got - dx) <= db + 2.0 ** -24 * np.abs(dx)).all()
    assert torch.isfinite(ws.grad).all() and ws.grad.any()


@pytest.mark.parametrize("B,N,V", [(1, 2, 60001), (2, 100, 3001)])
def test_results_are_reproducible(gpu_lib, B, N, V):
    args = normal(B, N, V, seed=4).bfloat16(), normal(B, N, V, seed=5).bfloat16(), \
        torch.randint(0, V, (B, N), device="cuda")
    first = program(gpu_lib, *args)
    for _ in range(5):
        for a, b in zip(first, program(gpu_lib, *args)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("direction", ["fwd", "rev"])
@pytest.mark.parametrize("R", [3, 500])
def test_a_token_with_many_entries_is_reproducible(gpu_lib, R, direction):
    """Whichever of its entries is written last."""
    V, K = 70001, 96
    x = normal(R, V, seed=14)
    ids = torch.randint(0, 9, (R, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * 7001
    t = torch.log_softmax(normal(R, K + 1, seed=15), -1)[:, :K].contiguous()
    loss, stats, first = gpu_lib.topk_distill_step(x, ids, t, direction=direction)
    back = gpu_lib.topk_distill_bwd(x, ids, t, stats, direction=direction)
    for _ in range(8):
        again = gpu_lib.topk_distill_step(x, ids, t, direction=direction)
        assert torch.equal(again[0], loss) and torch.equal(again[2], first)
        assert torch.equal(gpu_lib.topk_distill_bwd(x, ids, t, stats, direction=direction), back)


@pytest.mark.parametrize("B,N,V", [(1, 2, 60001), (2, 100, 3001)])
def test_captured_and_replayed(gpu_lib, B, N, V):
    """Two graphs with workspaces of their own, replayed with eager work and other inputs in between."""
    def inputs(seed):
        return (normal(B, N, V, seed=seed).bfloat16(), normal(B, N, V, seed=seed + 1).bfloat16(),
                torch.randint(0, V, (B, N), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))

    graphs = []
    for seed in (10, 20):
        held = [t.clone() for t in inputs(seed)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            program(gpu_lib, *held)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = program(gpu_lib, *held)
        graphs.append((g, held, out))
    for turn in range(3):
        for i, (g, held, out) in enumerate(graphs):
            new = inputs(100 * turn + 7 * i)
            for a, b in zip(held, new):
                a.copy_(b)
            g.replay()
            ref = program(gpu_lib, *new)
            torch.cuda.synchronize()
            for a, b in zip(out, ref):
                assert torch.equal(a, b)


def test_a_captured_training_step(gpu_lib):
    """Forward and backward through autograd in one graph, with an upstream gradient that changes between replays."""
    B, N, V, K = 2, 64, 2000, 8
    x = normal(B, N, V, seed=6).bfloat16().requires_grad_(True)
    best = gpu_lib.token_logprobs(normal(B, N, V, seed=7), top=K)
    w, scale = torch.rand(B, N, device="cuda"), torch.ones((), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(gpu_lib.topk_distill_loss(x, best.top_ids, best.top_logp, w), x, scale)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loss = gpu_lib.topk_distill_loss(x, best.top_ids, best.top_logp, w)
        grad, = torch.autograd.grad(loss, x, scale)
    for value in (1.0, 4.0, 1.0, 0.5):
        scale.fill_(value)
        x.data.copy_(normal(B, N, V, seed=int(8 * value)))
        g.replay()
        torch.cuda.synchronize()
        row, stats, one = gpu_lib.topk_distill_step(x.detach(), best.top_ids, best.top_logp, w)
        ref = one if value == 1.0 else gpu_lib.topk_distill_bwd(x.detach(), best.top_ids, best.top_logp, stats, w,
                                                                dfactor=scale)
        assert torch.equal(grad, ref)
        total = (row.double() * w.double()).sum()
        assert abs(float(loss.detach().double() - total)) <= 2.0 ** -23 * abs(float(total))


def test_other_streams(gpu_lib):
    """Calls on two streams at once, each in the order of its own stream, with workspaces of their own."""
    V = 60001
    data = [(normal(1, 3, V, seed=s).bfloat16(), normal(1, 3, V, seed=s + 1).bfloat16(),
             torch.zeros(1, 3, dtype=torch.int64, device="cuda")) for s in (30, 40)]
    ref = [program(gpu_lib, *d) for d in data]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                x = [t.clone() for t in data[i]]   # made on this stream, read on it
                got[i].append(program(gpu_lib, *x))
    torch.cuda.synchronize()
    for i in range(2):
        for out in got[i]:
            for a, b in zip(out, ref[i]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R", [1, 130])
def test_the_largest_vocabulary(gpu_lib, R, dtype):
    V = 1 << 22
    x = torch.zeros((R, V), dtype=dtype, device="cuda") if R > 1 else None
    last = normal(1, V, seed=9).to(dtype)
    if R > 1:
        x[-1] = last[0]
    else:
        x = last
    y, err = gpu_lib.token_logprobs_fwd(x, torch.full((R,), V - 1, dtype=torch.int64, device="cuda"), top=128, save=True)
    ref = lo.token_logprobs(np64(last), np.array([V - 1]), 1.0, 128)
    assert (y.top_ids[-1].cpu().numpy() == ref["top_ids"][0]).all()
    for n in ("logp", "entropy", "lse"):
        assert abs(float(getattr(y, n)[-1]) - ref[n][0][0]) <= ref[n][1][0]
    ids, t = y.top_ids[:, :20].contiguous(), y.top_logp[:, :20].contiguous() + 1.0
    loss, _, dx = gpu_lib.topk_distill_step(x, ids, t)
    value, bound, g, gb = lo.distill(np64(last), ids[-1:].cpu().numpy(), np64(t[-1:]), 1.0, 1.0, True, False)
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[dtype]
    assert abs(float(loss[-1]) - value[0]) <= bound[0]
    assert (np.abs(np64(dx[-1]) - g[0]) <= gb[0] + half * np.abs(g[0])).all()


def test_more_rows_than_an_axis_of_the_grid(gpu_lib):
    R, V = (1 << 21) + 5, 9
    x = torch.zeros((R, V), device="cuda")
    x[-5:] = normal(5, V, seed=12)
    t = torch.full((R,), 3, dtype=torch.int32, device="cuda")
    y, err = gpu_lib.token_logprobs_fwd(x, t, top=2, save=True)
    small = gpu_lib.token_logprobs(x[-5:].clone(), t[:5], top=2)
    for a, b in zip(y, small):
        assert torch.equal(a[-5:], b)
    up = torch.ones(R, device="cuda")
    dx = gpu_lib.token_logprobs_bwd(x, t, y.lse, err, dlogp=up)
    ref, bound = lo.token_logprobs_grad(np64(x[-5:]), np.full(5, 3), 1.0, np.ones(5), None, None)
    assert (np.abs(np64(dx[-5:]) - ref) <= bound + 2.0 ** -24 * np.abs(ref)).all() and torch.equal(dx[0], dx[(1 << 21) - 1])
    ids, v = y.top_ids, y.top_logp
    loss, _, g = gpu_lib.topk_distill_step(x, ids, v)
    few, _, h = gpu_lib.topk_distill_step(x[-5:].clone(), ids[-5:].clone(), v[-5:].clone())
    assert torch.equal(loss[-5:], few) and torch.equal(g[-5:], h) and torch.equal(g[0], g[(1 << 21) - 1])
