"""Differential attention on the GPU against the plain fp64 form, with elementwise bounds counted in roundings."""
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo

pytestmark = pytest.mark.gpu

NAMES = ("dq1", "dk1", "dq2", "dk2", "dv", "dlam")


def n64(t):
    return t.detach().double().cpu().numpy()


def within(got, ref, bound, what):
    err = np.abs(n64(got) - ref)
    bad = ~(err <= bound + 1e-30)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, worst {np.nanmax(err / (bound + 1e-30)):.2f} bounds"


def make(B, H, HK, NQ, NK, d, dv, seed=0, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda")   # noqa: E731
    t = [(size * mk(B, H, NQ, d)).bfloat16(), mk(B, HK, NK, d).bfloat16(), (size * mk(B, H, NQ, d)).bfloat16(),
         mk(B, HK, NK, d).bfloat16(), mk(B, HK, NK, dv).bfloat16()]
    lam = mk(H) * 0.7
    return (*t, lam), mk(B, H, NQ, dv).bfloat16()


def lens(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def check(sk, args, do, causal=False, ql=None, kl=None, scale=None, splits="auto", grads=True):
    """Forward, saved statistics and all gradients (float32) of one call against the oracle."""
    q1, v = args[0], args[4]
    s = 1 / math.sqrt(q1.shape[-1]) if scale is None else scale
    saved = sk.diff_fwd(*args, scale, causal, lens(ql), lens(kl), splits=splits, save=True)
    torch.cuda.synchronize()
    ref, tol = oo.diff(*(n64(a) for a in args), s, causal, ql, kl)
    within(saved[0], ref["out"], tol["out"], "out")
    within(saved[1], ref["out2"], tol["out2"], "out2")
    for n, t in (("lse1", saved[2]), ("lse2", saved[3])):
        r, g = ref[n], n64(t)
        assert (np.isneginf(r) == np.isneginf(g)).all(), n
        f = np.isfinite(r)
        # logits of d float32 terms and a sum of exponentials: F32 of a value of size |lse| + 1 covers both
        assert (np.abs(g[f] - r[f]) <= oo.F32 * (1 + np.abs(r[f]))).all(), n
    if not grads:
        return saved
    got = sk.diff_bwd(*args, do, *saved, scale, causal, lens(ql), lens(kl))
    torch.cuda.synchronize()
    rg, tg = oo.diff_backward(*(n64(a) for a in args), s, causal, n64(do), ql, kl)
    for n, t in zip(NAMES, got):
        assert t.dtype == torch.float32
        within(t, rg[n], tg[n], n)
    return saved


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("dv", [32, 64, 96, 128, 160, 192, 224, 256])
def test_head_dims(gpu_lib, d, dv, causal):
    args, do = make(1, 2, 1, 77, 90, d, dv, seed=d + dv)
    check(gpu_lib, args, do, causal)


@pytest.mark.parametrize("B,H,HK,NQ,NK", [
    (1, 1, 1, 1, 1), (2, 1, 1, 1, 31), (1, 3, 3, 1, 333), (1, 2, 2, 33, 32), (1, 2, 1, 97, 131), (1, 2, 2, 131, 97),
    (2, 6, 2, 129, 160), (1, 5, 1, 50, 65), (1, 8, 1, 7, 200), (3, 4, 4, 64, 64), (1, 1, 1, 300, 5), (1, 2, 2, 257, 513)])
@pytest.mark.parametrize("causal", [False, True])
def test_extents(gpu_lib, B, H, HK, NQ, NK, causal):
    """Lengths of one, odd ones, rows before the first key (causal, N_Q > N_K), shared heads."""
    args, do = make(B, H, HK, NQ, NK, 64, 64, seed=NQ)
    check(gpu_lib, args, do, causal)


@pytest.mark.parametrize("ql,kl", [([40, 70, 1], [40, 70, 1]), (None, [0, 90, 33]), ([0, 70, 32], None),
                                   ([70, 64, 5], [10, 200, 32]), ([-3, 31, 70], [90, -1, 64])])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(gpu_lib, ql, kl, causal):
    """Padded batches, empty sequences, lengths outside 0 .. N (clamped); what lies behind them is never read."""
    args, do = make(3, 4, 2, 70, 90, 64, 128, seed=3)
    args = [a.clone() for a in args]
    for b in range(3):
        nq = 70 if ql is None else min(max(ql[b], 0), 70)
        nk = 90 if kl is None else min(max(kl[b], 0), 90)
        for x in (args[0], args[2], do):
            x[b, :, nq:] = float("nan")
        for x in (args[1], args[3], args[4]):
            x[b, :, nk:] = float("inf") if b else float("nan")
    check(gpu_lib, args, do, causal, ql, kl)


@pytest.mark.parametrize("splits", [2, 3, 7, 64, 256])
@pytest.mark.parametrize("causal", [False, True])
def test_splits(gpu_lib, splits, causal):
    args, do = make(2, 6, 2, 3, 1000, 64, 96, seed=splits)
    check(gpu_lib, args, do, causal, None, [1000, 37], splits=splits)
    args, do = make(1, 2, 2, 150, 200, 128, 256, seed=splits)
    check(gpu_lib, args, do, causal, [150], [140], splits=splits, grads=False)


def test_split_workspace_contents_do_not_matter(gpu_lib):
    args, _ = make(2, 4, 2, 5, 700, 64, 64)
    n = gpu_lib.diff_workspace_bytes(2, 4, 5, 64, 5)
    ws = torch.full((n // 4,), float("nan"), device="cuda")
    a = gpu_lib.diff_fwd(*args, None, True, lens([3, 5]), lens([600, 0]), splits=5, workspace=ws)
    b = gpu_lib.diff_fwd(*args, None, True, lens([3, 5]), lens([600, 0]), splits=5)
    assert torch.equal(a, b)


@pytest.mark.parametrize("lam", [0.0, -1.5, 1e-38, -1e-42, 30.0])
def test_lambda(gpu_lib, lam):
    """Zero, negative, subnormal and large weights of the second map, mixed within a group of heads."""
    args, do = make(1, 4, 2, 60, 75, 64, 64)
    args[5][:] = torch.tensor([lam, 0.4, 0.4, lam], device="cuda")
    check(gpu_lib, args, do, True)


@pytest.mark.parametrize("size,causal", [(30.0, False), (30.0, True), (0.0, True)])
def test_large_and_equal_logits(gpu_lib, size, causal):
    """Maps of almost one key, where the exponent reference moves, and flat ones."""
    args, do = make(1, 2, 2, 65, 161, 64, 64, size=size)
    saved = gpu_lib.diff_fwd(*args, None, causal, save=True)
    ref, tol = oo.diff(*(n64(a) for a in args), 0.125, causal)
    # logits up to about 8 x 30 x 4: their float32 error, relative to the probability, is d 2^-24 times that
    slack = 2.0 ** -10 * (np.abs(ref["out"]) + 4.0 * np.ones_like(ref["out"])) if size > 1 else 0.0
    within(saved[0], ref["out"], tol["out"] + slack, "out")


def test_rising_logits_move_the_reference(gpu_lib):
    """Keys that grow along the axis: the reference has to follow by hundreds of doublings, up and not down."""
    args, do = make(1, 2, 1, 40, 640, 64, 64)
    q1, k1, q2, k2, v, lam = args
    u = torch.randn(64, device="cuda")
    u = u / u.norm()
    ramp = torch.linspace(0, 60, 640, device="cuda")
    for q, k, r in ((q1, k1, ramp), (q2, k2, ramp.flip(0))):
        q.copy_((q.float() * 0.1 + 8 * u).bfloat16())
        k.copy_((k.float() * 0.1 + r[:, None] * u).bfloat16())
    for causal in (False, True):
        saved = gpu_lib.diff_fwd(*args, 1.0, causal, save=True)
        ref, tol = oo.diff(*(n64(a) for a in args), 1.0, causal)
        # |logit| to 480 in float32: 480 x 2^-24 x a few for the sums, far below F32, which tol holds already
        within(saved[0], ref["out"], tol["out"], "out")
        assert (np.abs(n64(saved[2]) - ref["lse1"]) <= oo.F32 * (1 + np.abs(ref["lse1"]))).all()


def test_strided_inputs(gpu_lib):
    """Halves of one projection, values token-major, the filled part of a cache, a sequence shared by expansion."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()   # noqa: E731
    q, kc, vp = mk(2, 8, 50, 64), mk(2, 4, 200, 64), mk(2, 70, 2, 128)
    lam, do = torch.rand(4, device="cuda"), mk(2, 4, 50, 128)
    args = (q[:, :4], kc[:, :2, :70], q[:, 4:], kc[:, 2:, 100:170], vp.transpose(1, 2), lam)
    check(gpu_lib, args, do, True)
    tok = mk(2, 50, 4, 64)   # token-major queries
    args = (tok.transpose(1, 2), kc[:1, :2, :70].expand(2, 2, 70, 64), q[:, 4:], kc[:, 2:, :70],
            vp.transpose(1, 2), lam)
    check(gpu_lib, args, do, False)


def test_heads_beyond_4_gib(gpu_lib):
    """Row strides that put the last keys of a head 6 GiB behind the first."""
    NK, sn = 200, 1 << 24
    far = torch.empty(NK * sn, dtype=torch.bfloat16, device="cuda")
    args, do = make(1, 2, 1, 20, NK, 64, 64)
    k1 = far.as_strided((1, 1, NK, 64), (NK * sn, NK * sn, sn, 1))
    v = far[1024:].as_strided((1, 1, NK, 64), (NK * sn - 1024, NK * sn - 1024, sn, 1))
    k1.copy_(args[1])
    v.copy_(args[4])
    check(gpu_lib, (args[0], k1, args[2], args[3], v, args[5]), do, True)
    check(gpu_lib, (args[0], k1, args[2], args[3], v, args[5]), do, False, splits=3, grads=False)


def test_zero_extents(gpu_lib):
    args, do = make(2, 2, 1, 5, 0, 64, 64)
    saved = gpu_lib.diff_fwd(*args, save=True)
    assert not saved[0].any() and torch.isneginf(saved[2]).all()
    g = gpu_lib.diff_bwd(*args, do, *saved)
    assert not g[0].any() and not g[2].any() and not g[5].any() and g[1].numel() == 0
    args, do = make(2, 2, 1, 0, 5, 64, 64)
    saved = gpu_lib.diff_fwd(*args, save=True)
    g = gpu_lib.diff_bwd(*args, do, *saved)
    assert saved[0].numel() == 0 and not any(x.any() for x in g)


def test_gradient_subsets(gpu_lib):
    args, do = make(1, 4, 2, 70, 90, 64, 64)
    saved = gpu_lib.diff_fwd(*args, None, True, save=True)
    full = gpu_lib.diff_bwd(*args, do, *saved, None, True)
    for want in (("dq1",), ("dk2",), ("dlam",), ("dv",), ("dq2", "dk1"), ("dk1", "dk2", "dv")):
        part = gpu_lib.diff_bwd(*args, do, *saved, None, True, want=want)
        for n, a, b in zip(NAMES, part, full):
            assert (a is None) == (n not in want)
            assert a is None or torch.equal(a, b), n


def test_autograd(gpu_lib):
    """bf16 gradients are the float32 ones rounded once; only what is asked for comes back; a frozen lam works."""
    args, do = make(2, 4, 2, 45, 60, 64, 128)
    leaves = [a.requires_grad_(True) for a in args]
    out = gpu_lib.diff_attention(*leaves, causal=True, kv_len=lens([60, 20]))
    got = torch.autograd.grad(out, leaves, do, retain_graph=True)
    plain = [a.detach() for a in args]
    saved = gpu_lib.diff_fwd(*plain, None, True, None, lens([60, 20]), save=True)
    assert torch.equal(out, saved[0])
    ref = gpu_lib.diff_bwd(*plain, do, *saved, None, True, None, lens([60, 20]))
    for n, a, b in zip(NAMES, got, ref):
        assert a.dtype == (torch.float32 if n == "dlam" else torch.bfloat16)
        assert torch.equal(a, b.to(a.dtype)), n
    # an upstream gradient that is expanded, as from a sum
    one = torch.autograd.grad(out.sum(), leaves[:1])[0]
    assert torch.equal(one, gpu_lib.diff_bwd(*plain, torch.ones_like(do), *saved, None, True, None, lens([60, 20]),
                                             want=("dq1",), grad_dtype=torch.bfloat16)[0])
    frozen = gpu_lib.diff_attention(leaves[0], *plain[1:], causal=True)
    assert frozen.requires_grad
    with torch.no_grad():
        assert not gpu_lib.diff_attention(*leaves).requires_grad


def test_reproducible_on_streams_and_in_graphs(gpu_lib):
    """The same bits from every run, on another stream and from replays with eager work between them; two captured
    calls keep workspaces of their own."""
    args, do = make(2, 4, 2, 150, 200, 64, 128)
    few, _ = make(2, 4, 2, 2, 900, 64, 128, seed=1)
    many = (few[0], few[1], few[2], few[3], few[4], few[5])

    def step():
        saved = gpu_lib.diff_fwd(*args, None, True, save=True)
        return (*saved, *gpu_lib.diff_bwd(*args, do, *saved, None, True), gpu_lib.diff_fwd(*many, splits=6),
                gpu_lib.diff_fwd(*many, None, True, splits=5))

    ref = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(ref, other):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(4):
        for t in out:
            t.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(ref, out):
            assert torch.equal(a, b)


def test_captured_training_step(gpu_lib):
    """A whole step through autograd (norm, rotation, attention, gradients) recorded into a graph, with the warm-up's
    graph gone; replayed several times with new inputs and eager work in between."""
    B, N, H, d = 2, 60, 4, 64
    gen = torch.Generator(device="cuda").manual_seed(8)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()   # noqa: E731
    leaves = [mk(B, N, 2 * H, d), mk(B, N, 2 * H, d), mk(B, N, H, d), 1 + 0.1 * torch.randn(d, device="cuda"),
              torch.rand(H, device="cuda")]
    leaves = [t.requires_grad_(True) for t in leaves]
    table, do = gpu_lib.rope_table(N, d), mk(B, H, N, d)

    def step():
        yq, yk = gpu_lib.qk_norm_rope(leaves[0], leaves[1], leaves[3], None, table)
        (q1, q2), (k1, k2) = yq.split(H, 1), yk.split(H, 1)
        out = gpu_lib.diff_attention(q1, k1, q2, k2, leaves[2].transpose(1, 2), leaves[4], causal=True)
        return [out.detach(), *torch.autograd.grad(out, leaves, do)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        with torch.no_grad():
            for t in leaves[:3]:
                t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        ref = step()
        for t in out:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(ref, out):
            assert torch.equal(a, b), i


def test_second_derivatives_are_refused(gpu_lib):
    args, do = make(1, 1, 1, 8, 8, 64, 64)
    q = args[0].requires_grad_(True)
    g, = torch.autograd.grad(gpu_lib.diff_attention(q, *args[1:]), q, do.requires_grad_(True), create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.float().sum(), q)


def test_inputs_are_untouched(gpu_lib):
    args, do = make(1, 2, 1, 70, 90, 96, 160)
    before = [a.clone() for a in (*args, do)]
    saved = gpu_lib.diff_fwd(*args, None, True, save=True)
    kept = [s.clone() for s in saved]
    gpu_lib.diff_bwd(*args, do, *saved, None, True)
    for a, b in zip((*args, do, *saved), (*before, *kept)):
        assert torch.equal(a, b)


def test_layer_of_both_operators(gpu_lib):
    """Projections to gradients of projections as a model uses them: norm and rotation of both halves, differential
    attention with values as projected; against the plain forms in 64 bits, chained with the kernels' bf16 rounding of
    the rotated queries and keys."""
    B, N, H, HK, d, dv, eps = 2, 75, 4, 2, 64, 128, 1e-6
    gen = torch.Generator(device="cuda").manual_seed(21)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()   # noqa: E731
    xq, xk, xv = mk(B, N, 2 * H, d), mk(B, N, 2 * HK, d), mk(B, N, HK, dv)
    wq, wk = (1 + 0.2 * torch.randn(2, d, generator=gen, device="cuda")).unbind(0)
    leaves = [t.contiguous().requires_grad_(True) for t in (xq, xk, xv, wq, wk, torch.rand(H, generator=gen, device="cuda"))]
    table = gpu_lib.rope_table(N, d)
    yq, yk = gpu_lib.qk_norm_rope(leaves[0], leaves[1], leaves[3], leaves[4], table, eps=eps)
    q1, q2 = yq.split(H, 1)
    k1, k2 = yk.split(HK, 1)
    out = gpu_lib.diff_attention(q1, k1, q2, k2, leaves[2].transpose(1, 2), leaves[5], causal=True)
    do = mk(B, H, N, dv)
    got = torch.autograd.grad(out, leaves, do)
    # the kernels' own rotated tensors go into the second oracle, so that each is compared on its own inputs
    pos, tab = np.arange(N), n64(table)
    for x, w, y in ((leaves[0], leaves[3], yq), (leaves[1], leaves[4], yk)):
        ref, bound = oo.norm_rope(n64(x), n64(w), tab, pos, eps)
        within(y, ref, bound, "y")
    mid = [n64(t) for t in (q1, k1, q2, k2, leaves[2].transpose(1, 2), leaves[5])]
    ref, tol = oo.diff(*mid, d ** -0.5, True)
    within(out, ref["out"], tol["out"], "out")
    g, t = oo.diff_backward(*mid, d ** -0.5, True, n64(do), half=oo.HALF)
    within(got[2].transpose(1, 2), g["dv"], t["dv"], "dv")
    within(got[5], g["dlam"], t["dlam"], "dlam")
    for x, w, dx, dw, a, b in ((leaves[0], leaves[3], got[0], got[3], "dq1", "dq2"),
                               (leaves[1], leaves[4], got[1], got[4], "dk1", "dk2")):
        dy, e = np.concatenate([g[a], g[b]], 1), np.concatenate([t[a], t[b]], 1)
        rx, bx, rw, bw = oo.norm_rope_backward(n64(x), n64(w), tab, pos, eps, dy, half=oo.HALF)
        # the error of dy passes through the same linear map, with absolute coefficients: its bound is what bx is made
        # of (2^-16 of it), times 2^16
        _, ex, _, ew = oo.norm_rope_backward(n64(x), n64(w), tab, pos, eps, e)
        within(dx, rx, bx + 2.0 ** 16 * ex, "dx")
        within(dw, rw, bw + 2.0 ** 14 * ew, "dw")


def test_refusals(gpu_lib):
    args, do = make(2, 4, 2, 6, 8, 64, 64)
    q1, k1, q2, k2, v, lam = args
    bad = [dict(q1=q1.cpu()), dict(q1=q1.float()), dict(k1=k1[:, :, :7]), dict(k2=k2[..., :32]), dict(q2=q2[:, :2]),
           dict(v=v[:, :1]), dict(lam=lam.double()), dict(lam=lam[:2]), dict(v=v[0]),
           dict(k1=torch.cat((k1, k1[:, :1]), 1), k2=torch.cat((k2, k2[:, :1]), 1), v=torch.cat((v, v[:, :1]), 1)),
           dict(q_len=torch.zeros(2, dtype=torch.int64, device="cuda")),
           dict(kv_len=torch.zeros(3, dtype=torch.int32, device="cuda")),
           dict(q1=q1.transpose(2, 3).contiguous().transpose(2, 3)),
           dict(v=torch.randn(2, 2, 8, 68, device="cuda").bfloat16()[..., 4:])]
    for kw in bad:
        a = dict(q1=q1, k1=k1, q2=q2, k2=k2, v=v, lam=lam)
        a.update(kw)
        with pytest.raises(ValueError):
            gpu_lib.diff_attention(**a)
    for kw in (dict(scale=0.0), dict(scale=float("nan"))):
        with pytest.raises(gpu_lib.StreamKLError):
            gpu_lib.diff_attention(*args, **kw)
    wide, _ = make(1, 1, 1, 4, 4, 160, 64)
    with pytest.raises(gpu_lib.StreamKLError):
        gpu_lib.diff_attention(*wide)
    with pytest.raises(gpu_lib.StreamKLError):
        gpu_lib.diff_fwd(*args, splits=4, workspace=torch.empty(16, device="cuda"))
    saved = gpu_lib.diff_fwd(*args, save=True)
    with pytest.raises(ValueError):
        gpu_lib.diff_bwd(*args, do, *saved, want=("dq3",))
    with pytest.raises(ValueError):
        gpu_lib.diff_bwd(*args, do.float(), *saved)
    with pytest.raises(ValueError):
        gpu_lib.diff_bwd(*args, do, *saved, grad_dtype=torch.float16)


def test_workspace_refusals(gpu_lib):
    """A workspace on the host, or one whose elements lie apart, is not what the kernels write to."""
    args, do = make(2, 4, 2, 6, 600, 64, 64)
    n = gpu_lib.diff_workspace_bytes(2, 4, 6, 64, 4)
    m = gpu_lib.diff_bwd_workspace_bytes(2, 4, 2, 6, 600, 64, 64, False)
    saved = gpu_lib.diff_fwd(*args, save=True)
    for make_ws in (lambda n: torch.empty(n, dtype=torch.uint8),
                    lambda n: torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            gpu_lib.diff_fwd(*args, splits=4, workspace=make_ws(n))
        with pytest.raises(ValueError):
            gpu_lib.diff_bwd(*args, do, *saved, workspace=make_ws(m))


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_a_non_finite_row_stays_alone(gpu_lib, value, splits):
    """A query row that is not finite spoils its own output and dQ, and no other row's, nor those of other heads."""
    (q1, k1, q2, k2, v, lam), do = make(1, 4, 2, 70, 200, 64, 96)
    clean = gpu_lib.diff_fwd(q1, k1, q2, k2, v, lam, splits=splits, save=True)
    g = gpu_lib.diff_bwd(q1, k1, q2, k2, v, lam, do, *clean, want=("dq1", "dq2"))
    bad = q1.clone()
    bad[0, 1, 33, 5] = value
    dirty = gpu_lib.diff_fwd(bad, k1, q2, k2, v, lam, splits=splits, save=True)
    h = gpu_lib.diff_bwd(bad, k1, q2, k2, v, lam, do, *dirty, want=("dq1", "dq2"))
    keep = torch.ones(1, 4, 70, dtype=torch.bool, device="cuda")
    keep[0, 1, 33] = False
    assert not torch.isfinite(dirty[0][0, 1, 33]).any()
    for a, b in ((clean[0], dirty[0]), (clean[1], dirty[1]), (g[0], h[0]), (g[2], h[2])):
        assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("d,dv", [(64, 128), (96, 96), (128, 128), (64, 192), (32, 256), (128, 160)])
@pytest.mark.parametrize("B,H,HK,NQ,NK,ql,kl", [
    (1, 1, 1, 1, 1, None, None), (1, 2, 1, 1, 63, None, None), (1, 2, 1, 65, 64, None, None), (1, 2, 2, 131, 65, None, None),
    (2, 4, 2, 70, 150, [70, 33], [129, 17]), (2, 2, 2, 40, 70, [0, 40], [70, 0]), (1, 8, 1, 300, 200, None, [190])])
@pytest.mark.parametrize("causal", [False, True])
def test_key_blocks(gpu_lib, d, dv, B, H, HK, NQ, NK, ql, kl, causal):
    """Extents around the blocks of 16, 64 and 128 keys and the tiles of 32 rows, shared heads, split row ranges."""
    args, do = make(B, H, HK, NQ, NK, d, dv, seed=d + NK)
    check(gpu_lib, args, do, causal, ql, kl)


@pytest.mark.parametrize("d,dv", [(64, 64), (64, 128), (128, 128), (128, 256)])
def test_bf16_gradients_of_every_key_form(gpu_lib, d, dv):
    """The float32 gradients, rounded once; the last key block is ragged."""
    args, do = make(2, 2, 1, 130, 201, d, dv, seed=d)
    saved = gpu_lib.diff_fwd(*args, None, True, save=True)
    a = gpu_lib.diff_bwd(*args, do, *saved, None, True)
    b = gpu_lib.diff_bwd(*args, do, *saved, None, True, grad_dtype=torch.bfloat16)
    for n, x, y in zip(NAMES, a, b):
        assert torch.equal(x if n == "dlam" else x.bfloat16(), y), n
