"""Norm and rotation of queries and keys on the GPU against the plain fp64 form, with bounds counted in roundings."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def n64(t):
    return t.detach().double().cpu().numpy()


def within(got, ref, bound, what):
    err = np.abs(n64(got) - ref)
    bad = ~(err <= bound + 1e-30)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, worst {np.nanmax(err / (bound + 1e-30)):.2f} bounds"


def make(B, NQ, NK, H, HK, d, rot, dtype="bf16", seed=0, n_pos=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(B, NQ, H, d, generator=gen, device="cuda").to(TYPES[dtype])
    k = (3 * torch.randn(B, NK, HK, d, generator=gen, device="cuda")).to(TYPES[dtype])
    wq, wk = (1 + 0.3 * torch.randn(2, d, generator=gen, device="cuda")).unbind(0)
    return q, k, wq.contiguous(), wk.contiguous()


def check(sk, q, k, wq, wk, table, eps=1e-6, qp=None, kp=None, interleaved=False, expand=False, dy32=False, seed=1):
    """Forward and gradients of one call against the oracle."""
    copies = q.shape[2] // k.shape[2] if expand else 1
    NQ, NK = q.shape[1], k.shape[1]
    yq, yk = sk.qk_norm_rope_fwd(q, k, wq, wk, table, eps, qp, kp, interleaved, expand)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.float32 if dy32 else torch.bfloat16
    dyq, dyk = (torch.randn(y.shape, generator=gen, device="cuda").to(t) for y in (yq, yk))
    got = sk.qk_norm_rope_bwd(q, k, dyq, dyk, wq, wk, table, eps, qp, kp, interleaved, expand)
    torch.cuda.synchronize()
    assert yq.is_contiguous() and yk.is_contiguous() and yq.dtype == yk.dtype == torch.bfloat16
    tab = None if table is None else n64(table)
    for x, w, y, dy, dx, dw, pos, cp, n in ((q, wq, yq, dyq, got[0], got[2], qp, 1, "q"),
                                            (k, wk, yk, dyk, got[1], got[3], kp, copies, "k")):
        pos = np.arange(x.shape[1]) + (NK - NQ if n == "q" else 0) if pos is None else pos.cpu().numpy()
        w64 = None if w is None else n64(w)
        ref, bound = oo.norm_rope(n64(x), w64, tab, pos, eps, interleaved, cp)
        within(y, ref, bound, "y" + n)
        half = torch.finfo(x.dtype).eps / 2
        rx, bx, rw, bw = oo.norm_rope_backward(n64(x), w64, tab, pos, eps, n64(dy), interleaved, cp, half)
        assert dx.dtype == x.dtype and dx.shape == x.shape
        # fp16: gradients below its normal range are off by half of its smallest step
        within(dx, rx, bx + (2.0 ** -25 if x.dtype == torch.float16 else 0), "dx" + n)
        within(dw, rw, bw, "dw" + n)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_head_dims_and_types(gpu_lib, d, dtype):
    q, k, wq, wk = make(2, 21, 21, 6, 2, d, d, dtype)
    check(gpu_lib, q, k, wq, wk, gpu_lib.rope_table(21, d))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(32, 16), (64, 48), (96, 96), (96, 16), (128, 64), (160, 80), (256, 112), (128, 0)])
def test_partial_rotations(gpu_lib, d, rot, interleaved):
    q, k, wq, wk = make(3, 13, 17, 4, 4, d, rot, "fp32", seed=d)
    check(gpu_lib, q, k, wq, wk, gpu_lib.rope_table(17, rot) if rot else None, interleaved=interleaved, dy32=True)


@pytest.mark.parametrize("B,NQ,NK,H,HK", [(1, 1, 1, 1, 1), (5, 1, 1, 3, 1), (1, 1, 333, 2, 2), (1, 333, 333, 1, 1),
                                          (7, 3, 5, 12, 4), (2, 700, 701, 33, 11)])
def test_extents(gpu_lib, B, NQ, NK, H, HK):
    q, k, wq, wk = make(B, NQ, NK, H, HK, 64, 64, seed=NQ)
    check(gpu_lib, q, k, wq, wk, gpu_lib.rope_table(NK, 64))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dy32", [False, True])
def test_expanded_keys(gpu_lib, interleaved, dtype, dy32):
    q, k, wq, wk = make(2, 19, 23, 12, 4, 96, 96, dtype)
    check(gpu_lib, q, k, wq, wk, gpu_lib.rope_table(23, 96), interleaved=interleaved, expand=True, dy32=dy32)


@pytest.mark.parametrize("kind", ["int32", "int64"])
@pytest.mark.parametrize("shared", [False, True])
def test_positions(gpu_lib, kind, shared):
    """Positions out of order, repeated and far out; at 10^5 a float32 angle would be off by 4e-3."""
    q, k, wq, wk = make(3, 9, 14, 4, 2, 64, 64, "fp32")
    gen = torch.Generator(device="cuda").manual_seed(5)
    t = torch.int32 if kind == "int32" else torch.int64
    qp, kp = (torch.randint(0, 120000, (n,) if shared else (3, n), generator=gen, device="cuda").to(t) for n in (9, 14))
    check(gpu_lib, q, k, wq, wk, gpu_lib.rope_table(120000, 64), qp=qp, kp=kp)
    check(gpu_lib, q, k, wq, wk, gpu_lib.rope_table(120000, 64), kp=kp)


def test_table_values(gpu_lib):
    t = n64(gpu_lib.rope_table(200001, 32, base=5e5))
    p = np.array([0, 1, 99999, 200000])
    a = p[:, None] * 5e5 ** (-np.arange(0, 32, 2) / 32)
    # float64 angles up to 2e5 are off by 2e5 2^-53 and a few steps of the power; the values are rounded to float32
    np.testing.assert_allclose(t[p], np.concatenate([np.cos(a), np.sin(a)], 1), rtol=2.0 ** -24, atol=1e-9)


def test_positions_outside_the_table_give_nan(gpu_lib):
    q, k, wq, wk = make(1, 4, 4, 2, 2, 64, 32)
    kp = torch.tensor([0, 7, 8, -1], dtype=torch.int64, device="cuda")
    yq, yk = gpu_lib.qk_norm_rope(q, k, wq, wk, gpu_lib.rope_table(8, 32), k_positions=kp)
    assert torch.isfinite(yk[:, :, :2]).all() and torch.isfinite(yq).all()
    assert torch.isnan(yk[:, :, 2:, :32]).all() and torch.isfinite(yk[:, :, 2:, 32:]).all()


def test_without_weights_one_side_and_zero_rows(gpu_lib):
    q, k, wq, wk = make(2, 6, 6, 4, 2, 64, 64, "fp32")
    q[0, 1, 2] = 0.0
    table = gpu_lib.rope_table(6, 64)
    check(gpu_lib, q, k, None, None, table, eps=1e-3)
    yq, yk = gpu_lib.qk_norm_rope(q, k, wq, wk, table)
    only_q, nothing = gpu_lib.qk_norm_rope(q, None, wq, None, table)
    assert nothing is None and torch.equal(only_q, yq) and not yq[0, 2, 1].any()
    nothing, only_k = gpu_lib.qk_norm_rope(None, k, None, wk, table)
    assert nothing is None and torch.equal(only_k, yk)


def test_strided_inputs(gpu_lib):
    """Parts of one projection, head-major inputs, and a head shared by expansion (stride 0)."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    joint = torch.randn(2, 11, 8, 64, generator=gen, device="cuda").bfloat16()
    w = 1 + 0.1 * torch.randn(64, generator=gen, device="cuda")
    table = gpu_lib.rope_table(11, 64)
    check(gpu_lib, joint[:, :, :6], joint[:, :, 6:], w, w, table)
    major = torch.randn(2, 4, 11, 64, generator=gen, device="cuda").bfloat16().transpose(1, 2)
    check(gpu_lib, major, joint[:, 3:9, :1].expand(2, 6, 4, 64)[:, :, :4], w, w, table,
          qp=torch.arange(11, dtype=torch.int32, device="cuda"))


def test_autograd_matches_the_calls(gpu_lib):
    q, k, wq, wk = make(2, 15, 15, 6, 2, 64, 64)
    table = gpu_lib.rope_table(15, 64)
    leaves = [t.requires_grad_(True) for t in (q, k, wq, wk)]
    yq, yk = gpu_lib.qk_norm_rope(*leaves, table, expand_k=True)
    dq, dk = torch.randn_like(yq), torch.randn_like(yk)
    got = torch.autograd.grad((yq, yk), leaves, (dq, dk), retain_graph=True)
    ref = gpu_lib.qk_norm_rope_bwd(q.detach(), k.detach(), dq, dk, wq.detach(), wk.detach(), table, expand_k=True)
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    # an output that the loss does not reach, and an upstream gradient that is not contiguous
    part = torch.autograd.grad(yq, leaves, dq.transpose(2, 3).contiguous().transpose(2, 3), retain_graph=True,
                               allow_unused=True)
    assert torch.equal(part[0], ref[0]) and torch.equal(part[2], ref[2])
    part = torch.autograd.grad(yk, leaves[1:2], dk)
    assert torch.equal(part[0], ref[1])
    with torch.no_grad():
        assert not gpu_lib.qk_norm_rope(*leaves, table)[0].requires_grad


def test_reproducible_on_streams_and_in_graphs(gpu_lib):
    """Every run, on any stream and replayed from a graph, gives the same bits; eager work between the replays."""
    q, k, wq, wk = make(2, 300, 300, 8, 4, 128, 128)
    table = gpu_lib.rope_table(300, 128)
    dq, dk = torch.randn(2, 8, 300, 128, device="cuda").bfloat16(), torch.randn(2, 4, 300, 128, device="cuda").bfloat16()
    step = lambda: (*gpu_lib.qk_norm_rope_fwd(q, k, wq, wk, table),   # noqa: E731
                    *gpu_lib.qk_norm_rope_bwd(q, k, dq, dk, wq, wk, table))
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


def test_attention_kl_from_projections(gpu_lib):
    """attention_kl_proj is the norms, the rotation and attention_kl in a row: the divergence of the prepared tensors
    against its own oracle, gradients equal to those of the steps taken one by one."""
    import oracle
    B, N, H, d1, d2 = 1, 80, 4, 64, 32
    gen = torch.Generator(device="cuda").manual_seed(31)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda")   # noqa: E731
    q1, k1, q2, k2 = mk(B, N, H, d1).bfloat16(), mk(B, N, 2, d1).bfloat16(), mk(B, N, H, d2), mk(B, N, 1, d2)
    w = [(1 + 0.2 * mk(d)).requires_grad_(d == d2) for d in (d1, d1, d2, d2)]
    t1, t2 = gpu_lib.rope_table(N, d1), gpu_lib.rope_table(N, 16)
    q2.requires_grad_(True), k2.requires_grad_(True)
    p1, p2 = gpu_lib.QKPrep(w[0], w[1], t1), gpu_lib.QKPrep(w[2], w[3], t2, 1e-5, True)
    kl = gpu_lib.attention_kl_proj(q1, k1, q2, k2, p1, p2, causal=True)
    leaves = [q2, k2, w[2], w[3]]
    got = torch.autograd.grad(kl.sum(), leaves)
    a1, b1 = gpu_lib.qk_norm_rope(q1, k1, w[0], w[1], t1, expand_k=True)
    a2, b2 = gpu_lib.qk_norm_rope(q2, k2, w[2], w[3], t2, eps=1e-5, interleaved=True, expand_k=True)
    step = gpu_lib.attention_kl(a1, b1, a2, b2, causal=True)
    assert torch.equal(kl, step)
    for a, b in zip(got, torch.autograd.grad(step.sum(), leaves)):
        assert torch.equal(a, b) and torch.isfinite(a).all() and a.any()
    ref = oracle.forward(*(n64(x) for x in (a1, b1, a2, b2)), d1 ** -0.5, d2 ** -0.5, True, 0)[0]
    assert (np.abs(n64(kl) - ref) <= 1e-3 + 1e-2 * np.abs(ref)).all()   # the bound that the divergence's own tests use
    rev = gpu_lib.attention_kl_proj(q1, k1, q2, k2, p1, p2, causal=True, direction="rev", return_lse=True)
    assert len(rev) == 3 and not torch.equal(rev[0], kl)


def test_refusals(gpu_lib):
    q, k, wq, wk = make(2, 6, 6, 4, 2, 64, 64)
    t = gpu_lib.rope_table(6, 64)
    bad = [dict(q=q.cpu()), dict(q=q.double()), dict(q=q[0]), dict(k=k.float()), dict(k=k[:1]), dict(wq=wq.bfloat16()),
           dict(wq=wq[:32]), dict(table=t.double()), dict(table=t[:, :24].contiguous()), dict(table=t.t()),
           dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)), dict(q=torch.randn(2, 9, 4, 64, device="cuda").bfloat16()),
           dict(q_positions=torch.zeros(6, device="cuda")), dict(q_positions=torch.zeros(7, dtype=torch.int32, device="cuda")),
           dict(q_positions=torch.zeros(6, dtype=torch.int32, device="cuda"),
                k_positions=torch.zeros(6, dtype=torch.int64, device="cuda")),
           dict(k=torch.randn(2, 6, 3, 64, device="cuda").bfloat16(), expand_k=True), dict(q=None, k=None),
           dict(q=torch.randn(2, 6, 4, 68, device="cuda").bfloat16()[..., 4:])]
    for kw in bad:
        a = dict(q=q, k=k, wq=wq, wk=wk, table=t)
        a.update(kw)
        with pytest.raises(ValueError):
            gpu_lib.qk_norm_rope(a.pop("q"), a.pop("k"), a.pop("wq"), a.pop("wk"), a.pop("table"), **a)
    with pytest.raises(gpu_lib.StreamKLError):
        gpu_lib.qk_norm_rope(q, k, wq, wk, t, eps=0.0)
    x = torch.randn(2, 6, 4, 48, device="cuda").bfloat16()
    with pytest.raises(gpu_lib.StreamKLError):
        gpu_lib.qk_norm_rope(x, None)
    with pytest.raises(ValueError):
        gpu_lib.rope_table(8, 24)


def test_more_workgroups_than_one_grid_axis_holds(gpu_lib):
    """2^30 + 5 tokens of one head: 2^24 + 1 workgroups, and offsets past 32 bits in every unit. All tokens are one row."""
    n = (1 << 30) + 5
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 64 GiB of outputs")
    row = torch.randn(1, 1, 1, 32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).bfloat16()
    expect, _ = gpu_lib.qk_norm_rope_fwd(row, None)
    y, _ = gpu_lib.qk_norm_rope_fwd(row.expand(1, n, 1, 32), None)
    step = 1 << 27
    for i in range(0, n, step):
        assert bool((y[0, 0, i:i + step] == expect[0, 0]).all()), i
    del y
    torch.cuda.empty_cache()


def test_workspace_refusals(gpu_lib):
    q, k, wq, wk = make(2, 6, 6, 4, 2, 64, 64)
    y = gpu_lib.qk_norm_rope_fwd(q, k, wq, wk)
    n = gpu_lib.lib.streamkl_qk_norm_rope_bwd_workspace_bytes(2, 4, 2, 6, 6, 64)
    for ws in (torch.empty(n, dtype=torch.uint8), torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            gpu_lib.qk_norm_rope_bwd(q, k, *y, wq, wk, workspace=ws)
    with pytest.raises(gpu_lib.StreamKLError):
        gpu_lib.qk_norm_rope_bwd(q, k, *y, wq, wk, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
