"""What autograd may ask of the operators around the divergence: tangents (refused), upstream gradients as graphs leave
them."""
import pytest
import torch
from torch.autograd import forward_ad as fw

pytestmark = pytest.mark.gpu


def norm_inputs(seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda")   # noqa: E731
    return [mk(2, 7, 4, 64).bfloat16(), mk(2, 7, 2, 64).bfloat16(), 1 + 0.1 * mk(64), 1 + 0.1 * mk(64)]


def diff_inputs(seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()   # noqa: E731
    return [mk(2, 4, 7, 64), mk(2, 2, 9, 64), mk(2, 4, 7, 64), mk(2, 2, 9, 64), mk(2, 2, 9, 96),
            torch.rand(4, generator=gen, device="cuda")]


@pytest.mark.parametrize("grad_mode", [True, False])
@pytest.mark.parametrize("name", ["qk_norm_rope", "diff_attention"])
def test_tangents_are_refused(gpu_lib, name, grad_mode):
    """A dual input has requires_grad False; its tangent must not be dropped."""
    call, inputs = getattr(gpu_lib, name), norm_inputs() if name == "qk_norm_rope" else diff_inputs()
    plain = call(*inputs)
    with fw.dual_level(), torch.set_grad_enabled(grad_mode):
        for i, x in enumerate(inputs):
            args = list(inputs)
            args[i] = fw.make_dual(x, torch.ones_like(x))
            with pytest.raises(RuntimeError):
                call(*args)
        same = call(*inputs)   # no tangents: as outside
    for a, b in zip(*((x if isinstance(x, tuple) else (x,)) for x in (plain, same))):
        assert torch.equal(a, b) and not b.requires_grad


def test_a_table_that_requires_a_gradient_is_refused(gpu_lib):
    q, k, wq, wk = norm_inputs()
    table = gpu_lib.rope_table(7, 64)
    plain = gpu_lib.qk_norm_rope(q, k, wq, wk, table)
    table.requires_grad_(True)
    with pytest.raises(ValueError):
        gpu_lib.qk_norm_rope(q, k, wq, wk, table)
    with torch.no_grad():
        same = gpu_lib.qk_norm_rope(q, k, wq, wk, table)
    for x in (same, gpu_lib.qk_norm_rope(q, k, wq, wk, table.detach())):
        assert torch.equal(x[0], plain[0]) and torch.equal(x[1], plain[1])


@pytest.mark.parametrize("name", ["qk_norm_rope", "diff_attention"])
@pytest.mark.parametrize("before", [1, 4, 8])
def test_upstream_gradients_of_a_concatenation(gpu_lib, name, before):
    """They are contiguous views that begin anywhere."""
    inputs = [x.requires_grad_(True) for x in (norm_inputs() if name == "qk_norm_rope" else diff_inputs())]
    outs = getattr(gpu_lib, name)(*inputs)
    outs = outs if isinstance(outs, tuple) else (outs,)
    pad = torch.zeros(before, dtype=torch.bfloat16, device="cuda")
    joint = torch.cat([y for out in outs for y in (pad, out.flatten())])
    g = torch.randn(joint.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).bfloat16()
    got = torch.autograd.grad(joint, inputs, g, retain_graph=True)
    parts, at = [], 0
    for out in outs:
        at += before
        parts.append(g[at:at + out.numel()].view(out.shape).clone())
        at += out.numel()
    for a, b in zip(got, torch.autograd.grad(outs, inputs, parts)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("q_rows,k_rows,n_pos,given,fits", [
    (7, 7, 6, "", False), (7, 7, 7, "", True), (2, 7, 6, "", False), (7, None, 6, "", False), (None, 7, 6, "", False),
    (2, 7, 6, "k", False), (2, 7, 6, "q", False), (2, 7, 3, "qk", True), (7, 7, None, "", True)])
def test_default_positions_have_to_be_in_the_table(gpu_lib, q_rows, k_rows, n_pos, given, fits):
    q, k, wq, wk = norm_inputs()
    q, k = (None if n is None else x[:, :n] for x, n in ((q, q_rows), (k, k_rows)))
    table = None if n_pos is None else gpu_lib.rope_table(n_pos, 32)
    opts = {n + "_positions": torch.arange(x.shape[1], device="cuda") % 3 for n, x in (("q", q), ("k", k)) if n in given}
    if fits:
        for y in gpu_lib.qk_norm_rope(q, k, wq, wk, table, **opts):
            assert torch.isfinite(y).all()
    else:
        with pytest.raises(ValueError):
            gpu_lib.qk_norm_rope(q, k, wq, wk, table, **opts)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("expand_k", [False, True])
def test_padding_outside_the_table_leaves_gradients_alone(gpu_lib, interleaved, expand_k):
    """A padded batch whose padding has position -1 and no upstream gradient: the gradients of the rows before it."""
    q, k, wq, wk = (x.requires_grad_(True) for x in norm_inputs())
    table = gpu_lib.rope_table(16, 32)
    at = torch.arange(7, dtype=torch.int32, device="cuda").repeat(2, 1)
    at[1, 4:] = -1
    opts = dict(interleaved=interleaved, expand_k=expand_k)
    out = gpu_lib.qk_norm_rope(q, k, wq, wk, table, q_positions=at, k_positions=at, **opts)
    assert torch.isnan(out[0][1, :, 4:, :32]).all() and torch.isfinite(out[0][1, :, :4]).all()
    gen = torch.Generator(device="cuda").manual_seed(2)
    up = [torch.randn(y.shape, generator=gen, device="cuda").bfloat16() for y in out]
    for u in up:
        u[1, :, 4:] = 0
    got = torch.autograd.grad(out, (q, k, wq, wk), up)
    assert not got[0][1, 4:].any() and not got[1][1, 4:].any()
    at[1, 4:] = 3   # inside the table, still no gradient
    ref = torch.autograd.grad(gpu_lib.qk_norm_rope(q, k, wq, wk, table, q_positions=at, k_positions=at, **opts),
                              (q, k, wq, wk), up)
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    up[0][1, 2, 5, 1] = 1.0   # a row that the loss reaches: NaN, not a number that is wrong
    out = gpu_lib.qk_norm_rope(q, k, wq, wk, table, q_positions=at.where(at != 3, -1), k_positions=at, **opts)
    assert torch.isnan(torch.autograd.grad(out, (wq,), up)[0]).any()


def test_gradients_of_a_side_that_is_not_there_are_refused(gpu_lib):
    q, k, wq, wk = norm_inputs()
    yq, yk = gpu_lib.qk_norm_rope_fwd(q, k, wq, wk)
    for args in ((q, k, None, yk), (q, k, yq, None), (q, None, yq, yk), (None, k, yq, yk), (q, None, None, None)):
        with pytest.raises(ValueError):
            gpu_lib.qk_norm_rope_bwd(*args, wq, wk)
