"""token_logprobs against the 64-bit oracle: values, best tokens, gradients; layouts, masks, rows that are nothing."""
import numpy as np
import pytest
import torch

from oracle import logits_oracle as lo

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}   # half a step among subnormal numbers


def logits(R, V, dtype, seed=0, spread=2.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((R, V), generator=gen, device="cuda") * spread).to(dtype)


def np64(t):
    return t.detach().double().cpu().numpy()


def near(got, ref, name):
    value, bound = ref
    got = np64(got)
    bad = ~((np.abs(got - value) <= bound) | (got == value) | (np.isnan(got) & np.isnan(value)))
    assert not bad.any(), (name, got[bad][:4], value[bad][:4], np.broadcast_to(bound, got.shape)[bad][:4])


def check_fwd(sk, x, tokens, scale, top):
    """x [R, V] or [B, N, V] on the GPU."""
    y = sk.token_logprobs(x, tokens, scale=scale, top=top)
    flat = np64(x).reshape(-1, x.shape[-1])
    ref = lo.token_logprobs(flat, None if tokens is None else tokens.cpu().numpy().reshape(-1), scale, top)
    for name in ("logp", "entropy", "lse"):
        got = getattr(y, name)
        if name not in ref:
            assert got is None
            continue
        assert got.shape == x.shape[:-1] and got.dtype is torch.float32
        near(got.reshape(-1), ref[name], name)
    if top:
        assert y.top_ids.shape == (*x.shape[:-1], top) and y.top_ids.dtype is torch.int32
        assert (y.top_ids.cpu().numpy().reshape(-1, top) == ref["top_ids"]).all()
        near(y.top_logp.reshape(-1, top), ref["top_logp"], "top_logp")
    else:
        assert y.top_ids is None and y.top_logp is None
    return y, ref


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("V,R", [(1, 3), (2, 5), (7, 3), (8, 9), (9, 700), (63, 5), (130, 4), (1000, 33), (4097, 6),
                                 (8192, 3), (50257, 5), (131072, 2), (140001, 3), (300007, 2)])
def test_values(gpu_lib, V, R, dtype):
    x = logits(R, V, dtype, seed=V)
    tokens = torch.randint(0, V, (R,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(V))
    tokens[R - 1] = -1
    for top in sorted({0, 1, min(5, V), min(64, V), min(128, V)}):
        check_fwd(gpu_lib, x, tokens if top != 1 else tokens.int(), 1.0 if top else 0.6, top)
    check_fwd(gpu_lib, x, None, 1.25, min(3, V))


@pytest.mark.parametrize("R", [1, 16, 17, 600])
@pytest.mark.parametrize("top", [0, 20, 128])
def test_few_and_many_rows(gpu_lib, R, top):
    """Rows cut into parts that are joined, and rows by a workgroup each, give the same best tokens."""
    V = 60001
    x = logits(R, V, torch.bfloat16, seed=1)
    y, _ = check_fwd(gpu_lib, x[:min(R, 40)], None, 1.0, top)
    whole = gpu_lib.token_logprobs(x, None, top=top)
    if top:
        assert torch.equal(whole.top_ids[:min(R, 40)], y.top_ids)
    near(whole.lse[:min(R, 40)], (np64(y.lse), 4 * HALF[torch.float32] * np.abs(np64(y.lse)) + 1e-5), "lse")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,R", [(1000, 3), (20000, 1), (20000, 520), (131072, 520), (200000, 1)])
@pytest.mark.parametrize("kind", ["equal", "two", "rising", "falling", "columns", "zeros", "few"])
def test_best_tokens_of_rows_that_are_no_noise(gpu_lib, kind, V, R, dtype):
    """Equal logits, few values, sorted rows, large logits all in one thread's chunks, signed zeros, few finite ones."""
    j = torch.arange(V, device="cuda")
    row = {"equal": torch.full((V,), 1.5, device="cuda"), "two": (j % 3 == 1).float(), "rising": j / 64.0,
           "falling": -j / 64.0, "columns": torch.where((j // 8) % 512 == 5, 4.0 + j % 7, 0.0),
           "zeros": torch.where(j % 2 == 0, -0.0, 0.0), "few": torch.where(j % (V // 50) == 3, j % 5 / 1.0, -torch.inf)}[kind]
    x = row.to(dtype).expand(R, V).clone()
    if R > 1:
        x[1:3, :V // 2] = logits(2, V // 2, dtype)
    for top in (5, 128):
        y = gpu_lib.token_logprobs(x, None, top=top)
        ref = lo.token_logprobs(np64(x[:3]), None, 1.0, top)
        assert (y.top_ids[:3].cpu().numpy() == ref["top_ids"]).all()
        near(y.top_logp[:3], ref["top_logp"], "top_logp")
        near(y.entropy[:3], ref["entropy"], "entropy")
        near(y.lse[:3], ref["lse"], "lse")
        assert torch.equal(y.top_ids[3:], y.top_ids[:1].expand(max(R - 3, 0), top))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("R", [6, 600])
def test_masked_logits(gpu_lib, R, dtype):
    """-inf, the type's lowest value, rows of nothing else, one logit left, far above and below the others."""
    V = 5003
    x = logits(R, V, dtype, seed=2)
    low = torch.finfo(dtype).min
    x[0, 100:] = -torch.inf
    x[1, :4000] = low
    x[2] = -torch.inf
    x[3] = low
    x[4] = -torch.inf
    x[4, 4321] = 3.0
    x[5, 7] = 60000.0
    x[5, 9] = low
    tokens = torch.tensor([5, 4500, 3, 17, 4321, 9] + [1] * (R - 6), device="cuda")
    y, _ = check_fwd(gpu_lib, x[:6].contiguous(), tokens[:6], 1.0, 12)
    assert y.lse[2] == -torch.inf and y.entropy[2] == 0 and y.logp[2] == -torch.inf
    assert y.entropy[4] == 0 and y.logp[4] == 0
    xg = x.clone().requires_grad_(True)
    z = gpu_lib.token_logprobs(xg, tokens)
    up = torch.ones(R, device="cuda")
    dx, = torch.autograd.grad((z.logp, z.entropy, z.lse), xg, (up, up, up))
    ref, bound = lo.token_logprobs_grad(np64(x[:6]), tokens[:6].cpu().numpy(), 1.0, *(np.ones(6),) * 3)
    near(dx[:6], (ref, bound + HALF[dtype] * np.abs(ref) + TINY[dtype]), "dx")
    assert torch.isfinite(dx).all() and not dx[2].any()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("R,V", [(3, 30000), (700, 3001)])
def test_a_value_that_is_none_spoils_its_row_only(gpu_lib, R, V, value):
    x = logits(R, V, torch.bfloat16, seed=3)
    tokens = torch.zeros(R, dtype=torch.int64, device="cuda")
    clean = gpu_lib.token_logprobs(x, tokens, top=9)
    x[1, 77] = value
    y = gpu_lib.token_logprobs(x, tokens, top=9)
    keep = torch.arange(R, device="cuda") != 1
    for a, b in zip(clean, y):
        assert torch.equal(a[keep], b[keep])
    for t in (y.logp, y.entropy, y.lse):
        assert torch.isnan(t[1])
    ids = y.top_ids[1]
    assert ((ids >= -1) & (ids < V)).all() and ids[ids >= 0].unique().numel() == (ids >= 0).sum()
    x[1] = float("nan")
    y = gpu_lib.token_logprobs(x, tokens, top=9)
    assert (y.top_ids[1] == -1).all() and torch.isnan(y.top_logp[1]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layouts(gpu_lib, dtype):
    """Rows anywhere: a sliced vocabulary, all positions but the last, transposed batches, one row for all, odd addresses;
    what lies beside them is not read (it is NaN)."""
    V = 1003
    pad = torch.full((3, 8, V + 21), float("nan"), dtype=dtype, device="cuda")
    tokens = torch.randint(0, V, (3, 7), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    for first in range(0, 21, 5):
        x = pad[:, :-1, first:first + V]
        x.copy_(logits(21, V, dtype, seed=first).view(3, 7, V))
        check_fwd(gpu_lib, x, tokens, 1.0, 6)
        xg = x.detach().requires_grad_(True)
        y = gpu_lib.token_logprobs(xg, tokens)
        dx, = torch.autograd.grad(y.logp.sum(), xg)
        base = x.contiguous().requires_grad_(True)
        ref, = torch.autograd.grad(gpu_lib.token_logprobs(base, tokens).logp.sum(), base)
        # the same sums in another order
        near(dx, (np64(ref), 2 * HALF[dtype] * np.abs(np64(ref)) + 2.0 ** -18 * np.abs(np64(ref))), "dx")
        pad.fill_(float("nan"))
    x = logits(21, V, dtype).view(7, 3, V).transpose(0, 1)
    check_fwd(gpu_lib, x, tokens, 1.0, 3)
    check_fwd(gpu_lib, logits(1, V, dtype).expand(7, V), tokens[0], 1.0, 3)
    check_fwd(gpu_lib, logits(5, V, dtype)[:, 4:5], torch.zeros(5, dtype=torch.int32, device="cuda"), 1.0, 1)


def test_no_rows(gpu_lib):
    for shape in ((0, 10), (2, 0, 10), (0, 3, 10)):
        x = torch.zeros(shape, dtype=torch.bfloat16, device="cuda", requires_grad=True)
        t = torch.zeros(shape[:-1], dtype=torch.int32, device="cuda")
        y = gpu_lib.token_logprobs(x, t, top=4)
        assert y.logp.shape == shape[:-1] and y.top_ids.shape == (*shape[:-1], 4)
        assert torch.autograd.grad(y.logp.sum(), x)[0].shape == shape


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("V,R", [(1, 3), (5, 4), (8, 3), (1001, 21), (50257, 4), (131072, 2), (270001, 2)])
@pytest.mark.parametrize("which", ["all", "logp", "entropy", "lse"])
def test_gradients(gpu_lib, V, R, dtype, which):
    x = logits(R, V, dtype, seed=V + 1).requires_grad_(True)
    gen = torch.Generator(device="cuda").manual_seed(V)
    tokens = torch.randint(0, V, (R,), device="cuda", generator=gen)
    tokens[0] = -1
    up = {n: torch.randn(R, generator=gen, device="cuda") for n in ("logp", "entropy", "lse")}
    scale = 0.8
    y = gpu_lib.token_logprobs(x, tokens, scale=scale)
    names = list(up) if which == "all" else [which]
    dx, = torch.autograd.grad([getattr(y, n) for n in names], x, [up[n] for n in names])
    assert dx.dtype is dtype
    ref, bound = lo.token_logprobs_grad(np64(x), tokens.cpu().numpy(), scale,
                                        *(np64(up[n]) if n in names else None for n in up))
    near(dx, (ref, bound + HALF[dtype] * np.abs(ref) + TINY[dtype]), "dx")


def test_gradients_against_differences(gpu_lib):
    V, h = 40, 2.0 ** -6
    x = logits(1, V, torch.float32, seed=9).requires_grad_(True)
    tok = torch.tensor([7], device="cuda")
    f = lambda t: (lambda y: y.logp + 0.5 * y.entropy - 0.3 * y.lse)(gpu_lib.token_logprobs(t, tok, scale=0.9))   # noqa: E731
    dx, = torch.autograd.grad(f(x).sum(), x)
    shift = torch.eye(V, device="cuda") * h
    toks = tok.expand(V).contiguous()
    g = lambda t: (lambda y: y.logp + 0.5 * y.entropy - 0.3 * y.lse)(gpu_lib.token_logprobs(t, toks, scale=0.9))   # noqa: E731
    d = (g(x.detach() + shift) - g(x.detach() - shift)) / (2 * h)
    # third derivatives of these are below 1, so that the difference is off by h^2 / 6; values by a few 2^-22
    assert (d - dx[0]).abs().max() <= h * h / 6 + 2.0 ** -20 / h


def test_rows_without_an_upstream_gradient_are_not_read(gpu_lib):
    x = logits(4, 3001, torch.bfloat16)
    x[2] = float("nan")
    tokens = torch.tensor([1, -1, 5, 3001], device="cuda")
    xg = x.requires_grad_(True)
    y = gpu_lib.token_logprobs(xg, tokens)
    assert y.logp[1] == 0 and torch.isnan(y.logp[2]) and torch.isnan(y.logp[3])
    up = torch.tensor([1.0, 1.0, 0.0, 0.0], device="cuda")
    dx, = torch.autograd.grad(y.logp, xg, up, retain_graph=True)
    assert torch.isfinite(dx).all() and dx[0].any() and not dx[1:].any()
    up[3] = 1.0   # a token outside the vocabulary that the loss reaches: NaN, not a number that is wrong
    dx, = torch.autograd.grad(y.logp, xg, up)
    assert torch.isnan(dx[3]).all() and not dx[1:3].any()


def test_gradients_in_place_and_beside_other_data(gpu_lib):
    for dtype in (torch.bfloat16, torch.float32):
        V = 40003
        x = logits(6, V, dtype, seed=4).view(2, 3, V)
        tokens = torch.randint(0, V, (2, 3), device="cuda")
        y, err = gpu_lib.token_logprobs_fwd(x, tokens, save=True)
        up = torch.randn(2, 3, device="cuda")
        ref = gpu_lib.token_logprobs_bwd(x, tokens, y.lse, err, y.entropy, up, up)
        wide = torch.full((2, 3, V + 9), 7.0, dtype=dtype, device="cuda")
        out = gpu_lib.token_logprobs_bwd(x, tokens, y.lse, err, y.entropy, up, up, out=wide[:, :, 3:V + 3])
        assert torch.equal(out, ref) and (wide[:, :, :3] == 7).all() and (wide[:, :, V + 3:] == 7).all()
        assert gpu_lib.token_logprobs_bwd(x, tokens, y.lse, err, y.entropy, up, up, out=x) is x
        assert torch.equal(x, ref)


def test_refusals(gpu_lib):
    x = logits(4, 100, torch.bfloat16)
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    call = gpu_lib.token_logprobs
    for bad in (lambda: call(x.cpu(), None), lambda: call(x.double(), None), lambda: call(x[0], None),
                lambda: call(x.t(), None), lambda: call(x[None, None], None), lambda: call(x, t[:3]),
                lambda: call(x, t.float()), lambda: call(x, t.cpu()), lambda: call(x, t.expand(2, 4).t()[:, 0].int()[::1][:2]),
                lambda: call(x, top=101), lambda: call(x, top=-1), lambda: call(x, t, scale=0.0),
                lambda: call(x, t, scale=float("nan")), lambda: call(x, t, scale=-1.0),
                lambda: call(logits(4, 200, torch.bfloat16), top=129)):
        with pytest.raises((ValueError, gpu_lib.StreamKLError)):
            bad()
    y, err = gpu_lib.token_logprobs_fwd(x, t, save=True)
    up = torch.ones(4, device="cuda")
    back = gpu_lib.token_logprobs_bwd
    for bad in (lambda: back(x, None, y.lse, dlogp=up), lambda: back(x, t, y.lse, dentropy=up),
                lambda: back(x, t, None, dlogp=up), lambda: back(x, t, y.lse, dlogp=up[:3]),
                lambda: back(x, t, y.lse, dlogp=up, out=x[:3]), lambda: back(x, t, y.lse, dlogp=up, out=x.float()),
                lambda: back(x, t, y.lse, dlogp=up, out=x[:1].expand(4, 100))):
        with pytest.raises((ValueError, gpu_lib.StreamKLError)):
            bad()
    with pytest.raises(ValueError):
        gpu_lib.token_logprobs_fwd(x, t, workspace=torch.empty(16))


def test_offsets_past_32_bits(gpu_lib):
    """The last of more than 2^32 bytes of logits, forward and backward."""
    V, R = 200003, 11000
    x = torch.zeros((R, V), dtype=torch.bfloat16, device="cuda")
    x[-2:] = logits(2, V, torch.bfloat16, seed=8)
    t = torch.full((R,), 5, dtype=torch.int64, device="cuda")
    t[-1] = V - 1
    y, err = gpu_lib.token_logprobs_fwd(x, t, top=7, save=True)
    check, _ = check_fwd(gpu_lib, x[-2:].clone(), t[-2:], 1.0, 7)
    assert torch.equal(y.top_ids[-2:], check.top_ids) and torch.equal(y.top_ids[0].cpu(), torch.arange(7, dtype=torch.int32))
    near(y.logp[-2:], (np64(check.logp), 1e-5), "logp")
    up = torch.ones(R, device="cuda")
    dx = gpu_lib.token_logprobs_bwd(x, t, y.lse, err, dlogp=up)
    ref, bound = lo.token_logprobs_grad(np64(x[-2:]), t[-2:].cpu().numpy(), 1.0, np.ones(2), None, None)
    near(dx[-2:], (ref, bound + 2.0 ** -8 * np.abs(ref)), "dx")
