"""Plain fp64 NumPy forms of the operators around the divergence, for the tests.

norm_rope / norm_rope_backward: norm of every head and rotation by its position (streamkl_qk_norm_rope_*).
diff / diff_backward: differential attention (streamkl_diff_*), with maps and logit gradients written out.

Every function also returns how far a computation may be from it that rounds operands and results to bf16 where the
kernels do and keeps everything else in float32. A rounding to bf16 is off by at most HALF = 2^-8 of the value. The
float32 part is covered by F32 times the sum of the absolute terms: a logit of d <= 128 terms is off by at most
d 2^-24 of its absolute terms, here with |q||k| s up to a few tens, which the exponential turns into a relative error
of the probability of up to about 128 * 32 * 2^-24 = 2^-12 in the worst case, and 2^-17 for errors that do not all
point one way; sums of up to 2^10 terms add 2^-14 at worst. F32 = 2^-12.
"""
import numpy as np

HALF = 2.0 ** -8
F32 = 2.0 ** -12


# --- norm and rotation ------------------------------------------------------------------------------------------------


def _turn(y, table, pos, interleaved, back=False):
    """Rotate the first rot columns of y [B, N, H, d] by the positions [N] or [B, N]."""
    rot = table.shape[1]
    out = y.copy()
    if rot == 0:
        return out
    t = table[np.asarray(pos)]
    t = (t[None] if t.ndim == 2 else t)[:, :, None, :]
    c, s = t[..., :rot // 2], t[..., rot // 2:]
    if back:
        s = -s
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * c - b * s, b * c + a * s
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        out[..., :rot // 2], out[..., rot // 2:rot] = a * c - b * s, b * c + a * s
    return out


def norm_rope(x, w, table, pos, eps, interleaved=False, copies=1):
    """x [B, N, H, d] -> (y [B, H copies, N, d], bound). w None: ones; table None: no rotation."""
    x = x.astype(np.float64)
    w = np.ones(x.shape[-1]) if w is None else w.astype(np.float64)
    table = np.zeros((1, 0)) if table is None else table.astype(np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r * w
    y = _turn(n, table, pos, interleaved)
    # float32: a handful of roundings and a sum of up to 256 squares, on the two terms of a rotated value
    terms = np.abs(n)
    if table.shape[1]:
        terms[..., :table.shape[1]] = np.hypot(*_pair_terms(n, table.shape[1], interleaved))
    bound = HALF * np.abs(y) + 2.0 ** -17 * terms
    heads = lambda z: np.repeat(z.transpose(0, 2, 1, 3), copies, axis=1)   # noqa: E731
    return heads(y), heads(bound)


def _pair_terms(n, rot, interleaved):
    a, b = (n[..., 0:rot:2], n[..., 1:rot:2]) if interleaved else (n[..., :rot // 2], n[..., rot // 2:rot])
    if interleaved:
        return np.repeat(np.abs(a), 2, -1), np.repeat(np.abs(b), 2, -1)
    return np.concatenate([np.abs(a)] * 2, -1), np.concatenate([np.abs(b)] * 2, -1)


def norm_rope_backward(x, w, table, pos, eps, dy, interleaved=False, copies=1, half=0.0):
    """(dx [B, N, H, d], its bound, dw [d], its bound) for dy [B, H copies, N, d]. half: relative rounding of dx."""
    x, dy = x.astype(np.float64), dy.astype(np.float64)
    w = np.ones(x.shape[-1]) if w is None else w.astype(np.float64)
    table = np.zeros((1, 0)) if table is None else table.astype(np.float64)
    B, N, H, d = x.shape
    g = dy.reshape(B, H, copies, N, d).sum(2).transpose(0, 2, 1, 3)
    g = _turn(g, table, pos, interleaved, back=True)
    ga = np.abs(dy).reshape(B, H, copies, N, d).sum(2).transpose(0, 2, 1, 3)
    if table.shape[1]:
        a, b = _pair_terms(ga, table.shape[1], interleaved)
        ga = ga.copy()
        ga[..., :table.shape[1]] = a + b
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh, h = x * r, g * w
    dx = r * (h - xh * (h * xh).mean(-1, keepdims=True))
    ha = ga * np.abs(w)
    bound = half * np.abs(dx) + 2.0 ** -16 * r * (ha + np.abs(xh) * (ha * np.abs(xh)).mean(-1, keepdims=True))
    dw = (g * xh).sum((0, 1, 2))
    return dx, bound, dw, 2.0 ** -14 * (ga * np.abs(xh)).sum((0, 1, 2))


# --- differential attention -------------------------------------------------------------------------------------------


def visible(nq, nk, qlen, klen, causal):
    """[nq, nk]: the pairs that take part."""
    rows, cols = np.arange(nq)[:, None], np.arange(nk)[None]
    ok = (rows < qlen) & (cols < klen)
    return ok & (cols <= rows + klen - qlen) if causal else ok


def _maps(q, k, scale, ok):
    z = np.where(ok, scale * (q @ k.T), -np.inf)
    m = z.max(1, initial=-np.inf)
    m0 = np.where(np.isfinite(m), m, 0.0)
    e = np.exp(z - m0[:, None])
    total = e.sum(1)
    with np.errstate(divide="ignore"):
        lse = m0 + np.log(total)
    return e / np.where(total > 0, total, 1.0)[:, None], lse


def _lengths(n, lens, B):
    return [n] * B if lens is None else [min(max(int(x), 0), n) for x in lens]


def _clean(x, n):
    """The first n rows of x [N, d]; the others hold nothing that is read."""
    y = x.astype(np.float64).copy()
    y[n:] = 0.0
    return y


def diff(q1, k1, q2, k2, v, lam, scale, causal, q_len=None, kv_len=None):
    """{"out", "out2", "lse1", "lse2"} and {"out", "out2"}: bounds. q [B, H, N_Q, d], k, v [B, HK, N_K, .]."""
    B, H, NQ, _ = q1.shape
    HK, NK, dv = v.shape[1:]
    res = {n: np.zeros((B, H, NQ, dv)) for n in ("out", "out2")}
    res.update({n: np.full((B, H, NQ), -np.inf) for n in ("lse1", "lse2")})
    tol = {n: np.zeros((B, H, NQ, dv)) for n in ("out", "out2")}
    for b, (nq, nk) in enumerate(zip(_lengths(NQ, q_len, B), _lengths(NK, kv_len, B))):
        ok = visible(NQ, NK, nq, nk, causal)
        for h in range(H):
            j = h // (H // HK)
            val = _clean(v[b, j], nk)
            p1, l1 = _maps(_clean(q1[b, h], nq), _clean(k1[b, j], nk), scale, ok)
            p2, l2 = _maps(_clean(q2[b, h], nq), _clean(k2[b, j], nk), scale, ok)
            o2 = p2 @ val
            out = p1 @ val - lam[h] * o2
            a1, a2 = p1 @ np.abs(val), p2 @ np.abs(val)
            res["out"][b, h], res["out2"][b, h], res["lse1"][b, h], res["lse2"][b, h] = out, o2, l1, l2
            t2 = (HALF + F32) * a2                        # P_2 rounded
            tol["out2"][b, h] = t2 + HALF * (np.abs(o2) + t2)
            t = (HALF + F32) * (a1 + abs(lam[h]) * a2)    # both maps
            tol["out"][b, h] = t + HALF * (np.abs(out) + t)
    return res, tol


def diff_backward(q1, k1, q2, k2, v, lam, scale, causal, dout, q_len=None, kv_len=None, half=0.0):
    """Gradients {"dq1", "dk1", "dq2", "dk2", "dv", "dlam"} and their bounds; half: relative rounding of a gradient."""
    B, H, NQ, _ = q1.shape
    HK, NK, _ = v.shape[1:]
    fwd, ftol = diff(q1, k1, q2, k2, v, lam, scale, causal, q_len, kv_len)
    shapes = {"dq1": q1.shape, "dk1": k1.shape, "dq2": q2.shape, "dk2": k2.shape, "dv": v.shape, "dlam": (H,)}
    g, t = ({n: np.zeros(s) for n, s in shapes.items()} for _ in range(2))
    for b, (nq, nk) in enumerate(zip(_lengths(NQ, q_len, B), _lengths(NK, kv_len, B))):
        ok = visible(NQ, NK, nq, nk, causal)
        for h in range(H):
            j, lh = h // (H // HK), float(lam[h])
            x1, x2 = _clean(q1[b, h], nq), _clean(q2[b, h], nq)
            y1, y2, val = (_clean(x[b, j], nk) for x in (k1, k2, v))
            do = _clean(dout[b, h], nq)
            p1, _ = _maps(x1, y1, scale, ok)
            p2, _ = _maps(x2, y2, scale, ok)
            dp, dpa = do @ val.T, np.abs(do) @ np.abs(val).T
            o2 = fwd["out2"][b, h]
            o1 = fwd["out"][b, h] + lh * o2
            d1, d2 = (do * o1).sum(1), (do * o2).sum(1)
            # D_t comes from the rounded outputs
            e2 = (np.abs(do) * ftol["out2"][b, h]).sum(1)
            e1 = (np.abs(do) * ftol["out"][b, h]).sum(1) + abs(lh) * e2
            for p, d, e, f, x, y, n in ((p1, d1, e1, 1.0, x1, y1, "1"), (p2, d2, e2, -lh, x2, y2, "2")):
                ds = f * p * (dp - d[:, None])
                err = abs(f) * p * (e[:, None] + F32 * (dpa + np.abs(d)[:, None]))
                err = err + HALF * (np.abs(ds) + err)
                g["dq" + n][b, h] = scale * (ds @ y)
                g["dk" + n][b, j] += scale * (ds.T @ x)
                t["dq" + n][b, h] = scale * (err @ np.abs(y))
                t["dk" + n][b, j] += scale * (err.T @ np.abs(x))
            g["dv"][b, j] += (p1 - lh * p2).T @ do
            t["dv"][b, j] += (HALF * np.abs(p1 - lh * p2) + F32 * (p1 + abs(lh) * p2)).T @ np.abs(do)
            g["dlam"][h] -= (p2 * dp).sum()
            t["dlam"][h] += F32 * (p2 * dpa).sum()
    for n in shapes:
        if n != "dlam":
            t[n] = t[n] + half * (np.abs(g[n]) + t[n])
    return g, t
