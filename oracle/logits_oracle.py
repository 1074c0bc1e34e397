"""Plain fp64 NumPy forms of the operators on rows of logits, for the tests.

token_logprobs / token_logprobs_grad: log probabilities, entropies, best tokens (streamkl_token_logprobs_*).
distill / distill_grad: divergence from a teacher's best tokens (streamkl_topk_distill_*).

Rows are [R, V]. Every function also returns how far a computation may be from it that holds sums and exponents in
float32, U = 2^-24 a rounding, and rounds each result once to its type (the caller's part). A probability is
exp2((x - r) c): the difference, the product and c are each off by U of themselves, which the exponential turns into
3 U |z - r| of the term, and the exponential by 2 U. A reference r is within 4 ln 2 < 3 of the largest logit it has
seen. The sums: at least 64 lanes share a row, so that a lane adds at most V / 64 terms. In long rows it adds far fewer
one after the other: the terms of a turn (at most 32 logits a lane) come in four chains of up to 8, 9 additions, and are
added to the lane's sum at once; 256 threads take at least 2048 logits a turn, of parts of at most 16384, and 512
threads at least 4096, so that there are at most V / 4096 + 9 turns. Three joins (a wave, a workgroup, parts) with 15
additions and three moves of a reference, 3 U each, come to 24 roundings; 20 of them count everywhere, short rows having
fewer levels. So a sum of exponentials, relative, and with it its logarithm, absolute, is off by at most
    SUM = U (3 (D + 3) + 22 + min(V / 64, V / 4096 + 24)),    D = sum_j p_j |z_j - max z|.
"""
import numpy as np

U = 2.0 ** -24
LEAST_REST = 2.0 ** -24


def _sum_error(d, V):
    """SUM, for d the distance D."""
    return U * (3 * (d + 3) + 22 + min(V / 64, V / 4096 + 24))


def _softmax(x, scale):
    """(log p, p, lse, error of lse) of rows; an empty row has p = 0, lse = log p = -inf. Log probabilities are formed from
    differences: a log-sum-exp near the type's lowest value swallows them even in 64 bits."""
    z = x.astype(np.float64) * scale
    m = z.max(-1, keepdims=True)
    safe = np.where(np.isneginf(m), 0.0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.exp(z - safe)
        total = e.sum(-1, keepdims=True)
        lse = np.where(total > 0, safe + np.log(total), -np.inf)
        p = np.where(total > 0, e / total, 0.0)
        d = np.where(p > 0, p * np.abs(z - safe), 0.0).sum(-1)
        lp = np.where(total > 0, (z - safe) - np.log(total), -np.inf)
    return lp, p, lse[:, 0], _sum_error(d, x.shape[-1])


def _entropy_terms(p, lp):
    return np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0)


def token_logprobs(x, tokens, scale, top):
    """dict of value, bound: logp, entropy, lse, top_logp, and top_ids."""
    R, V = x.shape
    lp, p, lse, err = _softmax(x, scale)
    ent = -_entropy_terms(p, lp).sum(-1)
    wide = np.abs(_entropy_terms(p, lp)).sum(-1) + 3
    out = {"lse": (lse, err + U * np.where(np.isfinite(lse), np.abs(lse), 0)),
           # l and a are both off by err of sum p |log p|, of logits relative to a reference up to 3 away
           "entropy": (ent, err * (2 + 2 * wide) + U * np.abs(ent))}
    if tokens is not None:
        t = np.asarray(tokens)
        ok = (t >= 0) & (t < V)
        v = np.where(ok, lp[np.arange(R), np.where(ok, t, 0)], np.where(t < 0, 0.0, np.nan))
        out["logp"] = (v, err + U * np.where(np.isfinite(v), np.abs(v), 0))
    if top:
        ids = np.argsort(-x.astype(np.float64), axis=-1, kind="stable")[:, :top]
        v = np.take_along_axis(lp, ids, -1)
        out["top_ids"] = ids
        out["top_logp"] = (v, err[:, None] + U * np.where(np.isfinite(v), np.abs(v), 0))
    return out


def token_logprobs_grad(x, tokens, scale, dlogp, dent, dlse):
    """(dx, bound) for upstream gradients [R] of logp, entropy and lse; the rounding of dx to its type is not in it."""
    R, V = x.shape
    lp, p, lse, err = _softmax(x, scale)
    lp = np.where(p > 0, lp, 0.0)
    ent = -_entropy_terms(p, lp).sum(-1)
    g, h, e = (np.zeros(R) if v is None else v.astype(np.float64) for v in (dlogp, dent, dlse))
    if tokens is not None:
        g = np.where(np.asarray(tokens) >= 0, g, 0.0)
    col = lambda v: v[:, None]   # noqa: E731
    dx = p * (col(e - g) - col(h) * (lp + col(ent)))
    size = p * (np.abs(col(e)) + np.abs(col(g)) + np.abs(col(h)) * (np.abs(lp) + np.abs(col(ent))))
    # p is off by 3 U |z - lse| and a few roundings, log p by 3 U |z - lse|, lse and the entropy by their own error
    rel = U * (3 * np.abs(lp) + 10) + col(err)
    bound = size * rel + p * np.abs(col(h)) * (rel + col(err * (2 + 2 * (np.abs(_entropy_terms(p, lp)).sum(-1) + 3))))
    if tokens is not None:
        t = np.asarray(tokens)
        rows = np.nonzero((t >= 0) & (t < V) & ~np.isneginf(lse))[0]
        dx[rows, t[rows]] += g[rows]
        bound[rows, t[rows]] += 4 * U * np.abs(g[rows])
    return scale * dx, scale * bound + 1e-36


def _row(z, ids, t, s1, rest, reverse):
    """Loss and d loss / dz of one row from the definition, over the buckets of its list and the rest; and the sizes that
    errors count with: (loss, dz, of the loss, of dz, |log q_r| with the relative error of q_r)."""
    V = z.shape[0]
    keep = ids >= 0
    ids, t = ids[keep], t[keep].astype(np.float64)
    if len(ids) == 0 or not np.isfinite(z).any():
        return 0.0, np.zeros(V), 0.0, np.zeros(V), (0.0, 0.0)
    lz = (z - z.max()) - np.log(np.exp(z - z.max()).sum())   # log q
    q, lq = np.exp(lz), lz[ids]
    outside = np.ones(V, bool)
    outside[ids] = False
    if rest:
        p, lp = np.exp(t), t
        pr = max(1.0 - p.sum(), LEAST_REST)
    else:
        u = s1 * (t - t.max())   # an absolute log-sum-exp would swallow what values near the type's lowest one differ by
        lp = u - np.log(np.exp(u).sum())
        p, pr = np.exp(lp), 0.0
    others = rest and np.isfinite(z[outside]).any()
    qr, lqr, err_r = 0.0, 0.0, 0.0
    if others:
        zr = z[outside]
        er = np.exp(zr - zr.max())
        err_r = _sum_error(np.where(er > 0, er * np.where(er > 0, zr.max() - zr, 0.0), 0.0).sum() / er.sum(), V)
        lqr = lz[outside].max() + np.log(er.sum())
        qr = np.exp(lqr)
    else:
        pr = 0.0
    lpr = np.log(pr) if pr > 0 else 0.0
    qk = np.exp(lq)
    dz, size = np.zeros(V), np.zeros(V)
    with np.errstate(invalid="ignore", divide="ignore"):
        if not reverse:
            loss = np.where(p > 0, p * (lp - lq), 0.0).sum() + (pr * (lpr - lqr) if others else 0.0)
            total = p.sum() + pr
            dz[:] = q * total
            np.add.at(dz, ids, -p)
            if others:   # the share of the bucket
                dz[outside] -= pr * er / er.sum()
            size[:] = q * total
            if others:
                size[outside] += pr * er / er.sum()
            np.add.at(size, ids, p * 2.0 ** -3)   # entries are added in float32
            moved = total
        else:
            r = np.where(qk > 0, lq - lp, 0.0)
            loss = (qk * r).sum() + (qr * (lqr - lpr) if others else 0.0)
            mass = qk.sum() + qr
            dz[:] = -q * (loss + mass)
            np.add.at(dz, ids, qk * (r + 1))
            size[:] = q * (abs(loss) + mass)
            np.add.at(size, ids, qk * (np.abs(r) + 2))
            moved = (qk * (np.abs(r) + 2)).sum()
            if others:
                dz[outside] += q[outside] * (lqr - lpr + 1)
                size[outside] += q[outside] * (abs(lqr - lpr) + 2)
                moved += qr * (abs(lqr - lpr) + 2)
            size += q * moved
    return float(loss), dz, float(moved), size, (abs(lqr), err_r)


def distill(x, ids, t, s1, s2, rest, reverse, g=None):
    """(loss [R], bound, dx [R, V], bound) for upstream gradients g [R] (None: ones). Rows whose lists name a token outside
    the vocabulary are NaN."""
    R, V = x.shape
    lp, p, _, err = _softmax(x, s2)
    z = x.astype(np.float64) * s2
    loss, lb = np.zeros(R), np.zeros(R)
    dx, db = np.zeros((R, V)), np.zeros((R, V))
    g = np.ones(R) if g is None else g.astype(np.float64)
    for r in range(R):
        if (ids[r] >= V).any():
            loss[r], dx[r] = np.nan, np.nan if g[r] else 0.0
            continue
        loss[r], dz, moved, size, (far, err_r) = _row(z[r], ids[r].astype(np.int64), t[r], s1, rest, reverse)
        both = err[r] + err_r
        lb[r] = 2 * both * moved + 2 * U * abs(loss[r]) + 1e-12
        with np.errstate(invalid="ignore"):   # probabilities are formed from z - lse_r = z - lse - log q_r
            rel = U * (3 * (np.where(p[r] > 0, np.abs(lp[r]), 0.0) + far) + 10) + 2 * both
        dx[r] = g[r] * s2 * dz
        db[r] = abs(g[r]) * s2 * size * rel + 1e-36
    return loss, lb, dx, db
