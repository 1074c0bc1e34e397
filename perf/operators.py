"""Performance cases of the operators around the divergence of two attention maps: what a program has them do.

  norm_rope    norms of queries and keys per head with the position rotation in the same pass (qk_norm_rope), from a
               projection's token-major [B, N, H, d] to the head-major bf16 that the attention operators read;
  diff         differential attention (diff_attention), O = (softmax(s q1 k1^T) - lam_h softmax(s q2 k2^T)) v.

``call`` is "fwd" (no gradients: evaluation, serving) or "step" (outputs and the gradients of everything learned).
With ``own`` false ``run`` computes the operators from elementary operations in 32 bits, rounded once at the end; with
``own`` true it calls the package's operators.
"""
import math

import torch

own = False


def _norm_rope(name, call, B, nq, nk, H, Hk, d, rot, dtype="bf16", interleaved=False, expand=False, far=False):
    return {"name": name, "op": "norm_rope", "call": call, "B": B, "nq": nq, "nk": nk, "H": H, "Hk": Hk, "d": d,
            "rot": rot, "dtype": dtype, "interleaved": interleaved, "expand": expand, "far": far}


def _diff(name, call, B, nq, nk, H, Hk, d, dv, causal, lengths=False, projected=False):
    return {"name": name, "op": "diff", "call": call, "B": B, "nq": nq, "nk": nk, "H": H, "Hk": Hk, "d": d, "dv": dv,
            "causal": causal, "lengths": lengths, "projected": projected}


def listed():
    return [
        # one new token per sequence of a served batch, each at a position of its own: launches are the cost
        _norm_rope("norm_rope_decode", "fwd", 16, 1, 1, 16, 4, 128, 128, far=True),
        # evaluation at a 4K context, shared key heads written once per query head, as attention_kl reads them
        _norm_rope("norm_rope_eval", "fwd", 2, 4096, 4096, 16, 4, 128, 128, expand=True),
        # fine-tuning on short ragged sequences in float32, a partial rotation of adjacent pairs, d no power of two
        _norm_rope("norm_rope_step_ragged", "step", 4, 1021, 1021, 12, 12, 96, 64, dtype="fp32", interleaved=True),
        # a training step at a 16K context with shared key heads
        _norm_rope("norm_rope_step_mid", "step", 1, 16384, 16384, 32, 8, 128, 128),
        # the smallest training step: one 256-token head, where launches and host work are the cost
        _diff("diff_step_tiny", "step", 1, 256, 256, 1, 1, 64, 64, False),
        # fine-tuning on a right-padded batch of short sequences, shared heads, dims that are no multiples of 64
        _diff("diff_step_padded", "step", 4, 1021, 1021, 12, 4, 96, 160, True, lengths=True),
        # a training step at a 4K context, values twice as wide as the keys, as they leave the value projection
        _diff("diff_step", "step", 2, 4096, 4096, 16, 16, 64, 128, True, projected=True),
        # a training step without the causal mask (an encoder), odd length
        _diff("diff_step_encoder", "step", 1, 6007, 6007, 8, 8, 128, 128, False),
        # the prompt of a 16K context, wide heads, shared keys and values
        _diff("diff_prefill", "fwd", 1, 16384, 16384, 16, 4, 128, 256, True),
        # one new token per sequence against caches of up to 64K tokens, filled to different lengths
        _diff("diff_decode", "fwd", 16, 1, 65536, 16, 4, 64, 128, True, lengths=True),
        # one new token of a single sequence: few rows and a long axis
        _diff("diff_decode_one", "fwd", 1, 1, 32768, 8, 8, 128, 128, True),
        # the last 8K tokens of a 128K context (causal by absolute position)
        _diff("diff_tail", "fwd", 1, 8192, 131072, 8, 2, 64, 64, True),
    ]


def draw(rng):
    """One more case of the listed ranges: every call, mask, type, head layout and head dim; sizes spread over their
    logarithms and mostly odd, no dearer than the dearest listed case of the operator."""
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {}
    for c in listed():
        w = work(c)
        for k in ("bytes", "flops"):
            most[c["op"], k] = max(most.get((c["op"], k), 0), w[k])
    while True:
        call = rng.choice(("fwd", "step"))
        B, Hk, G = rng.choice((1, 1, 2, 3, 4, 16)), logint(1, 16), rng.choice((1, 1, 2, 3, 4, 8))
        if rng.random() < 0.35:
            d = rng.choice((64, 128, 32, 96, 160, 192, 224, 256))
            n = logint(1, 16384)
            nk = n if rng.random() < 0.7 else logint(n, 32768)
            c = _norm_rope("", call, B, n, nk, Hk * G, Hk, d, rng.choice((d, d, d // 2, 0)),
                           dtype=rng.choice(("bf16", "bf16", "fp16", "fp32")), interleaved=rng.random() < 0.3,
                           expand=rng.random() < 0.3, far=rng.random() < 0.5)
        else:
            d, dv = rng.choice((64, 128, 64, 128, 32, 96)), rng.choice((64, 128, 256, 128, 32, 96, 160, 192, 224))
            shape = rng.choice(("square", "square", "few", "tail") if call == "fwd" else ("square", "square", "tail"))
            if shape == "square":
                nq = nk = logint(60, 16384)
            elif shape == "few":
                nq, nk = rng.choice((1, 1, 1, 2, 5, 16, 61)), logint(500, 66000)
            else:
                nk = logint(2000, 66000)
                nq = max(1, int(nk * rng.uniform(0.02, 0.2)))
            c = _diff("", call, B, nq, nk, Hk * G, Hk, d, dv, rng.random() < 0.7, lengths=rng.random() < 0.4,
                      projected=rng.random() < 0.4)
        del c["name"]
        w = work(c)
        if all(w[k] <= most[c["op"], k] for k in w) and B * Hk * G <= 128:
            return c


# --- inputs -----------------------------------------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    step = c["call"] == "step"
    s = {"case": c}
    if c["op"] == "norm_rope":
        t = _TYPES[c["dtype"]]
        # a projection's output: token-major, heads of unequal size
        s["q"] = (normal(c["B"], c["nq"], c["H"], c["d"]) * (0.5 + normal(c["H"], 1).abs())).to(t)
        s["k"] = (normal(c["B"], c["nk"], c["Hk"], c["d"]) * (0.5 + normal(c["Hk"], 1).abs())).to(t)
        s["wq"], s["wk"] = 1.0 + 0.2 * normal(c["d"]), 1.0 + 0.2 * normal(c["d"])
        first = 100000 if c["far"] else 0   # a context that went on for long
        if c["rot"]:
            # cosines, then sines, of every position: what a program lays out once
            pos = torch.arange(first + c["nk"] + 64, device="cuda", dtype=torch.float64)
            freq = 10000.0 ** (torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / -c["rot"])
            angle = pos[:, None] * freq[None, :]
            s["table"] = torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()
        else:
            s["table"] = None
        if c["far"] and c["rot"]:   # every sequence at a place of its own
            start = first + torch.randint(0, 64, (c["B"], 1), generator=gen, device="cuda")
            at = torch.arange(c["nk"], device="cuda")[None, :] + start
            s["kpos"] = at.to(torch.int32).contiguous()
            s["qpos"] = s["kpos"][:, c["nk"] - c["nq"]:].contiguous()
        else:
            s["kpos"] = s["qpos"] = None
        if step:
            g = c["H"] // c["Hk"] if c["expand"] else 1
            s["dq"] = normal(c["B"], c["H"], c["nq"], c["d"]).bfloat16()
            s["dk"] = normal(c["B"], c["Hk"] * g, c["nk"], c["d"]).bfloat16()
            for n in ("q", "k", "wq", "wk"):
                s[n].requires_grad_(True)
        return s
    for n, h, rows in (("q1", "H", "nq"), ("k1", "Hk", "nk"), ("q2", "H", "nq"), ("k2", "Hk", "nk")):
        s[n] = normal(c["B"], c[h], c[rows], c["d"]).bfloat16()   # normed and rotated queries and keys
    if c["projected"]:   # values stay where their projection wrote them, token-major
        s["v"] = normal(c["B"], c["nk"], c["Hk"], c["dv"]).bfloat16().transpose(1, 2)
    else:
        s["v"] = normal(c["B"], c["Hk"], c["nk"], c["dv"]).bfloat16()
    s["lam"] = 0.2 + 0.6 * torch.rand(c["H"], generator=gen, device="cuda")
    s["qlen"] = s["klen"] = None
    if c["lengths"]:
        u = torch.rand(c["B"], generator=gen, device="cuda")
        if c["nq"] == c["nk"]:   # a right-padded batch
            s["klen"] = s["qlen"] = (c["nk"] - (u * 0.6 * c["nk"]).int()).to(torch.int32)
        else:                    # caches filled to different lengths
            s["klen"] = (c["nk"] - (u * 0.6 * (c["nk"] - c["nq"])).int()).to(torch.int32)
    if step:
        s["do"] = normal(c["B"], c["H"], c["nq"], c["dv"]).bfloat16()
        for n in ("q1", "k1", "q2", "k2", "v", "lam"):
            s[n] = s[n].requires_grad_(True)
    return s


# --- one pass ---------------------------------------------------------------------------------------------------------


def run(state):
    s, c = state, state["case"]
    if c["op"] == "norm_rope":
        return _run_norm_rope(s, c) if own else _plain_norm_rope(s, c)
    return _run_diff(s, c) if own else _plain_diff(s, c)


def _run_norm_rope(s, c):
    from paper_2606_20005_amd import streamkl as sk
    opts = {"eps": EPS, "q_positions": s["qpos"], "k_positions": s["kpos"], "interleaved": c["interleaved"],
            "expand_k": c["expand"]}
    if c["call"] == "fwd":
        return sk.qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["table"], **opts)
    y = sk.qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["table"], **opts)
    grads = torch.autograd.grad(y, [s[n] for n in ("q", "k", "wq", "wk")], (s["dq"], s["dk"]))
    return [*(x.detach() for x in y), *grads]


def _run_diff(s, c):
    from paper_2606_20005_amd import streamkl as sk
    args = [s[n] for n in ("q1", "k1", "q2", "k2", "v", "lam")]
    out = sk.diff_attention(*args, causal=c["causal"], q_len=s["qlen"], kv_len=s["klen"])
    if c["call"] == "fwd":
        return out
    return [out.detach(), *torch.autograd.grad(out, args, s["do"])]


# --- the plain form ---------------------------------------------------------------------------------------------------


def _pairs(x, interleaved):
    """The two members of every rotated pair along the last axis."""
    if interleaved:
        return x[..., 0::2], x[..., 1::2]
    half = x.shape[-1] // 2
    return x[..., :half], x[..., half:]


def _joined(a, b, interleaved):
    return torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)


def _plain_side(x, w, dy, c, table, pos, start, copies):
    """One side: (y, dx, dw); x [B, N, H, d], y [B, H copies, N, d]."""
    xf, rot = x.detach().float(), c["rot"]
    r = torch.rsqrt((xf * xf).mean(-1, keepdim=True) + EPS)
    xh = xf * r
    y = xh * w.detach()
    if rot:
        if pos is None:
            cs = table[start:start + x.shape[1]][None, :, None, :]
        else:
            cs = table[pos.long()][:, :, None, :]
        co, si = cs[..., :rot // 2], cs[..., rot // 2:]
        a, b = _pairs(y[..., :rot], c["interleaved"])
        y = torch.cat((_joined(a * co - b * si, b * co + a * si, c["interleaved"]), y[..., rot:]), -1)
    out = y.transpose(1, 2).repeat_interleave(copies, 1).contiguous().bfloat16()
    if dy is None:
        return out, None, None
    B, N, H, d = x.shape
    g = dy.float().view(B, H, copies, N, d).sum(2).transpose(1, 2)
    if rot:
        a, b = _pairs(g[..., :rot], c["interleaved"])
        g = torch.cat((_joined(a * co + b * si, b * co - a * si, c["interleaved"]), g[..., rot:]), -1)
    h = g * w.detach()
    dx = r * (h - xh * (h * xh).mean(-1, keepdim=True))
    return out, dx.to(x.dtype), (g * xh).sum((0, 1, 2))


def _plain_norm_rope(s, c):
    copies = c["H"] // c["Hk"] if c["expand"] else 1
    dq, dk = (s["dq"], s["dk"]) if c["call"] == "step" else (None, None)
    yq, gq, gwq = _plain_side(s["q"], s["wq"], dq, c, s["table"], s["qpos"], c["nk"] - c["nq"], 1)
    yk, gk, gwk = _plain_side(s["k"], s["wk"], dk, c, s["table"], s["kpos"], 0, copies)
    return (yq, yk) if dq is None else [yq, yk, gq, gk, gwq, gwk]


def _visible_pairs(c, qlen, klen, r0, r1, dev):
    """Pairs of the rows r0 .. r1 - 1 that the masks leave, [B or 1, 1, 1, rows, N_K]."""
    rows = torch.arange(r0, r1, device=dev)[:, None]
    cols = torch.arange(c["nk"], device=dev)[None, :]
    nq = c["nq"] if qlen is None else qlen[:, None, None]
    nk = c["nk"] if klen is None else klen[:, None, None]
    seen = (cols < nk) & (rows < nq)
    if c["causal"]:
        seen = seen & (cols <= rows + (nk - nq))
    return seen.reshape(-1, 1, 1, r1 - r0, c["nk"])


def _plain_map(q, k, seen):
    """softmax of the visible logits of q [B, Hk, G, rows, d] (scaled) and k [B, Hk, N_K, d]; rows that see nothing: 0."""
    z = (q.flatten(2, 3) @ k.transpose(2, 3).contiguous()).view(*q.shape[:4], -1)
    z = z.masked_fill(~seen, -math.inf)
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
    return e / e.sum(-1, keepdim=True).clamp_min(1e-37)


def _plain_diff(s, c):
    step, G, scale = c["call"] == "step", c["H"] // c["Hk"], 1.0 / math.sqrt(c["d"])
    q1, q2 = (s[n].detach().float().unflatten(1, (c["Hk"], G)) for n in ("q1", "q2"))
    k1, k2, v = (s[n].detach().float().contiguous() for n in ("k1", "k2", "v"))
    lam = s["lam"].detach().view(c["Hk"], G, 1, 1)
    out = torch.empty(*q1.shape[:4], c["dv"], device=q1.device)
    if step:
        do = s["do"].float().unflatten(1, (c["Hk"], G))
        g1, h1, g2, h2, gv = (torch.zeros_like(x) for x in (q1, k1, q2, k2, v))
        gl = torch.zeros_like(lam)
    # the maps of all heads at once, as many rows at a time as keep one of them within 2 GB
    block = max(1, min(c["nq"], (1 << 29) // (c["B"] * c["H"] * c["nk"])))
    for r0 in range(0, c["nq"], block):
        r = slice(r0, min(c["nq"], r0 + block))
        seen = _visible_pairs(c, s["qlen"], s["klen"], r.start, r.stop, q1.device)
        p1, p2 = (_plain_map(q[:, :, :, r] * scale, k, seen) for q, k in ((q1, k1), (q2, k2)))
        p = (p1 - lam * p2).flatten(2, 3)
        out[:, :, :, r] = (p @ v).unflatten(2, (G, -1))
        if not step:
            continue
        dor = do[:, :, :, r].flatten(2, 3)
        gv += p.transpose(2, 3).contiguous() @ dor
        dp = (dor @ v.transpose(2, 3).contiguous()).view(p1.shape)
        d2 = (p2 * dp).sum(-1, keepdim=True)
        gl -= d2.sum((0, 3), keepdim=True)[0]
        ds1 = (p1 * (dp - (p1 * dp).sum(-1, keepdim=True)) * scale).flatten(2, 3)
        ds2 = (p2 * (dp - d2) * (-scale * lam)).flatten(2, 3)
        g1[:, :, :, r] = (ds1 @ k1).unflatten(2, (G, -1))
        g2[:, :, :, r] = (ds2 @ k2).unflatten(2, (G, -1))
        h1 += ds1.transpose(2, 3).contiguous() @ q1[:, :, :, r].flatten(2, 3)
        h2 += ds2.transpose(2, 3).contiguous() @ q2[:, :, :, r].flatten(2, 3)
    out = out.flatten(1, 2).bfloat16()
    if not step:
        return out
    return [out, *(x.bfloat16() for x in (g1.flatten(1, 2), h1, g2.flatten(1, 2), h2, gv)), gl.flatten()]


# --- what a pass cannot do without ------------------------------------------------------------------------------------


def _visible(c):
    """(query, key) pairs of one head and sequence that the causal mask leaves, lengths at their mean (0.7)."""
    nq, nk = float(c["nq"]), float(c["nk"])
    if c["lengths"]:
        if nq == nk:
            nq = nk = 0.7 * nk
        else:
            nk = nk - 0.3 * (nk - nq)
    if not c["causal"]:
        return nq * nk, nk
    first = nk - nq + 1
    return nq * (max(first, 1.0) + nk) / 2, nk


def work(case):
    """Inputs read once, outputs written once. Norm and rotation: about 10 operations an element forward, 25 more
    backward. Differential attention: 4 d (logits) and 4 dv (products with the values) operations a visible pair
    forward, 12 d + 4 dv in the backward pass (logits again, one product with the upstream gradient for both maps, and
    the gradients)."""
    c, step = case, case["call"] == "step"
    if c["op"] == "norm_rope":
        es = 4 if c["dtype"] == "fp32" else 2
        nx = c["B"] * (c["nq"] * c["H"] + c["nk"] * c["Hk"]) * c["d"]
        ny = c["B"] * (c["nq"] * c["H"] + c["nk"] * (c["H"] if c["expand"] else c["Hk"])) * c["d"]
        table = 4 * c["nk"] * c["rot"]
        n = nx * es + 2 * ny + table
        return {"bytes": n + (2 * nx * es + 2 * ny if step else 0), "flops": (35 if step else 10) * nx}
    pairs, keys = _visible(c)
    pairs *= c["B"] * c["H"]
    qo = 2 * c["B"] * c["H"] * c["nq"] * (2 * c["d"] + c["dv"])
    kv = int(2 * c["B"] * c["Hk"] * keys) * (2 * c["d"] + c["dv"])
    flops = 4 * (c["d"] + c["dv"]) + (12 * c["d"] + 4 * c["dv"] if step else 0)
    # a step reads the upstream gradient and writes the gradients too
    extra = qo + kv + 2 * c["B"] * c["H"] * c["nq"] * c["dv"] if step else 0
    return {"bytes": int(qo + kv + extra), "flops": int(flops * pairs)}


# --- the same in 64 bits, from the definitions ------------------------------------------------------------------------


def _exact_side(x, w, c, table, pos, start, copies):
    """y of one side as a function of x and w in float64; rotations as products with complex numbers."""
    y = x / torch.sqrt(torch.mean(x ** 2, dim=-1, keepdim=True) + EPS) * w
    y = y.permute(0, 2, 1, 3)
    rot = c["rot"]
    if rot:
        rows = table.double()
        rows = rows[start:start + x.shape[1]].unsqueeze(0) if pos is None else rows[pos.long()]
        turn = torch.complex(rows[..., :rot // 2], rows[..., rot // 2:]).unsqueeze(1)
        head = y[..., :rot]
        if c["interleaved"]:
            z = torch.view_as_complex(head.unflatten(-1, (rot // 2, 2)).contiguous()) * turn
            head = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(head[..., :rot // 2], head[..., rot // 2:]) * turn
            head = torch.cat((z.real, z.imag), -1)
        y = torch.cat((head, y[..., rot:]), -1)
    B, H, N, d = y.shape
    return y.unsqueeze(2).expand(B, H, copies, N, d).reshape(B, H * copies, N, d)


def _exact_norm_rope(s, c):
    step = c["call"] == "step"
    copies = c["H"] // c["Hk"] if c["expand"] else 1
    sides = []
    for x, w, dy, pos, start, n in ((s["q"], s["wq"], s.get("dq"), s["qpos"], c["nk"] - c["nq"], 1),
                                    (s["k"], s["wk"], s.get("dk"), s["kpos"], 0, copies)):
        x, w = x.detach().double().requires_grad_(step), w.detach().double().requires_grad_(step)
        y = _exact_side(x, w, c, s["table"], pos, start, n)
        sides.append((y.detach(), *(torch.autograd.grad(y, (x, w), dy.double()) if step else ())))
    (yq, *gq), (yk, *gk) = sides
    return [yq, yk, gq[0], gk[0], gq[1], gk[1]] if step else (yq, yk)


def _exact_diff(s, c):
    step, G = c["call"] == "step", c["H"] // c["Hk"]
    B, H, nq, dv = c["B"], c["H"], c["nq"], c["dv"]
    dev = s["q1"].device
    qlen = [nq] * B if s["qlen"] is None else s["qlen"].tolist()
    klen = [c["nk"]] * B if s["klen"] is None else s["klen"].tolist()
    names = ("q1", "k1", "q2", "k2", "v")
    out = torch.zeros(B, H, nq, dv, dtype=torch.float64, device=dev)
    grads = {n: torch.zeros(s[n].shape, dtype=torch.float64, device=dev) for n in names} if step else {}
    glam = torch.zeros(H, dtype=torch.float64, device=dev)
    for b in range(B):
        n, m = qlen[b], klen[b]
        for h in range(H):
            j = h // G
            q1, q2 = s["q1"].detach()[b, h, :n].double(), s["q2"].detach()[b, h, :n].double()
            k1, k2, v = (s[x].detach()[b, j, :m].double() for x in ("k1", "k2", "v"))
            lam = float(s["lam"][h])
            block = max(1, (1 << 26) // max(1, m))
            for lo in range(0, n, block):
                hi = min(n, lo + block)
                seen = max(0, min(m, m - n + hi)) if c["causal"] else m   # keys that any row of the block sees
                if seen == 0:
                    continue
                keys = torch.arange(seen, device=dev)
                last = torch.arange(lo, hi, device=dev) + (m - n)
                maps = []
                for q, k in ((q1, k1), (q2, k2)):
                    z = torch.matmul(q[lo:hi], k[:seen].t().contiguous()).div_(math.sqrt(c["d"]))
                    if c["causal"]:
                        z.masked_fill_(keys[None] > last[:, None], -math.inf)
                    maps.append(torch.softmax(z, dim=1).nan_to_num_(nan=0.0))   # rows that see nothing: 0
                a1, a2 = maps
                o1, o2 = a1 @ v[:seen], a2 @ v[:seen]
                out[b, h, lo:hi] = o1 - lam * o2
                if not step:
                    continue
                do = s["do"][b, h, lo:hi].double()
                dp = do @ v[:seen].t().contiguous()
                glam[h] -= (do * o2).sum()
                grads["v"][b, j, :seen] += a1.t().contiguous() @ do - lam * (a2.t().contiguous() @ do)
                for a, o, q, k, f, x in ((a1, o1, q1, k1, 1.0, "1"), (a2, o2, q2, k2, -lam, "2")):
                    dz = a * (dp - (do * o).sum(1)[:, None]) * (f / math.sqrt(c["d"]))
                    grads["q" + x][b, h, lo:hi] = dz @ k[:seen]
                    grads["k" + x][b, j, :seen] += dz.t().contiguous() @ q[lo:hi]
    return [out, *(grads[n] for n in names), glam] if step else out


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    return _exact_norm_rope(s, c) if c["op"] == "norm_rope" else _exact_diff(s, c)
