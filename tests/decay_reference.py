"""Plain 64-bit implementations of attention with a decay per head and of trees of drafted tokens, from their definitions, and
how far a kernel may be from them.

Bounds.  A kernel that rounds operands to the element type (half step u = finfo.eps / 2, relative) forms every result from terms
of which each has met one such rounding (a masked tile's value, or the state's copy) and rounds the result once; what it returns
in fp32 has operands in two parts, each product off by at most u^2 (fp32 rows: by nothing but fp32 rounding).  With
M = sum over j of |the terms' factors|, which also bounds what the state contributes, element by element

    |got - ref| <= u |ref| + (u + n 2^-23) M        results in the element type
    |got - ref| <= (2 u^2 + n 2^-23) M              states, ds

for sums of n terms and products of at most n more fp32 roundings; weights g^n add a few 2^-24, which the factor two of
2^-23 holds.  Second-order terms take SLACK.

In fp16 an operand below 2^-14 is off by up to 2^-25 however small it is.  That shows where everything that a row sees has
been forgotten but for such weights (its chunk's 64 values p_ij <= 1, each times a value; and the state's copy, times the
unit row q): `floor` is 2^-25 s (64 max |v| + sqrt(dk)) for O, with dO in v's place for dV.
"""
import torch

SLACK = 1.05
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def unit(x, eps):
    """Rows over max(norm, eps), and that divisor."""
    n = x.norm(dim=-1, keepdim=True).clamp(min=eps)
    return x / n, n


def weights(log_decay, n):
    """[H, n, n]: g^(i-j), 0 above the diagonal; g^0 = 1 also for log_decay = -inf."""
    i = torch.arange(n, dtype=torch.float64)
    apart = i[:, None] - i[None, :]
    w = powers(log_decay, apart.clamp(min=0))
    return torch.where(apart >= 0, w, torch.zeros_like(w))


def powers(log_decay, e):
    ld = torch.clamp(log_decay.double(), min=-1e30, max=0.0)
    return torch.exp(ld.view((-1,) + (1,) * e.dim()) * e)


def forward(Q, K, V, s, log_decay, lens=None, state_in=None, eps=1e-6):
    """float64 [B, H, N, d] in; (O, state, M_O, M_state)."""
    B, H, N, dk = Q.shape
    dv = V.shape[-1]
    O, MO = torch.zeros(B, H, N, dv, dtype=torch.float64), torch.zeros(B, H, N, dv, dtype=torch.float64)
    S, MS = torch.zeros(B, H, dk, dv, dtype=torch.float64), torch.zeros(B, H, dk, dv, dtype=torch.float64)
    for b in range(B):
        n = N if lens is None else int(min(max(lens[b], 0), N))
        sc = (s if lens is None else s[b]).double().view(H, 1, 1)
        qh, kh, v = unit(Q[b, :, :n], eps)[0], unit(K[b, :, :n], eps)[0], V[b, :, :n]
        w = weights(log_decay, n)
        at = torch.arange(n, dtype=torch.float64)
        O[b, :, :n] = sc * ((qh @ kh.transpose(1, 2) * w) @ v)
        MO[b, :, :n] = sc.abs() * ((qh.abs() @ kh.abs().transpose(1, 2) * w) @ v.abs())
        end = powers(log_decay, n - 1 - at)[..., None] if n else torch.zeros(H, 0, 1, dtype=torch.float64)
        S[b] = (kh * end).transpose(1, 2) @ v
        MS[b] = (kh * end).abs().transpose(1, 2) @ v.abs()
        if state_in is not None:
            since = powers(log_decay, at + 1)[..., None]
            O[b, :, :n] += sc * since * (qh @ state_in[b])
            MO[b, :, :n] += sc.abs() * since * (qh.abs() @ state_in[b].abs())
            keep = powers(log_decay, torch.tensor(float(n), dtype=torch.float64))[:, None, None]
            S[b] += keep * state_in[b]
            MS[b] += keep * state_in[b].abs()
    return O, S, MO, MS


def backward(Q, K, V, s, log_decay, dO, lens=None, state_in=None, rev_in=None, eps=1e-6):
    """{name: (gradient, M)} of dQ, dK, dV, ds and the reverse-time state `rev`; M of dQ, dK is what the error before the
    chain rule through the norm is measured by, taken through that rule."""
    B, H, N, dk = Q.shape
    dv = V.shape[-1]
    z = lambda *shape: torch.zeros(*shape, dtype=torch.float64)   # noqa: E731
    out = {k: (z(B, H, N, d), z(B, H, N, d)) for k, d in (("dQ", dk), ("dK", dk), ("dV", dv))}
    out["ds"] = (z(B, H), z(B, H))
    out["rev"] = (z(B, H, dk, dv), z(B, H, dk, dv))

    def through(dxh, m, xh, n, clamped, sc):
        t = torch.where(clamped, torch.zeros_like(n), (xh * dxh).sum(-1, keepdim=True))
        mt = torch.where(clamped, torch.zeros_like(n), (xh.abs() * m).sum(-1, keepdim=True))
        return sc * (dxh - xh * t) / n, sc.abs() * (m + xh.abs() * mt) / n

    for b in range(B):
        n = N if lens is None else int(min(max(lens[b], 0), N))
        sc = (s if lens is None else s[b]).double().view(H, 1, 1)
        q, k, v, g = Q[b, :, :n], K[b, :, :n], V[b, :, :n], dO[b, :, :n]
        (qh, qn), (kh, kn) = unit(q, eps), unit(k, eps)
        w = weights(log_decay, n)
        at = torch.arange(n, dtype=torch.float64)

        def grads(qh, kh, v, g, S0, R0):
            a, p = g @ v.transpose(1, 2) * w, qh @ kh.transpose(1, 2) * w
            dq, dk_, dv_ = a @ kh, a.transpose(1, 2) @ qh, p.transpose(1, 2) @ g
            o = p @ v
            rev = (qh * powers(log_decay, at)[..., None]).transpose(1, 2) @ g
            if S0 is not None:
                since = powers(log_decay, at + 1)[..., None]
                dq, o = dq + since * (g @ S0.transpose(1, 2)), o + since * (qh @ S0)
            if R0 is not None:
                until = powers(log_decay, n - at)[..., None]
                dk_, dv_ = dk_ + until * (v @ R0.transpose(1, 2)), dv_ + until * (kh @ R0)
                rev = rev + powers(log_decay, torch.tensor(float(n), dtype=torch.float64))[:, None, None] * R0
            return dq, dk_, dv_, (o * g).sum((1, 2)), rev

        S0 = None if state_in is None else state_in[b]
        R0 = None if rev_in is None else rev_in[b]
        ref = grads(qh, kh, v, g, S0, R0)
        big = grads(qh.abs(), kh.abs(), v.abs(), g.abs(), None if S0 is None else S0.abs(), None if R0 is None else R0.abs())
        for name, i, xh, nn, x in (("dQ", 0, qh, qn, q), ("dK", 1, kh, kn, k)):
            clamped = x.norm(dim=-1, keepdim=True) <= eps
            out[name][0][b, :, :n], out[name][1][b, :, :n] = through(ref[i], big[i], xh, nn, clamped, sc)
        out["dV"][0][b, :, :n], out["dV"][1][b, :, :n] = sc * ref[2], sc.abs() * big[2]
        for name, i in (("ds", 3), ("rev", 4)):
            out[name][0][b], out[name][1][b] = ref[i], big[i]
    if lens is None:
        out["ds"] = tuple(t.sum(0) for t in out["ds"])
    return out


def step(q, k, v, s, log_decay, state, eps=1e-6):
    """One token over `state` [B, H, dk, dv] (the parents'); (o, new state, M_o, M_state)."""
    qh, kh = unit(q, eps)[0], unit(k, eps)[0]
    keep = powers(log_decay, torch.tensor(1.0, dtype=torch.float64)).view(1, -1, 1, 1)
    new = keep * state + kh[..., :, None] * v[..., None, :]
    big = keep * state.abs() + kh.abs()[..., :, None] * v.abs()[..., None, :]
    sc = s.double().view(1, -1, 1)
    return (sc * (qh[..., None, :] @ new)[..., 0, :], new, sc.abs() * (qh.abs()[..., None, :] @ big)[..., 0, :], big)


def paths(parent):
    """For each node of a tree (a list of parents) the nodes from its root to itself."""
    found = []
    for i, p in enumerate(parent):
        found.append((found[p] if 0 <= p < i else []) + [i])
    return found


def tree(q, k, v, s, log_decay, parent, state, eps=1e-6):
    """Outputs token by token along each one's path; (o, M)."""
    B, H, T, _ = q.shape
    o, M = torch.zeros(v.shape, dtype=torch.float64), torch.zeros(v.shape, dtype=torch.float64)
    for b in range(B):
        for i, path in enumerate(paths(parent[b].tolist())):
            S, big = state[b:b + 1], state[b:b + 1].abs()
            for j in path:
                y, S, _, _ = step(q[b:b + 1, :, j], k[b:b + 1, :, j], v[b:b + 1, :, j], s, log_decay, S, eps)
                m, big, _, _ = step(q[b:b + 1, :, j].abs(), k[b:b + 1, :, j].abs(), v[b:b + 1, :, j].abs(), s.abs(), log_decay, big, eps)
            o[b, :, i], M[b, :, i] = y[0], m[0]
    return o, M


def accept(k, v, log_decay, parent, last, state, eps=1e-6):
    new, M = state.clone(), state.abs().clone()
    one = torch.ones(k.shape[1])
    for b in range(k.shape[0]):
        if not 0 <= int(last[b]) < k.shape[2]:
            continue
        for j in paths(parent[b].tolist())[int(last[b])]:
            x = (k[b:b + 1, :, j], k[b:b + 1, :, j], v[b:b + 1, :, j])
            new[b] = step(*x, one, log_decay, new[b:b + 1], eps)[1][0]
            M[b] = step(*(t.abs() for t in x), one, log_decay, M[b:b + 1], eps)[1][0]
    return new, M


def f16_floor(s, values, dk):
    return 2.0 ** -25 * float(s.abs().max()) * (64 * float(values.abs().max()) + dk ** 0.5)


def worst(got, ref, M, u, n, in_fp32=False, floor=0.0):
    """max over the elements of |got - ref| over what it may be; at most 1 is right."""
    got = got.detach().cpu().double()
    may = (2 * u * u + n * 2.0 ** -23) * M if in_fp32 else u * ref.abs() + (u + n * 2.0 ** -23) * M
    # what the element type (fp16) and fp32 have below their smallest normal number
    may = SLACK * may + floor + (2.0 ** -24 if u == 2.0 ** -11 and not in_fp32 else 0.0) + 1e-37
    off = (got - ref).abs()
    assert torch.isfinite(got).all()
    return float((off / may).max()) if off.numel() else 0.0


def norm_error(got, ref):
    got = got.detach().cpu().double()
    n = float(ref.norm())
    return float((got - ref).norm()) / n if n else float(got.norm())
