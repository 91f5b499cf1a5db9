"""Plain 64-bit implementations of the gated delta rule, token by token, and of rotary positions, from their definitions, and how
far a kernel may be from them.

Bounds.  u is half a step of the element type (finfo.eps / 2, relative).  A result in 16 bits is rounded once; what it is rounded
from, and every result in fp32, has met fp32 roundings alone (2^-24 each), or where the call asks for no fp32 result operands in
two bfloat16 parts, off by 2^-15 of a product at most.
  Norms.  A uniformly spread rounding is u / sqrt(3) in the root mean square at most: 0.58 u.  A token meets a chain of four
sums a chunk of at most 192 terms, 768 roundings whose signs are as good as random, sqrt(768) = 28 of 2^-24, handed on through
contractions: five chunks, the longest sequences here, add up to sqrt(5) times that, 63 2^-24 = 3.8e-6 of the result's norm; and
products in two parts 2^-14.
  Elements.  The same with all signs alike, 5 x 768 of 2^-24 = 2^-12, of the largest value of the sequence and head; in two parts
2^-14 sqrt(192) more, 2^-10.
  ds is the sum of a token's dO . o / s over all tokens, each off by as much of itself: by as much of the root of the sum of their
squares (ds_terms), which the sum itself may be far below.
"""
import torch

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def unit(x, eps=1e-6):
    """Rows over max(norm, eps)."""
    n2 = (x * x).sum(-1, keepdim=True)
    long = n2 > eps * eps
    return torch.where(long, x / torch.sqrt(torch.where(long, n2, torch.ones_like(n2))), x / eps)


def token(q, k, v, log_decay, beta, S, eps=1e-6):
    """(o / s, the state behind the token); q, k [B, H, dk], v [B, H, dv], gates [B, H], S [B, H, dk, dv], all float64."""
    kh = unit(k, eps)
    S = torch.exp(log_decay.clamp(max=0.0))[..., None, None] * S
    e = v - (kh[..., None] * S).sum(-2)
    S = S + (beta[..., None] * kh)[..., None] * e[..., None, :]
    return (unit(q, eps)[..., None] * S).sum(-2), S


def forward(Q, K, V, s, log_decay, beta, lens=None, state_in=None, eps=1e-6):
    """float64 in; (O, state).  s [H], or [B, H] with lens."""
    B, H, N, dk = Q.shape
    S = torch.zeros(B, H, dk, V.shape[-1], dtype=torch.float64) if state_in is None else state_in
    n = torch.full((B,), N) if lens is None else torch.as_tensor(lens).clamp(0, N)
    there = torch.arange(N) < n[:, None]
    out = []
    for t in range(N):
        here = there[:, t].view(B, 1, 1)
        row = lambda x: torch.where(here, x[:, :, t], torch.zeros_like(x[:, :, t]))   # noqa: E731
        gate = lambda x: torch.where(here[..., 0], x[:, :, t], torch.zeros_like(x[:, :, t]))   # noqa: E731
        o, S = token(row(Q), row(K), row(V), gate(log_decay), gate(beta), S, eps)
        out.append(torch.where(here, o, torch.zeros_like(o)))
    O = torch.stack(out, 2) if N else torch.zeros(B, H, 0, V.shape[-1], dtype=torch.float64)
    return s.view(-1, H, 1, 1) * O, S


def gradients(Q, K, V, s, log_decay, beta, dO, lens=None, state_in=None, dstate=None, eps=1e-6):
    """By autograd through the recurrence: {"dQ", .., "dstate_in"}."""
    x = [t.detach().clone().requires_grad_(True) for t in (Q, K, V, s, log_decay, beta)]
    S = state_in if state_in is not None else torch.zeros(Q.shape[0], Q.shape[1], Q.shape[3], V.shape[3], dtype=torch.float64)
    S = S.detach().clone().requires_grad_(True)
    O, state = forward(*x, lens=lens, state_in=S, eps=eps)
    there = torch.ones(dO.shape[0], 1, dO.shape[2], 1, dtype=torch.bool)
    if lens is not None:
        there = (torch.arange(dO.shape[2]) < torch.as_tensor(lens)[:, None]).view(-1, 1, dO.shape[2], 1)
    loss = (O * torch.where(there, dO, torch.zeros_like(dO))).sum()
    if dstate is not None:
        loss = loss + (state * dstate).sum()
    got = torch.autograd.grad(loss, x + [S], allow_unused=True)
    names = ("dQ", "dK", "dV", "ds", "dlog_decay", "dbeta", "dstate_in")
    return {n: torch.zeros_like(t) if g is None else g for n, t, g in zip(names, x + [S], got)}


def ds_terms(O, dO, s, lens=None):
    """The root of the sum of the squares of what ds adds up, [H], or with lens [B, H]."""
    there = torch.ones(dO.shape[:3], dtype=torch.bool)
    if lens is not None:
        there = (torch.arange(dO.shape[2]) < torch.as_tensor(lens)[:, None])[:, None].expand(dO.shape[:3])
    t = torch.where(there, (O * dO.double()).sum(-1) / s.double().view(-1, O.shape[1], 1), torch.zeros(1, dtype=torch.float64))
    return torch.sqrt((t * t).sum((0, 2) if lens is None else 2))


def check(name, got, want, dtype, two_parts=False, more=0.0, terms=None):
    """got: a result in fp32 or in `dtype`; want: float64, [B, H, ..] or [H]; more: added to either bound, relative; terms: what
    the result's own magnitude is replaced by where that is less."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, name
    assert bool(torch.isfinite(got).all()), name
    u = U["f32"] if dtype is None else U[dtype]
    size = want.abs() if terms is None else torch.maximum(want.abs(), terms)
    norm, off = float(size.norm()), float((got - want).norm())
    if norm == 0.0:
        assert off == 0.0, name
        return
    rel = 0.58 * u + 63 * U["f32"] + (2.0 ** -14 if two_parts else 0.0) + more
    assert off <= rel * norm, "%s: norm error %.3g of %.3g" % (name, off / norm, rel)
    most = want.abs().flatten(2).amax(2).view(want.shape[:2] + (1,) * (want.dim() - 2)) if want.dim() > 2 else size.max()
    bound = u * want.abs() + (2.0 ** -12 + (2.0 ** -10 if two_parts else 0.0) + more) * most
    worst = float(((got - want).abs() / torch.where(bound > 0, bound, torch.full_like(bound, 1e-300))).max())
    assert worst <= 1.0, "%s: %.3g of the bound" % (name, worst)


def rotary(X, positions, freq, axis=None, neighbours=False, inverse=False):
    """float64 X [B, H, N, d], positions [B, N, axes]."""
    p = len(freq)
    a, b = (2 * torch.arange(p), 2 * torch.arange(p) + 1) if neighbours else (torch.arange(p), torch.arange(p) + p)
    Y = X.clone()
    for j in range(p):
        ax = 0 if axis is None else int(axis[j])
        if not 0 <= ax < positions.shape[2]:
            continue
        phi = (positions[:, None, :, ax].double() * float(freq[j])) * (-1.0 if inverse else 1.0)
        u, v = X[..., a[j]], X[..., b[j]]
        Y[..., a[j]] = u * torch.cos(phi) - v * torch.sin(phi)
        Y[..., b[j]] = v * torch.cos(phi) + u * torch.sin(phi)
    return Y
