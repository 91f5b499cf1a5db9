"""GPU parity of the single-token step by the gated delta rule, and of rotary positions, against 64 bits; both in one run."""
import itertools

import pytest
import torch

import delta_reference as ref
from delta_reference import TYPES, U, check

pytestmark = pytest.mark.gpu
WIDTHS = list(itertools.product((32, 64, 128), repeat=2))


@pytest.fixture(scope="module")
def cottn():
    import paper_2409_18747_amd.binding as b
    yield b


def draw(B, H, dk, dv, dtype, seed, B_in=None):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    x = {"q": r(B, H, dk), "k": r(B, H, dk), "v": r(B, H, dv)}
    x = {k: v.to(TYPES[dtype]) for k, v in x.items()}
    return {**x, "s": r(H).abs() + 0.5, "log_decay": -r(B, H).abs(), "beta": torch.sigmoid(r(B, H))}, r(B_in or B, H, dk, dv)


def token(x, S):
    o, S = ref.token(*(x[k].double() for k in ("q", "k", "v", "log_decay", "beta")), S)
    return x["s"].double()[:, None] * o, S


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", WIDTHS)
@pytest.mark.parametrize("B", [1, 40])
def test_step_in_place(cottn, dtype, dk, dv, B):
    x, S = draw(B, 5, dk, dv, dtype, dk + dv + B)
    d, state, S = {k: v.cuda() for k, v in x.items()}, S.cuda(), S.double()
    for _ in range(3):
        o = cottn.cottn_step_delta(**d, state=state)
        want, S = token(x, S)
        check("o", o, want, dtype)
        check("state", state, S, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_beams(cottn, dtype):
    x, S = draw(6, 4, 64, 128, dtype, 3, B_in=4)
    parent = torch.tensor([2, 2, 0, -1, 3, 4], dtype=torch.int32)
    start = torch.stack([S[p] if 0 <= p < 4 else torch.zeros_like(S[0]) for p in parent.tolist()]).double()
    want, after = token(x, start)
    d, state = {k: v.cuda() for k, v in x.items()}, torch.empty(6, 4, 64, 128, device="cuda")
    from_ = S.cuda()
    o = cottn.cottn_step_delta(**d, state=state, state_in=from_, parent=parent.cuda())
    check("o", o, want, dtype)
    check("state", state, after, None)
    assert torch.equal(from_.cpu(), S)


def test_no_decay_and_nothing_kept(cottn):
    x, S = draw(2, 3, 32, 32, "f32", 4)
    d = {k: v.cuda() for k, v in x.items()}
    for ld, kept in ((None, 0.0), (torch.full((2, 3), -float("inf")), -500.0), (torch.full((2, 3), 3.0), 0.0)):
        state = S.cuda()
        o = cottn.cottn_step_delta(**{**d, "log_decay": None if ld is None else ld.cuda()}, state=state)
        want, after = token({**x, "log_decay": torch.full((2, 3), kept)}, S.double())
        check("o", o, want, "f32")
        check("state", state, after, None)


def turn_check(got, want, X, dtype):
    """A turned feature is the sum of two products with a sine and a cosine, off by a few 2^-24 of each, rounded once."""
    M = X.double().abs().amax(-1, keepdim=True) * 1.5
    off = (got.double().cpu() - want).abs()
    assert bool((off <= U[dtype] * want.abs() + 8 * 2.0 ** -24 * M).all()), float(off.max())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,pairs", [(32, 16), (32, 1), (64, 32), (64, 8), (64, 15), (128, 64), (128, 37), (128, 24)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rotary(cottn, dtype, d, pairs, neighbours):
    g = torch.Generator().manual_seed(d + pairs)
    B, H, N, axes = 2, 3, 37, 3
    X, Y = (torch.randn(B, H, N, d, generator=g).to(TYPES[dtype]) for _ in range(2))
    at = torch.randint(-2 ** 31, 2 ** 31, (B, N, axes), generator=g).to(torch.int32)
    at[:, ::2] %= 1000
    freq = (1e4 ** (-torch.arange(pairs) / pairs)).float()
    axis = torch.randint(-1, axes + 1, (pairs,), generator=g).to(torch.int32)
    for inverse in (False, True):
        Qr, Kr = cottn.cottn_rotary(X.cuda(), Y.cuda(), at.cuda(), freq.cuda(), axis=axis.cuda(), neighbours=neighbours, inverse=inverse)
        for got, t in ((Qr, X), (Kr, Y)):
            want = ref.rotary(t.double(), at, freq, axis, neighbours, inverse)
            turn_check(got, want, t, dtype)
            assert torch.equal(got[..., 2 * pairs:].cpu(), t[..., 2 * pairs:])


@pytest.mark.parametrize("B,H,N", [(1, 1, 1), (64, 16, 1), (1, 5, 1000), (3, 2, 4097)])
def test_rotary_shapes_in_place_and_alone(cottn, B, H, N):
    X = torch.randn(B, H, N, 64, device="cuda").to(torch.bfloat16)
    at = torch.randint(0, 1 << 20, (B, N), device="cuda").to(torch.int32)
    freq = (1e4 ** (-torch.arange(32, device="cuda") / 32)).float()
    Qr, none = cottn.cottn_rotary(X, None, at, freq)
    assert none is None
    turn_check(Qr, ref.rotary(X.cpu().double(), at[..., None].cpu(), freq.cpu()), X.cpu(), "bf16")
    Y, Z = X.clone(), X.clone()
    got = cottn.cottn_rotary(Y, Z, at, freq, Qr=Y, Kr=Z)
    assert got[0] is Y and torch.equal(Y, Qr) and torch.equal(Z, Qr)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_with_positions_then_tokens(cottn, dtype):
    """What a model does: turn the prompt's rows, take them in, then one token after the other from the prompt's state; against
    the whole sequence in one call, and against 64 bits."""
    g = torch.Generator().manual_seed(6)
    B, H, N, more, dk, dv = 2, 3, 90, 5, 64, 32
    T = N + more
    r = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    Q, K, V = (r(B, H, T, d).to(TYPES[dtype]).cuda() for d in (dk, dk, dv))
    s, ld, beta = (r(H).abs() + 0.5).cuda(), (-r(B, H, T).abs() / 8).cuda(), torch.sigmoid(r(B, H, T)).cuda()
    at = (torch.arange(T, dtype=torch.int32) + 70000).expand(B, T).contiguous().cuda()
    freq = (1e4 ** (-torch.arange(dk // 2) / (dk // 2))).float().cuda()
    Qr, Kr = cottn.cottn_rotary(Q, K, at, freq)
    whole = cottn.cottn_fwd_causal_delta(Qr, Kr, V, s, ld, beta)
    cut = lambda t, a, b: t[:, :, a:b].contiguous()   # noqa: E731
    state = torch.empty(B, H, dk, dv, device="cuda")
    q, k = cottn.cottn_rotary(cut(Q, 0, N), cut(K, 0, N), at[:, :N].contiguous(), freq)
    O = [cottn.cottn_fwd_causal_delta(q, k, cut(V, 0, N), s, cut(ld, 0, N), cut(beta, 0, N), state=state)]
    for t in range(N, T):
        q, k = cottn.cottn_rotary(cut(Q, t, t + 1), cut(K, t, t + 1), at[:, t:t + 1].contiguous(), freq)
        O.append(cottn.cottn_step_delta(q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), V[:, :, t].contiguous(), s,
                                        ld[:, :, t].contiguous(), beta[:, :, t].contiguous(), state)[:, :, None])
    want, _ = ref.forward(*(t.double().cpu() for t in (Qr, Kr, V, s, ld, beta)))
    check("in pieces", torch.cat(O, 2), want, dtype)
    check("whole", whole, want, dtype, two_parts=True)
