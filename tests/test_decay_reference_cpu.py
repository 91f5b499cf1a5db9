"""The 64-bit reference of the decay tests: against the recurrence, differences, and autograd through the definition."""
import torch

import decay_reference as ref


def draw(B, H, N, dk, dv, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)   # noqa: E731
    return r(B, H, N, dk), r(B, H, N, dk), r(B, H, N, dv), r(B, H, N, dv), r(B, H, dk, dv), r(B, H, dk, dv)


LD = torch.tensor([-0.3, 0.0, -2.0])
S = torch.tensor([0.7, 1.3, 1.0])


def test_forward_is_the_recurrence():
    Q, K, V, _, S0, _ = draw(2, 3, 9, 4, 5, 1)
    O, state, _, _ = ref.forward(Q, K, V, S, LD, state_in=S0)
    H = S0
    for i in range(9):
        o, H, _, _ = ref.step(Q[:, :, i], K[:, :, i], V[:, :, i], S, LD, H)
        assert torch.allclose(o, O[:, :, i], rtol=1e-12, atol=1e-12)
    assert torch.allclose(H, state, rtol=1e-12, atol=1e-12)


def test_lengths_and_nothing_kept():
    Q, K, V, _, S0, _ = draw(2, 3, 6, 4, 4, 2)
    ld = torch.tensor([float("-inf"), -0.1, 1.0])   # above 0 counts as 0
    s = S.repeat(2, 1)
    O, state, _, _ = ref.forward(Q, K, V, s, ld, lens=[4, 0], state_in=S0)
    assert torch.equal(O[0, :, 4:], torch.zeros(3, 2, 4, dtype=torch.float64)) and not O[1].any()
    assert torch.equal(state[1], S0[1])
    short = ref.forward(Q[:1, :, :4], K[:1, :, :4], V[:1, :, :4], S, torch.tensor([float("-inf"), -0.1, 0.0]), state_in=S0[:1])
    assert torch.allclose(O[:1, :, :4], short[0]) and torch.allclose(state[:1], short[1])
    kh, qh = ref.unit(K, 1e-6)[0], ref.unit(Q, 1e-6)[0]
    assert torch.allclose(O[0, 0, 2], S[0] * (qh[0, 0, 2] @ kh[0, 0, 2]) * V[0, 0, 2])
    assert torch.allclose(state[0, 0], torch.outer(kh[0, 0, 3], V[0, 0, 3]))


def test_gradients_against_differences():
    Q, K, V, G, S0, R0 = draw(2, 3, 7, 4, 5, 3)
    Q[0, 1, 2] *= 1e-9   # a row below eps
    got = ref.backward(Q, K, V, S, LD, G, state_in=S0, rev_in=R0, eps=1e-6)

    def loss(Q, K, V, S):
        # R0 is the gradient that rows behind put on the state: s g <R0, H> for the rows before
        O, H, _, _ = ref.forward(Q, K, V, S, LD, state_in=S0, eps=1e-6)
        return (O * G).sum() + (S.double().view(-1, 1, 1) * torch.exp(LD.double()).view(-1, 1, 1) * R0 * H).sum()

    h = 1e-6
    gen = torch.Generator().manual_seed(4)
    for name, x in (("dQ", Q), ("dK", K), ("dV", V)):
        for _ in range(6):
            d = torch.randn(x.shape, generator=gen, dtype=torch.float64)
            if name == "dQ":
                d[0, 1, 2] = 0.0   # 1e-9 is not to be left by a step of 1e-6
            args = {"dQ": Q, "dK": K, "dV": V}
            up, down = dict(args), dict(args)
            up[name], down[name] = x + h * d, x - h * d
            diff = (loss(*up.values(), S) - loss(*down.values(), S)) / (2 * h)
            assert abs(float(diff - (got[name][0] * d).sum())) < 1e-6 * (1 + abs(float(diff)))
    # the row below eps is q / eps: linear
    e = torch.zeros_like(Q)
    e[0, 1, 2, 0] = 1e-9
    diff = (loss(Q + e, K, V, S) - loss(Q - e, K, V, S)) / 2e-9
    assert abs(float(diff) - float(got["dQ"][0][0, 1, 2, 0])) < 1e-5 * abs(float(diff))
    O1 = ref.forward(Q, K, V, torch.ones(3), LD, state_in=S0)[0]
    assert torch.allclose(got["ds"][0], (O1 * G).sum((0, 2, 3)))


def test_reverse_state_carries_pieces():
    Q, K, V, G, S0, R0 = draw(1, 3, 10, 4, 5, 5)
    whole = ref.backward(Q, K, V, S, LD, G, state_in=S0, rev_in=R0)
    mid = ref.forward(Q[:, :, :6], K[:, :, :6], V[:, :, :6], S, LD, state_in=S0)[1]
    tail = ref.backward(Q[:, :, 6:], K[:, :, 6:], V[:, :, 6:], S, LD, G[:, :, 6:], state_in=mid, rev_in=R0)
    head = ref.backward(Q[:, :, :6], K[:, :, :6], V[:, :, :6], S, LD, G[:, :, :6], state_in=S0, rev_in=tail["rev"][0])
    for name in ("dQ", "dK", "dV"):
        assert torch.allclose(whole[name][0], torch.cat([head[name][0], tail[name][0]], 2))
    assert torch.allclose(whole["ds"][0], head["ds"][0] + tail["ds"][0])
    assert torch.allclose(whole["rev"][0], head["rev"][0])


def test_a_chain_is_a_sequence_and_accepting_it_its_state():
    Q, K, V, _, S0, _ = draw(2, 3, 8, 4, 5, 6)
    O, state, _, _ = ref.forward(Q, K, V, S, LD, state_in=S0)
    chain = torch.arange(-1, 7, dtype=torch.int32).repeat(2, 1)
    o, _ = ref.tree(Q, K, V, S, LD, chain, S0)
    assert torch.allclose(o, O)
    new, _ = ref.accept(K, V, LD, chain, torch.tensor([7, -1]), S0)
    assert torch.allclose(new[0], state[0]) and torch.equal(new[1], S0[1])
