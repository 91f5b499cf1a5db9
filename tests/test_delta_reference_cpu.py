"""The 64-bit reference of the gated delta rule: against the matrix form, closed forms and differences; that of rotary positions."""
import math

import torch

import delta_reference as ref


def draw(B, H, N, dk, dv, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)   # noqa: E731
    return dict(Q=r(B, H, N, dk), K=r(B, H, N, dk), V=r(B, H, N, dv), s=r(H).abs() + 0.5, log_decay=-r(B, H, N).abs(),
                beta=torch.sigmoid(r(B, H, N))), r(B, H, N, dv), r(B, H, dk, dv), r(B, H, dk, dv)


def test_forward_is_the_matrix_recurrence():
    x, _, S0, _ = draw(2, 3, 7, 4, 5)
    O, state = ref.forward(**x, state_in=S0)
    S = S0.clone()
    for t in range(7):
        k = ref.unit(x["K"])[:, :, t, :, None]
        g, b = torch.exp(x["log_decay"])[:, :, t, None, None], x["beta"][:, :, t, None, None]
        S = g * ((torch.eye(4) - b * k @ k.transpose(-1, -2)) @ S) + b * k @ x["V"][:, :, t, None]
        o = x["s"].view(1, 3, 1, 1) * ref.unit(x["Q"])[:, :, t, None] @ S
        assert torch.allclose(o[:, :, 0], O[:, :, t], rtol=1e-12, atol=1e-12)
    assert torch.allclose(S, state, rtol=1e-12, atol=1e-12)


def test_a_key_that_comes_again_is_replaced():
    """beta 1 and no decay: what is read back at a key is the value that came with it last."""
    x, _, _, _ = draw(1, 1, 4, 8, 3)
    x["K"][:, :, 3] = 2.5 * x["K"][:, :, 1]
    x["Q"][:, :, 3] = 0.3 * x["K"][:, :, 1]
    x["beta"].fill_(1.0)
    x["log_decay"].zero_()
    O, _ = ref.forward(**x)
    assert torch.allclose(O[:, :, 3], x["s"] * x["V"][:, :, 3])


def test_gradients_are_differences():
    x, dO, S0, dS = draw(2, 2, 5, 3, 4, seed=1)
    g = ref.gradients(**x, dO=dO, state_in=S0, dstate=dS)

    def loss(x, S0):
        O, state = ref.forward(**x, state_in=S0)
        return float((O * dO).sum() + (state * dS).sum())

    h = 1e-6
    for name in ("Q", "K", "V", "s", "log_decay", "beta", "state_in"):
        base = S0 if name == "state_in" else x[name]
        flat = g["d" + name].reshape(-1)
        for i in range(0, base.numel(), max(1, base.numel() // 7)):
            both = []
            for sign in (h, -h):
                t = base.clone()
                t.view(-1)[i] += sign
                both.append(loss(x, t) if name == "state_in" else loss({**x, name: t}, S0))
            assert abs((both[0] - both[1]) / (2 * h) - float(flat[i])) <= 1e-6 * max(1.0, float(flat.abs().max()))


def test_lengths():
    x, dO, S0, dS = draw(3, 2, 6, 4, 4, seed=2)
    x["s"] = x["s"].repeat(3, 1) * torch.tensor([[1.0], [2.0], [3.0]])
    O, state = ref.forward(**x, lens=[4, 0, 6], state_in=S0)
    short = {k: v[:1, :, :4] if v.dim() > 2 else v[:1] for k, v in x.items()}
    O1, state1 = ref.forward(**short, lens=[4], state_in=S0[:1])
    assert torch.allclose(O[:1, :, :4], O1) and torch.allclose(state[:1], state1) and torch.equal(state[1], S0[1])
    assert not O[0, :, 4:].any() and not O[1].any()
    g = ref.gradients(**x, dO=dO, lens=[4, 0, 6], state_in=S0, dstate=dS)
    assert not g["dK"][0, :, 4:].any() and not g["dbeta"][1].any() and torch.equal(g["dstate_in"][1], dS[1])


def test_rotary():
    X = torch.randn(1, 2, 3, 8, dtype=torch.float64)
    at = torch.tensor([[[0, 3], [1, -2], [100000, 7]]], dtype=torch.int32)
    freq, axis = torch.tensor([1.0, 0.25, 0.5]), torch.tensor([0, 1, 5])
    for neighbours in (False, True):
        Y = ref.rotary(X, at, freq, axis, neighbours)
        a, b = (2, 3) if neighbours else (1, 4)
        z = torch.complex(X[0, 0, 1, a], X[0, 0, 1, b]) * complex(math.cos(-0.5), math.sin(-0.5))
        assert abs(complex(Y[0, 0, 1, a], Y[0, 0, 1, b]) - complex(z)) < 1e-12
        assert torch.equal(Y[..., 6:], X[..., 6:])                       # behind the pairs
        a, b = (4, 5) if neighbours else (2, 5)
        assert torch.equal(Y[..., a], X[..., a]) and torch.equal(Y[..., b], X[..., b])   # an axis that there is not
        assert torch.allclose(ref.rotary(Y, at, freq, axis, neighbours, inverse=True), X)
        assert torch.allclose(Y.norm(dim=-1), X.norm(dim=-1))
