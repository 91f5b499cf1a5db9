"""Rows whose squares add up to less than fp32's least normal number are normalised all the same, by the calls by the gated delta
rule as by the others."""
import pytest
import torch

import delta_reference as ref
from delta_reference import TYPES, check
from test_gpu_delta import cottn, cuda, double, draw   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 64), (128, 64)])
def test_sums_of_squares_below_the_normal_numbers(cottn, dtype, dk, dv):   # noqa: F811
    """Some 2^-65 long: the squares add up to 2^-130, which has steps of 2^-149, so that the sum is off by 2^-20 of itself and half a
    step for each of dk squares, sqrt(dk) 2^-20 with random signs, and the norm by half of that."""
    x, more = draw(1, 2, 90, dk, dv, dtype, dk)
    short = {"Q": (4, 70), "K": (9, 33)}
    for name, rows in short.items():
        x[name][:, :, rows] = (x[name][:, :, rows].double() * (2.0 ** -65 / dk ** 0.5)).to(x[name].dtype)
    off = (1 + dk ** 0.5) * 2.0 ** -21
    want_O, want_S = ref.forward(**double(x), eps=1e-25)
    want = ref.gradients(**double(x), dO=more["dO"].double(), eps=1e-25)
    d, m = cuda(x), cuda(more)
    state = torch.empty_like(m["state_in"])
    O = cottn.cottn_fwd_causal_delta(**d, state=state, eps=1e-25)
    got = cottn.cottn_bwd_causal_delta(**d, dO=m["dO"], eps=1e-25)
    check("O", O, want_O, dtype, more=off)
    check("state", state, want_S, None, more=off)
    for name, t in zip(("dQ", "dK"), got):
        far = torch.zeros(90, dtype=torch.bool)
        far[list(short[name[1]])] = True
        check(name, t[:, :, far], want[name][:, :, far], dtype, more=2 * off)
        check(name, t[:, :, ~far], want[name][:, :, ~far], dtype, more=off)
    check("dV", got[2], want["dV"], dtype, more=off)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_prompt_normalises_as_a_token_does(cottn, dtype):   # noqa: F811
    """Rows of one feature, whose normalised feature is 1 or -1: with unit values the state of one token is that, off by the rounding of
    the square (half of 2^-24 in the norm), of the reciprocal root (a unit, 2 of 2^-24, or a square root and a division) and of the
    products (parts of three bfloat16, 2^-24, and two roundings)."""
    B, H, d = 64, 8, 32
    g = torch.Generator().manual_seed(2)
    K = torch.zeros(B, H, 1, d)
    a = torch.rand(B, H, generator=g) * 3.0 + 0.5
    K[:, :, 0, 7] = a
    K = K.to(TYPES[dtype]).cuda()
    V, s, gate = torch.ones_like(K), torch.ones(H, device="cuda"), torch.ones(B, H, 1, device="cuda")
    state = torch.empty(B, H, d, d, device="cuda")
    cottn.cottn_fwd_causal_delta(K, K, V, s, None, gate, state=state)
    after = torch.zeros_like(state)
    k, v = K[:, :, 0].contiguous(), V[:, :, 0].contiguous()
    cottn.cottn_step_delta(k, k, v, s, None, gate[:, :, 0].contiguous(), after)
    want = torch.zeros_like(state)
    want[:, :, 7] = 1.0
    for t in (state, after):
        assert float((t - want).abs().max()) <= 5.5 * 2.0 ** -24
