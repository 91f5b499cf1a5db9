"""Calls by the gated delta rule where 1 / eps is so large that two of them multiplied, or one times a value, leave fp32: zero rows,
rows that do not exist (which are filled with zeros) and short ones.  A normalised row is 1 long at most all the same; gradients
with respect to rows below eps are those with respect to the normalised ones over eps."""
import pytest
import torch

import delta_reference as ref
from delta_reference import check, ds_terms
from test_gpu_delta import cottn, cuda, double, draw, train_workspace   # noqa: F401
from test_gpu_delta_step import draw as draw_tokens

pytestmark = pytest.mark.gpu

# two factors together beyond fp32; one and a value; 1 / eps itself
EPS = [1e-25, 1e-30, 1e-37, 1e-42]
ZERO_Q, ZERO_K = (3, 40, 70), (3, 17, 64)


def shorten(x, dtype):
    """Zero rows of Q and K, the same one and different ones, and all others times 2^-57 (some 1e-16 long; fp16 has no such)."""
    for name, zero in (("Q", ZERO_Q), ("K", ZERO_K)):
        if dtype != "f16":
            x[name] = (x[name].double() * 2.0 ** -57).to(x[name].dtype)
        x[name][:, :, [i for i in zero if i < x[name].shape[2]]] = 0
    return x


def apart(name, got, want, zero, dtype, eps):
    """The rows below eps, whose gradients are 1 / eps times as large (fp16 has no such, nor fp32 from 1e-37 on), and the others."""
    far = torch.zeros(want.shape[2], dtype=torch.bool)
    far[[i for i in zero if i < want.shape[2]]] = True
    check(name, got[:, :, ~far], want[:, :, ~far], dtype)
    if dtype != "f16" and eps >= 1e-30:
        check(name + " below eps", got[:, :, far], want[:, :, far], dtype)


@pytest.mark.parametrize("eps", EPS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv,G", [(64, 64, 1), (64, 64, 3), (128, 128, 2), (32, 128, 1), (128, 32, 3)])
def test_rows(cottn, dtype, dk, dv, G, eps):   # noqa: F811
    x, more = draw(2, 3, 150, dk, dv, dtype, dk + dv)
    x = shorten(x, dtype)
    S = more["state_in"].double()
    want_O, want_S = ref.forward(**double(x), state_in=S, eps=eps)
    want = ref.gradients(**double(x), dO=more["dO"].double(), state_in=S, dstate=more["dstate"].double(), eps=eps)
    d, m = cuda(x), cuda(more)
    cottn.cottn_tune_segments(G)
    try:
        ws = train_workspace(cottn, d).fill_(255)   # (what is not written first is NaN)
        state, dstate_in = torch.empty_like(m["state_in"]), torch.empty_like(m["state_in"])
        O = cottn.cottn_fwd_causal_delta(**d, state_in=m["state_in"], state=state, workspace=ws, eps=eps)
        dQ, dK, dV, ds, dlog_decay, dbeta = cottn.cottn_bwd_causal_delta(
            **d, dO=m["dO"], state_in=m["state_in"], dstate=m["dstate"], dstate_in=dstate_in, fwd_workspace=ws, eps=eps)
    finally:
        cottn.cottn_tune_segments(0)
    check("O", O, want_O, dtype)
    check("state", state, want_S, None)
    apart("dQ", dQ, want["dQ"], ZERO_Q, dtype, eps)
    apart("dK", dK, want["dK"], ZERO_K, dtype, eps)
    check("dV", dV, want["dV"], dtype)
    check("ds", ds, want["ds"], None, terms=ds_terms(want_O, more["dO"], x["s"]))
    for name, t in (("dlog_decay", dlog_decay), ("dbeta", dbeta), ("dstate_in", dstate_in)):
        check(name, t, want[name], None)


@pytest.mark.parametrize("eps", EPS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_outputs_alone(cottn, dtype, d, eps):   # noqa: F811
    x, _ = draw(2, 3, 150, d, d, dtype, d)
    x = shorten(x, dtype)
    want, _ = ref.forward(**double(x), eps=eps)
    check("O", cottn.cottn_fwd_causal_delta(**cuda(x), eps=eps), want, dtype, two_parts=dtype != "f32")


@pytest.mark.parametrize("eps", EPS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_tokens(cottn, dtype, eps):   # noqa: F811
    x, S = draw_tokens(4, 3, 64, 128, dtype, 3)
    for name, zero in (("q", (0, 1)), ("k", (0, 2))):
        if dtype != "f16":
            x[name] = (x[name].double() * 2.0 ** -57).to(x[name].dtype)
        x[name][list(zero)] = 0
    o, after = ref.token(*(x[k].double() for k in ("q", "k", "v", "log_decay", "beta")), S.double(), eps)
    state = S.cuda()
    got = cottn.cottn_step_delta(**cuda(x), state=state, eps=eps)
    check("o", got, x["s"].double()[:, None] * o, dtype)
    check("state", state, after, None)
    assert not got[:2].any()
