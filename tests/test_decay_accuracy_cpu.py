"""The bounds on states and ds that are returned in fp32 (decay_accuracy) against the chunked form with its weighted operands in one,
two and three parts and 64 bits otherwise: three bfloat16 parts and two of fp16 lie well within them, one part fewer well
outside."""
import pytest
import torch

import decay_accuracy as acc
import decay_reference as ref

CHUNK = 64


def in_parts(x, parts, dtype):
    """x as a sum of `parts` numbers of the element type, each the rest rounded; fp16 ones in units of 2^-14, so that the
    rests are normal numbers.  None: x."""
    if parts is None:
        return x
    scale = 2.0 ** 14 if dtype == "f16" else 1.0
    out = torch.zeros_like(x)
    for _ in range(parts):
        out = out + (scale * x - out).to(ref.TYPES[dtype]).double()
    return out / scale


def chunked(x, log_decay, parts, dtype):
    """(state, reverse-time state, ds [B, H]) chunk by chunk."""
    B, H, N, dk = x["Q"].shape
    qh, kh = ref.unit(x["Q"].double(), 1e-6)[0], ref.unit(x["K"].double(), 1e-6)[0]
    v, g = x["V"].double(), x["dO"].double()
    S, R = (torch.zeros(B, H, dk, v.shape[-1], dtype=torch.float64) for _ in range(2))
    ds = torch.zeros(B, H, dtype=torch.float64)
    for b in range(0, N, CHUNK):
        e = min(N, b + CHUNK)
        at = torch.arange(e - b, dtype=torch.float64)
        once, whole = (ref.powers(log_decay, torch.tensor(float(i), dtype=torch.float64))[:, None, None] for i in (1, e - b))
        G = in_parts(qh[:, :, b:e] * ref.powers(log_decay, at)[..., None], parts, dtype).transpose(-1, -2) @ g[:, :, b:e]
        K = in_parts(kh[:, :, b:e] * ref.powers(log_decay, e - b - 1 - at)[..., None], parts, dtype)
        p = qh[:, :, b:e] @ kh[:, :, b:e].transpose(-1, -2) * ref.weights(log_decay, e - b)
        ds += (once * S * G).sum((2, 3)) + ((p @ v[:, :, b:e]) * g[:, :, b:e]).sum((2, 3))
        R += ref.powers(log_decay, torch.tensor(float(b), dtype=torch.float64))[:, None, None] * G
        S = whole * S + K.transpose(-1, -2) @ v[:, :, b:e]
    return S, R, ds


@pytest.mark.parametrize("dtype,enough", [("bf16", 3), ("f16", 2)])
@pytest.mark.parametrize("N,dk,dv", [(130, 64, 64), (260, 128, 128), (260, 32, 128), (130, 128, 32)])
def test_bounds_tell_the_parts_apart(dtype, enough, N, dk, dv):
    B, H = 3, 6
    g = torch.Generator().manual_seed(N + dk)
    x = {k: torch.randn(B, H, N, d, generator=g).to(ref.TYPES[dtype]) for k, d in (("Q", dk), ("K", dk), ("V", dv), ("dO", dv))}
    ld = -torch.exp(torch.linspace(-9.0, -3.0, H))
    S, R, ds = chunked(x, ld, None, dtype)
    f = {k: t.double() for k, t in x.items()}
    want = ref.backward(f["Q"], f["K"], f["V"], torch.ones(B, H), ld, f["dO"], lens=[N] * B)
    assert torch.allclose(ds, want["ds"][0], rtol=1e-9, atol=1e-9) and torch.allclose(R, want["rev"][0], rtol=1e-9, atol=1e-9)
    terms = acc.ds_terms(x, ld)
    for parts in (enough - 1, enough):
        s, r, d = chunked(x, ld, parts, dtype)
        found = [acc.state_error(s, S) / acc.state_bound(N), acc.state_error(r, R) / acc.state_bound(N),
                 acc.ds_error(d, ds, terms) / acc.ds_bound(N, dk, dv, CHUNK)]
        print(parts, found)
        assert all(e < 0.5 for e in found) if parts == enough else all(e > 1.3 for e in found)
