"""Thousands of (sequence, head) pairs with a decay: some of them against 64 bits, ds of all against the sum over calls of parts."""
import pytest
import torch

import decay_reference as ref
from decay_reference import TYPES, U, worst

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cottn():
    import paper_2409_18747_amd.binding as b
    b.cottn_tune_segments(0)
    yield b


@pytest.mark.parametrize("dtype,B,H,N,dk,dv", [("bf16", 300, 41, 70, 32, 32), ("bf16", 101, 33, 130, 128, 128), ("f16", 700, 7, 33, 64, 128),
                                               ("f32", 130, 17, 65, 64, 64), ("bf16", 5000, 3, 1, 64, 64), ("f32", 63, 21, 40, 128, 128)])
@pytest.mark.parametrize("padded", [False, True])
def test_some_of_many(cottn, dtype, B, H, N, dk, dv, padded):
    g = torch.Generator(device="cuda").manual_seed(B)
    Q, K, V, dO = (torch.randn(B, H, N, d, generator=g, device="cuda").to(TYPES[dtype]) for d in (dk, dk, dv, dv))
    S = torch.randn(B, H, dk, dv, generator=g, device="cuda")
    ld = -torch.exp(torch.linspace(-7.0, 0.0, H))
    s = torch.rand((B, H) if padded else (H,), generator=g, device="cuda") + 0.5
    lens = torch.randint(0, N + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if padded else None
    state = torch.empty_like(S)
    O = cottn.cottn_fwd_causal_decay(Q, K, V, s, ld.cuda(), seq_len=lens, state_in=S, state=state)
    dQ, dK, dV, ds = cottn.cottn_bwd_causal_decay(Q, K, V, s, ld.cuda(), dO, seq_len=lens, state_in=S)
    at = [0, 1, B // 3, B - 2, B - 1]
    f = [t[at].cpu().double() for t in (Q, K, V, dO, S)]
    n_at = None if lens is None else lens[at].tolist()
    sc = s[at].cpu() if padded else s.cpu()
    O64, S64, M, MS = ref.forward(*f[:3], sc, ld, n_at, f[4])
    want = ref.backward(*f[:3], sc, ld, f[3], n_at, f[4])
    n, u = N + max(dk, dv) + 40, U[dtype]
    floors = [ref.f16_floor(sc, t, dk) if dtype == "f16" else 0.0 for t in (f[2], f[3])]
    assert worst(O[at], O64, M, u, n, floor=floors[0]) <= 1.0 and worst(state[at], S64, MS, u, n, in_fp32=True) <= 1.0
    for got, name, floor in ((dQ, "dQ", 0.0), (dK, "dK", 0.0), (dV, "dV", floors[1])):
        assert worst(got[at], *want[name], u, n, floor=floor) <= 1.0, name
    if padded:
        assert worst(ds[at], *want["ds"], u, n + N + dk, in_fp32=True) <= 1.0
        return
    # each part adds up B / 4 heads' sums in fp32: of B terms at most a rounding each, relative to what they add up to in the mean
    parts = [cottn.cottn_bwd_causal_decay(Q[i::4].contiguous(), K[i::4].contiguous(), V[i::4].contiguous(), s, ld.cuda(), dO[i::4].contiguous(),
                                          state_in=S[i::4].contiguous())[3].double() for i in range(4)]
    ones = torch.ones(B, H, device="cuda")
    terms = cottn.cottn_bwd_causal_decay(Q, K, V, ones, ld.cuda(), dO, seq_len=torch.full((B,), N, dtype=torch.int32, device="cuda"),
                                         state_in=S)[3].double()
    assert ((ds.double() - sum(parts)).abs() <= B * 2.0 ** -23 * terms.abs().sum(0)).all()
    assert ((ds.double() - terms.sum(0)).abs() <= B * 2.0 ** -23 * terms.abs().sum(0)).all()
