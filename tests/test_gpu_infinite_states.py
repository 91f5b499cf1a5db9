"""States with infinite elements.  g inf is inf for every g above 0, and a token adds something finite, so such an element stays what
it is, as in the calls without a decay, and the elements beside it are what they are without it.  Outputs read a whole column
of a state: those of its column are infinite, or NaN, and no others are touched.  What a state is multiplied by over many rows is
one fp32 number, g^n; where that is 0 an infinite element is NaN."""
import math

import pytest
import torch

import decay_reference as ref
from test_gpu_decode_decay import cuda, draw, random_tree

pytestmark = pytest.mark.gpu

INF = float("inf")
# none given, nothing forgotten, hardly anything (1 - g), and more than half (g itself)
DECAYS = [None, 0.0, -1e-4, -1.0]
AT = {(0, 0, 3, 5): INF, (0, 1, 17, 30): -INF, (1, 2, 31, 0): INF, (1, 0, 9, 9): INF, (1, 0, 20, 9): -INF}


@pytest.fixture(scope="module")
def cottn():
    import paper_2409_18747_amd.binding as b
    b.cottn_tune_segments(0)
    yield b
    b.cottn_tune_segments(0)


def planted(S):
    S = S.clone()
    for at, x in AT.items():
        S[at] = x
    return S


def same_but_for(infinite, finite, kept=True):
    """The planted elements are where they were (infinite or NaN, unless `kept`), all others what they are without them, to the
    bit."""
    mask = torch.zeros(infinite.shape, dtype=torch.bool)
    for at, x in AT.items():
        assert float(infinite[at]) == x or not (kept or torch.isfinite(infinite[at])), at
        mask[at] = True
    a, b = infinite.cpu(), finite.cpu()
    assert torch.equal(a[~mask], b[~mask])


def columns_apart(o, o_finite):
    """Outputs [B, H, .., dv]: columns of planted elements are not finite, the others the same."""
    mask = torch.zeros(o.shape, dtype=torch.bool)
    for b, h, _, c in AT:
        mask[b, h, ..., c] = True
    o, o_finite = o.cpu(), o_finite.cpu()
    assert not torch.isfinite(o[mask].float()).any()
    assert torch.equal(o[~mask], o_finite[~mask])


def decay(ld, H):
    return None if ld is None else torch.full((H,), ld, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("ld", DECAYS)
@pytest.mark.parametrize("B", [2, 46])
def test_step(cottn, dtype, ld, B):
    x = draw(B, 3, None, 64, 128, dtype, 1)   # 46 x 3: whole columns to a workgroup
    d = cuda(x)
    a, b = planted(d["S"]), d["S"].clone()
    oa = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], decay(ld, 3), a)
    ob = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], decay(ld, 3), b)
    same_but_for(a, b)
    columns_apart(oa, ob)
    if ld is None:
        c = planted(d["S"])
        oc = cottn.cottn_step_dkdv(d["q"], d["k"], d["v"], d["s"], c)
        for at, y in AT.items():
            assert float(c[at]) == y
        assert torch.equal(torch.isnan(oa), torch.isnan(oc)) and torch.equal(oa[torch.isinf(oa)], oc[torch.isinf(oc)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ld", DECAYS)
@pytest.mark.parametrize("B", [2, 46])
def test_accept(cottn, dtype, ld, B):
    T = 9
    x, parent = draw(B, 3, T, 64, 128, dtype, 2), random_tree(B, T, 3).cuda()
    d, last = cuda(x), torch.full((B,), T - 1, dtype=torch.int32).cuda()
    a, b = planted(d["S"]), d["S"].clone()
    for S in (a, b):
        cottn.cottn_tree_accept(d["k"], d["v"], S, parent, last, log_decay=decay(ld, 3))
    same_but_for(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("ld", DECAYS[1:] + [-0.05])
@pytest.mark.parametrize("dk,dv,segments", [(64, 64, 1), (64, 64, 3), (128, 128, 0), (32, 64, 2), (64, 128, 0)])
def test_rows(cottn, dtype, ld, dk, dv, segments):
    """A prompt from such a state, and a backward from such a reverse-time one, over whole chunks and a part of one."""
    B, H, N = 2, 3, 200
    g = torch.Generator().manual_seed(4)
    Q, K, V, dO = (torch.randn(B, H, N, d, generator=g).to(ref.TYPES[dtype]).cuda() for d in (dk, dk, dv, dv))
    S = torch.randn(B, H, dk, dv, generator=g).cuda()
    s, ld = torch.ones(H, device="cuda"), torch.full((H,), ld, device="cuda")
    cottn.cottn_tune_segments(segments)
    try:
        fwd, bwd = [], []
        for S0 in (planted(S), S):
            state, rev = torch.empty_like(S), torch.empty_like(S)
            O = cottn.cottn_fwd_causal_decay(Q, K, V, s, ld, state_in=S0, state=state)
            dQ, dK, dV, ds = cottn.cottn_bwd_causal_decay(Q, K, V, s, ld, dO, rev_state_in=S0, rev_state_out=rev)
            fwd.append((state, O))
            bwd.append((rev, dQ, dV))
    finally:
        cottn.cottn_tune_segments(0)
    kept = math.exp(float(ld[0]) * N) > 2.0 ** -126
    same_but_for(fwd[0][0], fwd[1][0], kept)
    same_but_for(bwd[0][0], bwd[1][0], kept)
    columns_apart(fwd[0][1], fwd[1][1])
    assert torch.equal(bwd[0][1], bwd[1][1])   # dQ does not see what comes behind
    columns_apart(bwd[0][2], bwd[1][2])
