"""Steps, trees and acceptances of many sequences, whose workgroups take whole columns of a state and stream what the caches do not
hold, against 64 bits."""
import pytest
import torch

import decay_reference as ref
from decay_reference import U, norm_error, worst
from test_gpu_decode_decay import cuda, draw, random_tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cottn():
    import paper_2409_18747_amd.binding as b
    yield b


def tree(q, k, v, s, log_decay, parent, state):
    """decay_reference.tree for all sequences at once, each node's state from its parent's; (o, M)."""
    B, H, T, dk = q.shape
    dv = v.shape[-1]
    ones = torch.arange(B)
    S, big = (torch.zeros(B, T + 1, H, dk, dv, dtype=torch.float64) for _ in range(2))
    S[:, T], big[:, T] = state, state.abs()   # the roots' parent
    o, M = torch.zeros(v.shape, dtype=torch.float64), torch.zeros(v.shape, dtype=torch.float64)
    for i in range(T):
        up = parent[:, i].long()
        up = torch.where((up >= 0) & (up < i), up, torch.full_like(up, T))
        o[:, :, i], S[:, i], M[:, :, i], big[:, i] = step(q[:, :, i], k[:, :, i], v[:, :, i], s, log_decay, S[ones, up], big[ones, up])
    return o, M


def step(q, k, v, s, log_decay, state, big):
    o, new, _, _ = ref.step(q, k, v, s, log_decay, state)
    M, new_big, _, _ = ref.step(q.abs(), k.abs(), v.abs(), s.abs(), log_decay, big)
    return o, new, M, new_big


def accept(k, v, log_decay, parent, last, state):
    """decay_reference.accept for all sequences at once; (new state, M)."""
    B, H, T, dk = k.shape
    S, big = state.clone(), state.abs()
    at = [ref.paths(p)[e] if 0 <= e < T else [] for p, e in zip(parent.tolist(), last)]
    one = torch.ones(H)
    for depth in range(max(map(len, at))):
        b = torch.tensor([i for i in range(B) if depth < len(at[i])])
        j = torch.tensor([at[i][depth] for i in b.tolist()])
        _, S[b], _, big[b] = step(k[b, :, j], k[b, :, j], v[b, :, j], one, log_decay, S[b], big[b])
    return S, big


def test_references_agree():
    x, parent = draw(3, 2, 9, 4, 5, "f32", 1), random_tree(3, 9, 1)
    parent[1, 4], parent[1, 6] = 7, 2 ** 31 - 1
    q, k, v, S = (x[n].double() for n in ("q", "k", "v", "S"))
    for mine, theirs in ((tree(q, k, v, x["s"], x["ld"], parent, S), ref.tree(q, k, v, x["s"], x["ld"], parent, S)),
                         (accept(k, v, x["ld"], parent, [8, -1, 5], S), ref.accept(k, v, x["ld"], parent, [8, -1, 5], S))):
        for a, b in zip(mine, theirs):
            assert torch.allclose(a, b, rtol=1e-12, atol=1e-12)


WIDE = [(32, 64), (64, 64), (128, 64), (32, 128), (64, 128), (128, 128), (64, 32)]
# (sequences, heads, widths): from 129 states on whole columns; 515 of 128 x 128 are 34 MB and pass the caches
STATES = [(27, 5, w) for w in WIDE] + [(103, 5, (128, 128))]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,H,widths", STATES)
def test_step(cottn, dtype, B, H, widths):
    x = draw(B, H, None, *widths, dtype, sum(widths))
    d = cuda(x)
    S = x["S"].double()
    want, new, M, MS = ref.step(x["q"].double(), x["k"].double(), x["v"].double(), x["s"], x["ld"], S)
    state = d["S"].clone()
    o = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], d["ld"], state)
    assert worst(o, want, M, U[dtype], widths[0] + 40) <= 1.0
    assert worst(state, new, MS, U["f32"], widths[0] + 20, in_fp32=True) <= 1.0
    # beams: groups of four change places
    parent = torch.randint(0, 4, (B,), generator=torch.Generator().manual_seed(B)) + torch.arange(B) // 4 * 4
    parent[::9] = B   # none
    S = torch.cat([S, torch.zeros_like(S[:1])])[parent.clamp(max=B)]
    want, new, M, MS = ref.step(x["q"].double(), x["k"].double(), x["v"].double(), x["s"], x["ld"], S)
    state.fill_(float("nan"))
    o = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], d["ld"], state, state_in=d["S"], parent=parent.clamp(max=B).to(torch.int32).cuda())
    assert worst(o, want, M, U[dtype], widths[0] + 40) <= 1.0
    assert worst(state, new, MS, U["f32"], widths[0] + 20, in_fp32=True) <= 1.0
    assert torch.equal(d["S"].cpu(), x["S"])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv,T", [(128, 128, T) for T in (1, 13, 16, 17, 32, 33, 48, 64)] + [(64, 64, T) for T in (1, 13, 17, 32, 33, 64)]
                         + [(32, 128, 13), (32, 128, 31), (64, 128, 40), (128, 64, 16), (128, 64, 20), (32, 64, 64), (32, 32, 50)])
def test_tree(cottn, dtype, dk, dv, T):
    B, H = 13, 5   # 65 states: whole columns (fp32 two parts of 64)
    x, parent = draw(B, H, T, dk, dv, dtype, T + dk), random_tree(B, T, T)
    d = cuda(x)
    o = torch.full_like(d["v"], float("nan"))
    cottn.cottn_tree(d["q"], d["k"], d["v"], d["s"], d["S"], parent.cuda(), log_decay=d["ld"], o=o)
    want, M = tree(x["q"].double(), x["k"].double(), x["v"].double(), x["s"], x["ld"], parent, x["S"].double())
    assert worst(o, want, M, U[dtype], T + dk + 40) <= 1.0
    assert norm_error(o, want) <= 0.8 * U[dtype] + 2e-6   # two roundings of 0.43 u (see test_gpu_decay)
    assert torch.equal(d["S"].cpu(), x["S"])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T", [5, 30, 61])
def test_tree_past_the_caches(cottn, dtype, T):
    """515 states of 128 x 128; the first, the last and one between against 64 bits, all against calls of a third each."""
    B, H = 103, 5
    x, parent = draw(B, H, T, 128, 128, dtype, T), random_tree(B, T, T)
    d, p = cuda(x), parent.cuda()
    o = cottn.cottn_tree(d["q"], d["k"], d["v"], d["s"], d["S"], p, log_decay=d["ld"])
    for lo, hi in ((0, 35), (35, 70), (70, 103)):
        part = [d[k][lo:hi].contiguous() for k in ("q", "k", "v")]
        assert torch.equal(o[lo:hi], cottn.cottn_tree(*part, d["s"], d["S"][lo:hi].contiguous(), p[lo:hi].contiguous(), log_decay=d["ld"]))
    at = [0, 51, 102]
    want, M = tree(*(x[k][at].double() for k in ("q", "k", "v")), x["s"], x["ld"], parent[at], x["S"][at].double())
    assert worst(o[at], want, M, U[dtype], T + 168) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,H,widths", STATES)
def test_accept(cottn, dtype, B, H, widths):
    """Paths of up to 40 tokens, none, and ones that are no tokens."""
    T = 40
    x, parent = draw(B, H, T, *widths, dtype, sum(widths) + 1), random_tree(B, T, 6)
    parent[2] = torch.arange(-1, T - 1)
    last = [(i * 7) % T for i in range(B)]
    last[:6] = [-1, 0, 39, 17, 40, 2 ** 31 - 1]
    d = cuda(x)
    S = d["S"].clone()
    cottn.cottn_tree_accept(d["k"], d["v"], S, parent.cuda(), torch.tensor(last, dtype=torch.int32).cuda(), log_decay=d["ld"])
    want, M = accept(x["k"].double(), x["v"].double(), x["ld"], parent, last, x["S"].double())
    assert worst(S, want, M, U["f32"], 3 * T + widths[0], in_fp32=True) <= 1.0
    for b in (0, 4, 5):
        assert torch.equal(S[b].cpu(), x["S"][b])
