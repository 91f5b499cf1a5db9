"""GPU parity of the single-token step with a decay and beams, and of trees of drafted tokens, against 64 bits."""
import itertools

import pytest
import torch

import decay_reference as ref
from decay_reference import TYPES, U, norm_error, worst

pytestmark = pytest.mark.gpu

WIDTHS = list(itertools.product((32, 64, 128), repeat=2))


@pytest.fixture(scope="module")
def cottn():
    import paper_2409_18747_amd.binding as b
    yield b


def draw(B, H, T, dk, dv, dtype, seed, B_in=None):
    """T None: single tokens."""
    g = torch.Generator().manual_seed(seed)
    shape = (B, H) if T is None else (B, H, T)
    x = {k: torch.randn(*shape, d, generator=g).to(TYPES[dtype]) for k, d in (("q", dk), ("k", dk), ("v", dv))}
    x["s"] = torch.rand(H, generator=g) + 0.5
    x["ld"] = -torch.exp(torch.linspace(-6.0, 1.0, H))
    x["S"] = torch.randn(B_in or B, H, dk, dv, generator=g)
    return x


def random_tree(B, T, seed):
    g = torch.Generator().manual_seed(seed)
    p = torch.arange(T) - torch.randint(1, 5, (B, T), generator=g)
    p = p.clamp(min=-1).to(torch.int32)
    p[:, 0] = -1
    return p


def cuda(x):
    return {k: v.cuda() for k, v in x.items()}


def none_or(ld):
    return torch.zeros(16) if ld is None else ld


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", WIDTHS)
@pytest.mark.parametrize("B", [1, 7])
def test_step_in_place(cottn, dtype, dk, dv, B):
    x = draw(B, 5, None, dk, dv, dtype, dk + dv + B)
    d = cuda(x)
    state, S = d["S"].clone(), x["S"].double()
    for t in range(3):
        o = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], d["ld"], state)
        want, S, M, MS = ref.step(x["q"].double(), x["k"].double(), x["v"].double(), x["s"], x["ld"], S)
        assert worst(o, want, M, U[dtype], dk + 40) <= 1.0
        # the state is fp32 arithmetic throughout
        assert worst(state, S, MS, U["f32"], 3 * (dk + 20), in_fp32=True) <= 1.0
        S = state.cpu().double()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (32, 64), (64, 32)])
def test_step_beams(cottn, dtype, dk, dv):
    """Parents twice, in another order, outside: below, above, and far."""
    B_in, parent = 4, [2, 2, 0, 3, 3, 3, -1, 4, 1, 2 ** 31 - 1, -2 ** 31, 0]
    B = len(parent)
    x = draw(B, 3, None, dk, dv, dtype, 3, B_in=B_in)
    d = cuda(x)
    state = torch.full((B, 3, dk, dv), float("nan"), device="cuda")
    o = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], d["ld"], state, state_in=d["S"],
                               parent=torch.tensor(parent, dtype=torch.int32).cuda())
    zero = torch.zeros(3, dk, dv, dtype=torch.float64)
    S = torch.stack([x["S"][p].double() if 0 <= p < B_in else zero for p in parent])
    want, S, M, MS = ref.step(x["q"].double(), x["k"].double(), x["v"].double(), x["s"], x["ld"], S)
    assert worst(o, want, M, U[dtype], dk + 40) <= 1.0
    assert worst(state, S, MS, U["f32"], dk + 20, in_fp32=True) <= 1.0
    assert torch.equal(d["S"].cpu(), x["S"])


def test_step_from_another_buffer_and_without_decay(cottn):
    x = draw(3, 4, None, 64, 64, "bf16", 4)
    d = cuda(x)
    a, b, c = d["S"].clone(), torch.empty_like(d["S"]), d["S"].clone()
    oa = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], None, a)
    ob = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], torch.zeros(4).cuda(), b, state_in=d["S"])
    oc = cottn.cottn_step(d["q"], d["k"], d["v"], d["s"], c)
    assert torch.equal(a, b) and torch.equal(oa, ob)
    assert norm_error(a, c.cpu().double()) < 1e-6 and norm_error(oa, oc.cpu().double()) < U["bf16"]


@pytest.mark.parametrize("ld", [0.0, float("-inf"), -50.0, 3.0])
def test_step_decays(cottn, ld):
    x = draw(2, 2, None, 32, 32, "f32", 5)
    x["ld"] = torch.tensor([ld, -0.1])
    d = cuda(x)
    o = cottn.cottn_step_decay(d["q"], d["k"], d["v"], d["s"], d["ld"], d["S"])
    want, S, M, MS = ref.step(x["q"].double(), x["k"].double(), x["v"].double(), x["s"], x["ld"], x["S"].double())
    assert worst(o, want, M, U["f32"], 72) <= 1.0 and worst(d["S"], S, MS, U["f32"], 52, in_fp32=True) <= 1.0


def hardly_forgetting():
    """A log_decay near -2e-4 whose exp lies far from every fp32 number."""
    ld = (-2e-4 * (1 + torch.arange(4096) * 2.0 ** -12)).float()
    g = torch.exp(ld.double())
    return ld[torch.argmax(torch.abs(g.float().double() - g))]


def test_many_steps_hardly_forget(cottn):
    """2000 calls without a key: what is left of a state is g^2000.  A factor rounded to fp32 would be off by nearly 2^-25 with
    the same sign in each, 6e-5 in all; roundings of the products (2^-24 at most, of either sign) stay within four times
    sqrt(2000) of them, 1.1e-5, and accepting 500 paths of four tokens within half of that."""
    ld, S = hardly_forgetting(), torch.randn(2, 1, 64, 64, generator=torch.Generator().manual_seed(8))
    zero = torch.zeros(2, 1, 64).cuda()
    state, accepted, one, d_ld = S.cuda(), S.cuda(), torch.ones(1).cuda(), ld[None].cuda()
    parent, last = torch.tensor([[-1, 0, 1, 2]] * 2, dtype=torch.int32).cuda(), torch.full((2,), 3, dtype=torch.int32).cuda()
    drafts = torch.zeros(2, 1, 4, 64).cuda()
    for t in range(2000):
        cottn.cottn_step_decay(zero, zero, zero, one, d_ld, state)
        if t % 4 == 0:
            cottn.cottn_tree_accept(drafts, drafts, accepted, parent, last, log_decay=d_ld)
    want = S.double() * torch.exp(2000 * ld.double())
    assert norm_error(state, want) <= 1.1e-5 and norm_error(accepted, want) <= 0.6e-5


def test_rejected_drafts_are_not_read(cottn):
    """Tokens off the accepted path may hold anything."""
    x, parent = draw(2, 3, 6, 64, 128, "bf16", 12), torch.tensor([[-1, 0, 0, 2, 1, 3]] * 2, dtype=torch.int32)
    last = torch.tensor([5, 4], dtype=torch.int32)   # by 0 2 3 and by 0 1
    y = dict(x, k=x["k"].clone(), v=x["v"].clone())
    for b, off in enumerate(([1, 4], [2, 3, 5])):
        y["k"][b, :, off] = float("nan")
        y["v"][b, :, off] = float("inf")
    states = []
    for z in (x, y):
        d = cuda(z)
        states.append(cottn.cottn_tree_accept(d["k"], d["v"], d["S"], parent.cuda(), last.cuda(), log_decay=d["ld"]))
    assert torch.equal(*states) and torch.isfinite(states[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", WIDTHS)
@pytest.mark.parametrize("T", [1, 13, 32, 64])
def test_tree(cottn, dtype, dk, dv, T):
    x, parent = draw(2, 3, T, dk, dv, dtype, T + dk), random_tree(2, T, T)
    d = cuda(x)
    o = torch.full_like(d["v"], float("nan"))
    cottn.cottn_tree(d["q"], d["k"], d["v"], d["s"], d["S"], parent.cuda(), log_decay=d["ld"], o=o)
    want, M = ref.tree(x["q"].double(), x["k"].double(), x["v"].double(), x["s"], x["ld"], parent, x["S"].double())
    assert worst(o, want, M, U[dtype], T + dk + 40) <= 1.0
    assert norm_error(o, want) <= 0.8 * U[dtype] + 2e-6   # two roundings of 0.43 u (see test_gpu_decay)
    assert torch.equal(d["S"].cpu(), x["S"])


@pytest.mark.parametrize("T", [2, 16, 17, 33, 48, 49, 63])
@pytest.mark.parametrize("kind", ["chain", "star", "roots", "odd"])
def test_tree_shapes(cottn, T, kind):
    """A chain, all on the first, all roots, and parents that are none (themselves, later ones, far outside)."""
    x = draw(2, 2, T, 64, 64, "bf16", T)
    parent = {"chain": torch.arange(-1, T - 1), "star": torch.zeros(T, dtype=torch.long), "roots": torch.full((T,), -1),
              "odd": torch.tensor([(i, T + 5, 2 ** 31 - 1, -2 ** 31, i + 1, i - 1, i // 2)[i % 7] for i in range(T)])}[kind]
    parent = parent.to(torch.int32).repeat(2, 1)
    parent[1] = random_tree(1, T, T)[0]
    d = cuda(x)
    for ld in (d["ld"], None):
        o = cottn.cottn_tree(d["q"], d["k"], d["v"], d["s"], d["S"], parent.cuda(), log_decay=ld)
        want, M = ref.tree(x["q"].double(), x["k"].double(), x["v"].double(), x["s"], x["ld"] if ld is not None else torch.zeros(2),
                           parent, x["S"].double())
        assert worst(o, want, M, U["bf16"], T + 104) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", WIDTHS)
def test_accept(cottn, dtype, dk, dv):
    """Nothing accepted, the first, the last, outside."""
    T, last = 40, [-1, 0, 39, 17, 40, 2 ** 31 - 1, 25]
    B = len(last)
    x, parent = draw(B, 3, T, dk, dv, dtype, dk + dv), random_tree(B, T, 6)
    parent[2] = torch.arange(-1, T - 1)   # a path of 40
    d = cuda(x)
    S = d["S"].clone()
    got = cottn.cottn_tree_accept(d["k"], d["v"], S, parent.cuda(), torch.tensor(last, dtype=torch.int32).cuda(), log_decay=d["ld"])
    assert got is S
    want, M = ref.accept(x["k"].double(), x["v"].double(), x["ld"], parent, last, x["S"].double())
    assert worst(S, want, M, U["f32"], 3 * T + dk, in_fp32=True) <= 1.0
    for b in (0, 4, 5):
        assert torch.equal(S[b].cpu(), x["S"][b])


def test_together(cottn):
    """A prompt, a tree over its state, what was accepted of it, and a token more: as if all had been fed one by one."""
    B, H, N, T, d = 2, 4, 150, 11, 64
    x = draw(B, H, N + T + 1, d, d, "bf16", 7)
    g = cuda(x)
    rows = lambda k, lo, hi: g[k][:, :, lo:hi].contiguous()   # noqa: E731
    state = torch.empty(B, H, d, d, device="cuda")
    cottn.cottn_fwd_causal_decay(*(rows(k, 0, N) for k in "qkv"), g["s"], g["ld"], state=state)
    parent = torch.tensor([[-1, 0, 0, 1, 1, 2, 3, 3, 6, -1, 9]] * B, dtype=torch.int32).cuda()
    drafts = [rows(k, N, N + T) for k in "qkv"]
    o = cottn.cottn_tree(*drafts, g["s"], state, parent, log_decay=g["ld"])
    last = torch.tensor([8, 10], dtype=torch.int32).cuda()
    cottn.cottn_tree_accept(drafts[1], drafts[2], state, parent, last, log_decay=g["ld"])
    end = cottn.cottn_step_decay(*(g[k][:, :, -1].contiguous() for k in "qkv"), g["s"], g["ld"], state)
    for b, path in enumerate([[0, 1, 3, 6, 8], [9, 10]]):
        at = list(range(N)) + [N + j for j in path] + [N + T]
        q, k, v = (x[n][b:b + 1, :, at].double() for n in "qkv")
        O, S, MO, MS = ref.forward(q, k, v, x["s"], x["ld"])
        assert worst(o[b, :, path], O[0, :, N:-1], MO[0, :, N:-1], U["bf16"], N + 200) <= 1.0
        assert worst(end[b], O[0, :, -1], MO[0, :, -1], U["bf16"], N + 200) <= 1.0
        assert worst(state[b], S[0], MS[0], U["bf16"], N + 200, in_fp32=True) <= 1.0


def test_captured(cottn):
    """A step between two buffers, a tree and its acceptance in one graph, replayed with eager work between."""
    B, H, T, d = 3, 4, 9, 64
    x = cuda(draw(B, H, T, d, d, "bf16", 8))
    S, S2, o, o1 = x["S"].clone(), torch.empty_like(x["S"]), torch.empty_like(x["v"]), torch.empty(B, H, d, device="cuda", dtype=torch.bfloat16)
    one = [x[k][:, :, 0].contiguous() for k in "qkv"]
    parent, last = random_tree(B, T, 9).cuda(), torch.tensor([3, -1, 8], dtype=torch.int32).cuda()
    beams = torch.tensor([2, 0, 2], dtype=torch.int32).cuda()

    def call():
        cottn.cottn_step_decay(*one, x["s"], x["ld"], S2, state_in=S, parent=beams, o=o1)
        cottn.cottn_tree(x["q"], x["k"], x["v"], x["s"], S2, parent, log_decay=x["ld"], o=o)
        cottn.cottn_tree_accept(x["k"], x["v"], S2, parent, last, log_decay=x["ld"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        S.normal_()
        call()
        torch.cuda.synchronize()
        want = [t.clone() for t in (S2, o, o1)]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((S2, o, o1), want):
            assert torch.equal(a, b)
