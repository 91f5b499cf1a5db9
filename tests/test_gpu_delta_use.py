"""The calls by the gated delta rule and of rotary positions as programs use them: states replaced in place, captured in graphs,
on a stream of their own, at sizes drawn over the whole range, long, many, and beyond 32-bit offsets."""
import random

import pytest
import torch

import delta_reference as ref
from delta_reference import check
from test_gpu_delta import cuda, double, draw, run_both, run_both_padded, train_workspace

pytestmark = pytest.mark.gpu


@pytest.fixture
def cottn():
    import paper_2409_18747_amd.binding as b
    yield b
    b.cottn_tune_segments(0)


@pytest.mark.parametrize("G", [1, 2, 4])
@pytest.mark.parametrize("dk,dv,dtype", [(32, 32, "bf16"), (64, 128, "bf16"), (128, 64, "bf16"), (128, 64, "f32")])
def test_states_in_place(cottn, G, dk, dv, dtype):
    """state for state_in and dstate_in for dstate: the same results as apart, also where the segments' workgroups are more than
    the chip has room for, so that the last one of a sequence can be done before the first begins."""
    cottn.cottn_tune_segments(G)
    B, H, N = 24, 16, 200
    x, more = draw(B, H, N, dk, dv, dtype, G, per_unit=True)
    d, m = cuda(x), cuda(more)
    lens = torch.randint(0, N + 1, (B,), generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    ws = train_workspace(cottn, d)
    state, dstate_in = torch.empty_like(m["state_in"]), torch.empty_like(m["state_in"])
    O = cottn.cottn_fwd_causal_delta(**d, seq_len=lens, state_in=m["state_in"], state=state, workspace=ws)
    both = dict(dO=m["dO"], seq_len=lens, state_in=m["state_in"])
    apart = cottn.cottn_bwd_causal_delta(**d, **both, dstate=m["dstate"], dstate_in=dstate_in, fwd_workspace=ws)
    S, D = m["state_in"].clone(), m["dstate"].clone()
    assert torch.equal(cottn.cottn_fwd_causal_delta(**d, seq_len=lens, state_in=S, state=S, workspace=ws), O)
    assert torch.equal(S, state)
    got = cottn.cottn_bwd_causal_delta(**d, **both, dstate=D, dstate_in=D, fwd_workspace=ws)
    assert torch.equal(D, dstate_in)
    for a, b in zip(apart, got):
        assert torch.equal(a, b)


def test_a_backward_by_itself_is_that_after_a_forward(cottn):
    for G, dtype in ((1, "bf16"), (3, "bf16"), (3, "f32")):
        cottn.cottn_tune_segments(G)
        x, more = draw(2, 3, 270, 64, 64, dtype, 5)
        d, m, _, _, got = run_both(cottn, x, more, dtype)
        D = torch.empty_like(m["dstate"])
        alone = cottn.cottn_bwd_causal_delta(**d, dO=m["dO"], state_in=m["state_in"], dstate=m["dstate"], dstate_in=D)
        for a, b in zip(got, alone):
            assert torch.equal(a, b)


@pytest.mark.parametrize("G", [1, 3])
def test_in_graphs(cottn, G):
    """A training step in two graphs that share the forward's workspace, and a token with its rotation in a third: every replay
    gives what the calls give, for the inputs of the time."""
    cottn.cottn_tune_segments(G)
    B, H, N, dk, dv = 2, 3, 200, 64, 32
    x, more = draw(B, H, N, dk, dv, "bf16", 7)
    d, m = cuda(x), cuda(more)
    ws = train_workspace(cottn, d)
    at = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, N).contiguous()
    freq = (1e4 ** (-torch.arange(dk // 2, device="cuda") / (dk // 2))).float()
    S = m["state_in"].clone()

    def forward():
        q, k = cottn.cottn_rotary(d["Q"], d["K"], at, freq)
        return cottn.cottn_fwd_causal_delta(**{**d, "Q": q, "K": k}, state_in=m["state_in"], workspace=ws)

    def backward():
        q, k = cottn.cottn_rotary(d["Q"], d["K"], at, freq)
        got = cottn.cottn_bwd_causal_delta(**{**d, "Q": q, "K": k}, dO=m["dO"], state_in=m["state_in"], dstate=m["dstate"], fwd_workspace=ws)
        return cottn.cottn_rotary(got[0], got[1], at, freq, inverse=True) + got[2:]

    first = lambda t: t[:, :, 0].contiguous()   # noqa: E731

    def step():
        q, k = cottn.cottn_rotary(d["Q"][:, :, :1].contiguous(), d["K"][:, :, :1].contiguous(), at[:, 5:6].contiguous(), freq)
        return cottn.cottn_step_delta(first(q), first(k), first(d["V"]), d["s"], first(d["log_decay"]), first(d["beta"]), S)

    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for f in (forward, backward, step):   # (loads the kernels)
            f()
        side.synchronize()
        for f in (forward, backward, step):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = f()
            graphs.append((graph, out if isinstance(out, tuple) else (out,)))
    torch.cuda.synchronize()
    for turn in range(4):
        for t in (d["Q"], d["V"], m["dO"], d["beta"]):   # other inputs, by eager work between the replays
            t.mul_(0.9)
        S.copy_(m["state_in"])
        want = [(forward(),), backward(), (step(),)]
        want_S = S.clone()
        S.copy_(m["state_in"])
        torch.cuda.synchronize()
        ws.zero_()
        for graph, out in graphs:
            for t in out:
                t.zero_()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, out), w in zip(graphs, want):
            for a, b in zip(out, w):
                assert torch.equal(a, b), turn
        assert torch.equal(S, want_S), turn


def test_on_another_stream(cottn):
    """On the stream that is given, and on the current one: the same."""
    x, more = draw(2, 3, 200, 64, 64, "bf16", 8)
    d, m = cuda(x), cuda(more)
    at, freq = torch.arange(200, dtype=torch.int32, device="cuda").expand(2, 200).contiguous(), torch.ones(32, device="cuda")
    token = {n: d[n][:, :, 3].contiguous() for n in ("Q", "K", "V", "log_decay", "beta")}

    def all_of_it(S, ws, **on):
        q, k = cottn.cottn_rotary(d["Q"], d["K"], at, freq, **on)
        O = cottn.cottn_fwd_causal_delta(**{**d, "Q": q, "K": k}, state_in=S, state=S, workspace=ws, **on)
        got = cottn.cottn_bwd_causal_delta(**{**d, "Q": q, "K": k}, dO=m["dO"], fwd_workspace=ws, **on)
        o = cottn.cottn_step_delta(token["Q"], token["K"], token["V"], d["s"], token["log_decay"], token["beta"], S, **on)
        return (q, k, O, o, S) + got

    want = all_of_it(m["state_in"].clone(), train_workspace(cottn, d))
    S, ws, side = m["state_in"].clone(), train_workspace(cottn, d), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = all_of_it(S, ws, stream=side)
    side.synchronize()
    with torch.cuda.stream(side):
        S = m["state_in"].clone()
        current = all_of_it(S, ws)
    side.synchronize()
    for a, b, c in zip(want, got, current):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("seed", range(24))
def test_drawn_sizes(cottn, seed):
    """Of the ranges that the bounds of delta_reference were derived for."""
    rng = random.Random(seed)
    B, H, N = rng.randint(1, 5), rng.randint(1, 9), int(320 ** rng.random())
    dk, dv, dtype = rng.choice([32, 64, 128]), rng.choice([32, 64, 128]), rng.choice(["bf16", "bf16", "f16", "f32"])
    cottn.cottn_tune_segments(rng.choice([0, 0, 1, 2, 5]))
    padded, states = rng.random() < 0.4, rng.random() < 0.5
    print(seed, B, H, N, dk, dv, dtype, padded, states, flush=True)
    x, more = draw(B, H, N, dk, dv, dtype, seed, per_unit=padded)
    if padded:
        run_both_padded(cottn, x, more, dtype, [rng.randint(0, N) for _ in range(B)])
    else:
        run_both(cottn, x, more, dtype, states=states)


@pytest.mark.parametrize("dtype,dk,G", [("bf16", 64, 0), ("bf16", 64, 1), ("f32", 64, 0), ("f32", 128, 0)])
def test_a_long_sequence(cottn, dtype, dk, G):
    """64 chunks, forward and back again: 768 roundings a chunk and walk, whose signs are as good as random, sqrt(2 x 64 x 768) =
    313 of 2^-24 on top of what the shorter ones are given."""
    cottn.cottn_tune_segments(G)
    x, more = draw(1, 2, 4096, dk, 32, dtype, 9)
    run_both(cottn, x, more, dtype, off=313 * 2.0 ** -24)


def test_many_sequences(cottn):
    """More workgroups than a chip takes at once, of one chunk and of a few rows."""
    x, more = draw(700, 5, 3, 32, 32, "bf16", 10)
    run_both(cottn, x, more, "bf16")
    x, more = draw(300, 3, 70, 32, 64, "f16", 11)
    run_both(cottn, x, more, "f16")


def test_rows_beyond_32_bits(cottn):
    """Rows, states and errors whose places in a tensor pass 2^31: of each of two heads the last rows, which strong decays have
    let forget what was before, against the same rows alone."""
    B, H, N, dk, dv, tail = 1, 2, (1 << 23) + 70, 128, 64, 200
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    g = torch.Generator(device="cuda").manual_seed(12)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16)   # noqa: E731
    x = {"Q": r(B, H, N, dk), "K": r(B, H, N, dk), "V": r(B, H, N, dv)}
    assert x["Q"].numel() > 1 << 31
    x["s"] = torch.ones(H, device="cuda")
    x["log_decay"] = torch.full((B, H, N), -1.0, device="cuda")
    x["beta"] = torch.full((B, H, N), 0.5, device="cuda")
    dO = r(B, H, N, dv)
    ws = train_workspace(cottn, x)
    state = torch.empty(B, H, dk, dv, device="cuda")
    O = cottn.cottn_fwd_causal_delta(**x, state=state, workspace=ws)
    got = cottn.cottn_bwd_causal_delta(**x, dO=dO, fwd_workspace=ws)
    torch.cuda.synchronize()
    cut = {k: (v if k == "s" else v[:, :, -tail:].contiguous().cpu()) for k, v in x.items()}
    cut["s"] = cut["s"].cpu()
    want_O, want_S = ref.forward(**double(cut))
    want = ref.gradients(**double(cut), dO=dO[:, :, -tail:].cpu().double())
    known = slice(100, None)   # what was before the tail is e^-100 of itself by then
    check("O", O[:, :, -tail:][:, :, known], want_O[:, :, known], "bf16")
    check("state", state, want_S, None)
    for name, t in zip(("dQ", "dK", "dV"), got):
        check(name, t[:, :, -tail:][:, :, known], want[name][:, :, known], "bf16")
    for name, t in (("dlog_decay", got[4]), ("dbeta", got[5])):
        check(name, t[:, :, -tail:][:, :, known, None], want[name][:, :, known, None], None)


def test_states_beyond_32_bits(cottn):
    """A step of so many sequences that the last one's state is behind 2^31 elements, and rotary rows as far out."""
    B, H, d = 4500, 32, 128
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    g = torch.Generator(device="cuda").manual_seed(13)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    state = r(B, H, d, d)
    assert state.numel() > 1 << 31
    q, k, v = (r(B, H, d).to(torch.bfloat16) for _ in range(3))
    s, ld, beta = torch.ones(H, device="cuda"), -r(B, H).abs(), torch.sigmoid(r(B, H))
    before = state[-1:].cpu().double()
    o = cottn.cottn_step_delta(q, k, v, s, ld, beta, state)
    want, after = ref.token(*(t[-1:].cpu().double() for t in (q, k, v, ld, beta)), before)
    check("o", o[-1:], want, "bf16")
    check("state", state[-1:], after, None)
    del state
    N = (1 << 19) + 3
    X = r(1, 33, N, d).to(torch.bfloat16)
    assert X.numel() > 1 << 31
    at, freq = torch.arange(N, dtype=torch.int32, device="cuda")[None], (1e4 ** (-torch.arange(64, device="cuda") / 64)).float()
    Y, _ = cottn.cottn_rotary(X, None, at, freq, Qr=X.clone())
    assert torch.equal(Y[:, -1:, -64:], cottn.cottn_rotary(X[:, -1:, -64:].contiguous(), None, at[:, -64:].contiguous(), freq)[0])
