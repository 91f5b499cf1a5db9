"""GPU parity of causal attention with a decay per head, forward and backward, against 64 bits (decay_reference)."""
import itertools

import pytest
import torch

import decay_reference as ref
from decay_reference import TYPES, U, norm_error, worst

pytestmark = pytest.mark.gpu

WIDTHS = list(itertools.product((32, 64, 128), repeat=2))
# in 2-norm: an element of a result meets two roundings, of an operand and its own, each at most u and for mantissas of all
# sizes (uniform in 1 .. 2) 0.43 u in the mean square: 0.6 u together
NORM = 0.8


@pytest.fixture(scope="module")
def cottn():
    import paper_2409_18747_amd.binding as b
    b.cottn_tune_segments(0)
    yield b
    b.cottn_tune_segments(0)


def draw(B, H, N, dk, dv, dtype, seed, lens=None, states=False):
    g = torch.Generator().manual_seed(seed)
    x = {k: torch.randn(B, H, N, d, generator=g).to(TYPES[dtype]) for k, d in (("Q", dk), ("K", dk), ("V", dv), ("dO", dv))}
    x["s"] = torch.rand((H,) if lens is None else (B, H), generator=g) + 0.5
    # from keeping everything to forgetting most within a row
    x["log_decay"] = -torch.exp(torch.linspace(-9.0, 1.0, H))
    x["log_decay"][0] = 0.0
    if states:
        x["state_in"], x["rev_in"] = (torch.randn(B, H, dk, dv, generator=g) for _ in range(2))
    return x


def run(cottn, x, lens=None, eps=1e-6, share=True, stream=None):
    d = {k: v.cuda() for k, v in x.items()}
    B, H, N, dk = x["Q"].shape
    dv = x["V"].shape[-1]
    code = {torch.float32: cottn.COTTN_F32, torch.bfloat16: cottn.COTTN_BF16, torch.float16: cottn.COTTN_F16}[x["Q"].dtype]
    n = cottn.cottn_workspace_bytes_dkdv(cottn.OP_FWD_DECAY, B, H, N, dk, dv, 0, code)
    ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")   # what is not written first is NaN
    sl = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
    state, rev = (torch.full((B, H, dk, dv), float("nan"), device="cuda") for _ in range(2))
    O = torch.full_like(d["V"], float("nan"))
    out = {"O": cottn.cottn_fwd_causal_decay(d["Q"], d["K"], d["V"], d["s"], d["log_decay"], seq_len=sl,
                                             state_in=d.get("state_in"), O=O, state=state, workspace=ws[:n] if n else None, eps=eps),
           "state": state}
    m = cottn.cottn_workspace_bytes_dkdv(cottn.OP_BWD_DECAY, B, H, N, dk, dv, 0, code)
    ws2 = torch.full((m,), 0xFF, dtype=torch.uint8, device="cuda")
    grads = [torch.full_like(d[k], float("nan")) for k in ("Q", "K", "V")]
    out["dQ"], out["dK"], out["dV"], out["ds"] = cottn.cottn_bwd_causal_decay(
        d["Q"], d["K"], d["V"], d["s"], d["log_decay"], d["dO"], seq_len=sl, state_in=d.get("state_in"), rev_state_in=d.get("rev_in"),
        dQ=grads[0], dK=grads[1], dV=grads[2], rev_state_out=rev, workspace=ws2, eps=eps,
        fwd_workspace=ws[:n] if share and n else None)
    out["rev"] = rev
    torch.cuda.synchronize()
    return out


def check(out, x, dtype, lens=None, eps=1e-6, norms=True):
    f = {k: v.double() for k, v in x.items()}
    f["s"], f["log_decay"] = x["s"], x["log_decay"]
    O, state, MO, MS = ref.forward(f["Q"], f["K"], f["V"], x["s"], x["log_decay"], lens, f.get("state_in"), eps)
    want = ref.backward(f["Q"], f["K"], f["V"], x["s"], x["log_decay"], f["dO"], lens, f.get("state_in"), f.get("rev_in"), eps)
    want["O"], want["state"] = (O, MO), (state, MS)
    N, d = x["Q"].shape[2], max(x["Q"].shape[3], x["V"].shape[3])
    n, u = N + d + 40, U[dtype]
    found = {}
    for name, (r, M) in want.items():
        fp32 = name in ("state", "ds", "rev")
        terms = n + (x["Q"].shape[0] * N + d if name == "ds" else 0)
        floor = ref.f16_floor(x["s"], x["V" if name == "O" else "dO"], x["Q"].shape[3]) if dtype == "f16" and name in ("O", "dV") else 0.0
        found[name] = (worst(out[name], r, M, u, terms, fp32, floor), norm_error(out[name], r))
    print({k: "%.2g %.2g" % v for k, v in found.items()})
    for name, (most, norm) in found.items():
        assert most <= 1.0, (name, found)
        if norms and name != "ds":
            # (fp32: 2^-24 a rounding, and states' operands in two parts u^2 each)
            fp32 = name in ("state", "rev")
            assert norm <= (2 * u * u + 2e-6 if fp32 else NORM * u + 2e-6), (name, found)
    for name in ("O", "dQ", "dK", "dV"):
        if lens is not None:
            for b, n_b in enumerate(lens):
                assert not out[name][b, :, max(0, n_b):].any(), name


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", WIDTHS)
def test_widths(cottn, dtype, dk, dv):
    x = draw(2, 3, 200, dk, dv, dtype, 10 + dk + dv, states=True)
    cottn.cottn_tune_segments(0)
    check(run(cottn, x), x, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 777])
def test_lengths(cottn, dtype, N):
    x = draw(1, 4, N, 64, 64, dtype, N)
    check(run(cottn, x), x, dtype)


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 64, 64), ("f16", 128, 128), ("f32", 32, 64)])
@pytest.mark.parametrize("segments", [1, 2, 3, 5, 40])
@pytest.mark.parametrize("share", [True, False])
def test_segments(cottn, dtype, dk, dv, segments, share):
    """Any split gives the result, with the states handed on or formed again (40: carried)."""
    x = draw(2, 3, 1337, dk, dv, dtype, segments, states=True)
    cottn.cottn_tune_segments(segments)
    try:
        out = run(cottn, x, share=share)
    finally:
        cottn.cottn_tune_segments(0)
    check(out, x, dtype)


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 64, 64), ("f16", 64, 128), ("f32", 64, 64), ("bf16", 128, 128)])
@pytest.mark.parametrize("segments", [0, 1, 4, 30])
def test_padded(cottn, dtype, dk, dv, segments):
    """Lengths of zero, one, the ends of chunks and segments, beyond N and below zero."""
    lens = [0, 1, 63, 64, 65, 256, 257, 511, 700, 900, -3, 128]
    x = draw(len(lens), 2, 700, dk, dv, dtype, 5, lens=lens, states=True)
    cottn.cottn_tune_segments(segments)
    try:
        out = run(cottn, x, lens=lens)
    finally:
        cottn.cottn_tune_segments(0)
    check(out, x, dtype, lens=[min(700, max(0, n)) for n in lens])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("ld", [[0.0, float("-inf")], [-100.0, -20.0], [-5.0, -1e-7], [-1e30, -3e38], [0.5, float("inf")]])
def test_decays(cottn, dtype, ld):
    x = draw(2, 2, 260, 64, 64, dtype, 7, states=True)
    x["log_decay"] = torch.tensor(ld)
    check(run(cottn, x), x, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv,tuned", [(64, 64, 0), (128, 128, 2), (32, 128, 1)])
def test_short_and_long_rows(cottn, dtype, dk, dv, tuned):
    """Zero rows, rows below eps, rows whose 1 / norm is beyond fp16, and large ones, next to ordinary ones."""
    x = draw(1, 3, 150, dk, dv, dtype, 8)
    tiny = 2e-6 if dtype == "f16" else 1e-9
    for name, at in (("Q", 3), ("K", 4)):
        x[name][:, :, at] = 0
        x[name][:, :, at + 10] *= tiny / 16
        x[name][:, :, at + 20] *= 1e-3
        x[name][:, :, at + 30] *= 1e3
        x[name][:, :, at + 70] *= tiny
    x["V"][:, :, 60:70] = 0
    # dQ of a row of norm 1e-9 .. 1e-3 is 1e3 .. 1e6 (eps) times an ordinary one: beyond fp16, whose rows are scaled down
    if dtype == "f16":
        x["dO"] *= 2.0 ** -9
    cottn.cottn_tune_segments(tuned)
    try:
        out = run(cottn, x, eps=1e-3 if dtype == "f16" else 1e-6)
    finally:
        cottn.cottn_tune_segments(0)
    check(out, x, dtype, eps=1e-3 if dtype == "f16" else 1e-6, norms=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,H,N,dk,dv", [(1, 5, 100, 128, 128), (2, 33, 63, 64, 128), (3, 40, 97, 128, 64), (5, 40, 33, 32, 128),
                                         (1, 3, 190, 32, 64), (2, 50, 380, 64, 64), (1, 16, 5, 128, 128), (2, 8, 380, 128, 128)])
@pytest.mark.parametrize("padded", [False, True])
def test_forward_alone(cottn, dtype, B, H, N, dk, dv, padded):
    """Without a workspace for a backward: one segment in parts of the value columns, from a state and with lengths."""
    lens = [N - 7 * b if b % 3 else b for b in range(B)] if padded else None
    x = draw(B, H, N, dk, dv, dtype, N + B, lens=lens, states=True)
    d = {k: v.cuda() for k, v in x.items()}
    state = torch.full((B, H, dk, dv), float("nan"), device="cuda")
    O = cottn.cottn_fwd_causal_decay(d["Q"], d["K"], d["V"], d["s"], d["log_decay"], state_in=d["state_in"], state=state,
                                     seq_len=None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda(),
                                     O=torch.full_like(d["V"], float("nan")))
    f = {k: v.double() for k, v in x.items()}
    want, S, M, MS = ref.forward(f["Q"], f["K"], f["V"], x["s"], x["log_decay"], lens, f["state_in"])
    n = N + max(dk, dv) + 40
    assert worst(O, want, M, U[dtype], n) <= 1.0 and worst(state, S, MS, U[dtype], n, in_fp32=True) <= 1.0
    assert norm_error(O, want) <= NORM * U[dtype] + 2e-6 and norm_error(state, S) <= 2 * U[dtype] ** 2 + 2e-6


def test_no_decay_is_the_call_without(cottn):
    x = draw(2, 3, 300, 64, 64, "bf16", 9)
    x["log_decay"] = torch.zeros(3)
    out = run(cottn, x)
    d = {k: v.cuda() for k, v in x.items()}
    O = cottn.cottn_fwd_causal(d["Q"], d["K"], d["V"], d["s"])
    grads = cottn.cottn_bwd_causal(d["Q"], d["K"], d["V"], d["s"], d["dO"])
    for a, b in zip((out["O"], out["dQ"], out["dK"], out["dV"]), (O,) + grads[:3]):
        assert norm_error(a, b.cpu().double()) <= 4 * U["bf16"]   # (that call rounds the normalised rows too)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces(cottn, dtype):
    """A sequence in three pieces, the states handed on, is the sequence."""
    N, cuts = 500, [0, 130, 131, 500]
    x = draw(2, 3, N, 64, 32, dtype, 11)
    d = {k: v.cuda() for k, v in x.items()}
    S, states, O = None, [], []
    pieces = list(zip(cuts[:-1], cuts[1:]))
    part = lambda k, lo, hi: d[k][:, :, lo:hi].contiguous()   # noqa: E731
    for lo, hi in pieces:
        states.append(S)
        S = torch.empty(2, 3, 64, 32, device="cuda")
        O.append(cottn.cottn_fwd_causal_decay(*(part(k, lo, hi) for k in "QKV"), d["s"], d["log_decay"], state_in=states[-1], state=S))
    R, out, ds = None, {"dQ": [], "dK": [], "dV": []}, 0
    for (lo, hi), S0 in zip(reversed(pieces), reversed(states)):
        R2 = torch.empty(2, 3, 64, 32, device="cuda")
        g = cottn.cottn_bwd_causal_decay(*(part(k, lo, hi) for k in "QKV"), d["s"], d["log_decay"], part("dO", lo, hi), state_in=S0,
                                         rev_state_in=R, rev_state_out=R2)
        R = R2
        ds = ds + g[3]
        for k, t in zip(out, g):
            out[k].insert(0, t)
    got = {k: torch.cat(v, 2) for k, v in out.items()}
    got.update(O=torch.cat(O, 2), state=S, rev=R, ds=ds)
    check(got, x, dtype)


def test_nothing_to_do(cottn):
    S0 = torch.randn(2, 3, 32, 64, device="cuda")
    e = lambda d: torch.empty(2, 3, 0, d, device="cuda", dtype=torch.bfloat16)   # noqa: E731
    s, ld = torch.ones(3, device="cuda"), torch.zeros(3, device="cuda")
    state = torch.empty_like(S0)
    cottn.cottn_fwd_causal_decay(e(32), e(32), e(64), s, ld, state_in=S0, state=state)
    assert torch.equal(state, S0)
    cottn.cottn_fwd_causal_decay(e(32), e(32), e(64), s, ld, state=state)
    assert not state.any()
    rev = torch.empty_like(S0)
    ds = cottn.cottn_bwd_causal_decay(e(32), e(32), e(64), s, ld, e(64), rev_state_in=S0, rev_state_out=rev)[3]
    assert torch.equal(rev, S0) and not ds.any()


def test_rows_that_do_not_exist_are_not_read(cottn):
    lens = [70, 3, 0]
    x = draw(3, 2, 150, 64, 64, "bf16", 12, lens=lens)
    y = {k: v.clone() for k, v in x.items()}
    for b, n in enumerate(lens):
        for k in ("Q", "K", "V", "dO"):
            y[k][b, :, n:] = float("nan")
    a, b = run(cottn, x, lens=lens), run(cottn, y, lens=lens)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_same_bits_on_another_stream_and_again(cottn):
    x = draw(2, 8, 900, 64, 64, "bf16", 13, states=True)
    a = run(cottn, x)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = run(cottn, x)
    side.synchronize()
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_captured(cottn):
    """Forward and backward in a graph: every replay, with eager work between, gives the eager bits."""
    B, H, N, d = 2, 8, 700, 64
    x = {k: v.cuda() for k, v in draw(B, H, N, d, d, "bf16", 14).items()}
    n, m = (cottn.cottn_workspace_bytes_dkdv(op, B, H, N, d, d, 0, cottn.COTTN_BF16) for op in (cottn.OP_FWD_DECAY, cottn.OP_BWD_DECAY))
    ws, ws2 = (torch.empty(max(i, 1), dtype=torch.uint8, device="cuda") for i in (n, m))
    O, dQ, dK, dV = (torch.empty_like(x["Q"]) for _ in range(4))
    ds, state = torch.empty(H, device="cuda"), torch.empty(B, H, d, d, device="cuda")

    def call():
        cottn.cottn_fwd_causal_decay(x["Q"], x["K"], x["V"], x["s"], x["log_decay"], O=O, state=state, workspace=ws)
        cottn.cottn_bwd_causal_decay(x["Q"], x["K"], x["V"], x["s"], x["log_decay"], x["dO"], dQ=dQ, dK=dK, dV=dV, ds=ds,
                                     workspace=ws2, fwd_workspace=ws)

    outs = (O, dQ, dK, dV, ds, state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        new = draw(B, H, N, d, d, "bf16", 15 + i)
        for k in ("Q", "K", "V", "dO"):
            x[k].copy_(new[k])
        call()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("B,N,segments", [(5, 16384, 0), (160, 2048, 1)])
def test_more_than_the_caches_hold(cottn, B, N, segments):
    """Calls of 0.3 and 1.3 GB: the last sequence's results are those of a call of its own, both within two roundings of the
    true ones."""
    H, d = 8, 64
    g = torch.Generator(device="cuda").manual_seed(21)
    Q, K, V, dO = (torch.randn(B, H, N, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(4))
    s, ld = torch.ones(H, device="cuda"), -torch.exp(torch.linspace(-6.0, 0.0, H)).cuda()
    one = [t[-1:].contiguous() for t in (Q, K, V, dO)]
    cottn.cottn_tune_segments(segments)
    try:
        got = [cottn.cottn_fwd_causal_decay(Q, K, V, s, ld), *cottn.cottn_bwd_causal_decay(Q, K, V, s, ld, dO)[:3]]
    finally:
        cottn.cottn_tune_segments(0)
    want = [cottn.cottn_fwd_causal_decay(*one[:3], s, ld), *cottn.cottn_bwd_causal_decay(*one[:3], s, ld, one[3])[:3]]
    for a, b in zip(got, want):
        assert norm_error(a[-1:], b.cpu().double()) <= 2 * NORM * U["bf16"]


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 128, 128), ("f16", 64, 128), ("f32", 64, 64), ("bf16", 32, 64)])
@pytest.mark.parametrize("N", [64, 65, 160, 257, 449, 1100])
def test_rows_dealt_to_workgroups(cottn, dtype, dk, dv, N):
    """One segment of few sequences, whose rows several workgroups share: lengths that end in each of them, and none."""
    lens = [N, N // 2 + 1, N // 4, 1, 0]
    x = draw(5, 2, N, dk, dv, dtype, N, lens=lens, states=True)
    d = {k: v.cuda() for k, v in x.items()}
    f = {k: v.double() for k, v in x.items()}
    n = N + max(dk, dv) + 40
    cottn.cottn_tune_segments(1)
    try:
        for some in (None, lens):
            state = torch.full((5, 2, dk, dv), float("nan"), device="cuda")
            s = x["s"] if some is not None else x["s"][0].contiguous()
            O = cottn.cottn_fwd_causal_decay(d["Q"], d["K"], d["V"], s.cuda(), d["log_decay"], state_in=d["state_in"], state=state,
                                             seq_len=None if some is None else torch.tensor(some, dtype=torch.int32).cuda(),
                                             O=torch.full_like(d["V"], float("nan")))
            want, S, M, MS = ref.forward(f["Q"], f["K"], f["V"], s, x["log_decay"], some, f["state_in"])
            assert worst(O, want, M, U[dtype], n) <= 1.0 and worst(state, S, MS, U[dtype], n, in_fp32=True) <= 1.0
            assert norm_error(O, want) <= NORM * U[dtype] + 2e-6 and norm_error(state, S) <= 2 * U[dtype] ** 2 + 2e-6
            if some is not None:
                assert all(not O[b, :, m:].any() for b, m in enumerate(some))
    finally:
        cottn.cottn_tune_segments(0)
