"""The launches that training steps and large calls make, against 64 bits: calls that ask for no state (whose operands are in fewer
parts), the 32-row scan of many 128 x 128 sequences, and totals that a launch of its own carries, at every kind of width."""
import itertools

import pytest
import torch

import decay_reference as ref
from decay_reference import U, norm_error, worst
from test_gpu_decay import NORM, check, cottn, draw, run   # noqa: F401

pytestmark = pytest.mark.gpu


def train(cottn, x, lens=None, share=True):   # noqa: F811
    """A training step: neither the state nor a reverse-time one is asked for."""
    d = {k: v.cuda() for k, v in x.items()}
    B, H, N, dk = x["Q"].shape
    dv = x["V"].shape[-1]
    code = {torch.float32: cottn.COTTN_F32, torch.bfloat16: cottn.COTTN_BF16, torch.float16: cottn.COTTN_F16}[x["Q"].dtype]
    n = cottn.cottn_workspace_bytes_dkdv(cottn.OP_FWD_DECAY, B, H, N, dk, dv, 0, code)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None   # what is not written first is NaN
    sl = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
    nan = lambda k: torch.full_like(d[k], float("nan"))   # noqa: E731
    out = {"O": cottn.cottn_fwd_causal_decay(d["Q"], d["K"], d["V"], d["s"], d["log_decay"], seq_len=sl, state_in=d.get("state_in"),
                                             O=nan("V"), workspace=ws)}
    m = cottn.cottn_workspace_bytes_dkdv(cottn.OP_BWD_DECAY, B, H, N, dk, dv, 0, code)
    out["dQ"], out["dK"], out["dV"], out["ds"] = cottn.cottn_bwd_causal_decay(
        d["Q"], d["K"], d["V"], d["s"], d["log_decay"], d["dO"], seq_len=sl, state_in=d.get("state_in"), rev_state_in=d.get("rev_in"),
        dQ=nan("Q"), dK=nan("K"), dV=nan("V"), workspace=torch.full((m,), 0xFF, dtype=torch.uint8, device="cuda"),
        fwd_workspace=ws if share else None)
    torch.cuda.synchronize()
    return out


def check_training(cottn, x, dtype, lens=None, share=True, segments=0):   # noqa: F811
    cottn.cottn_tune_segments(segments)
    try:
        out = train(cottn, x, lens, share)
        asked = run(cottn, x, lens)
    finally:
        cottn.cottn_tune_segments(0)
    check({**asked, **out}, x, dtype, lens=None if lens is None else [min(x["Q"].shape[2], max(0, n)) for n in lens])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", list(itertools.product((32, 64, 128), repeat=2)))
@pytest.mark.parametrize("segments,share,states", [(0, True, False), (1, True, True), (3, False, True)])
def test_training(cottn, dtype, dk, dv, segments, share, states):   # noqa: F811
    x = draw(2, 3, 200, dk, dv, dtype, 20 + dk + dv, states=states)
    check_training(cottn, x, dtype, share=share, segments=segments)


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 64, 64), ("bf16", 128, 128), ("f16", 64, 128), ("f32", 128, 64)])
@pytest.mark.parametrize("segments", [0, 4])
def test_training_of_padded_batches(cottn, dtype, dk, dv, segments):   # noqa: F811
    lens = [0, 1, 64, 65, 257, 400, -3, 500]
    x = draw(len(lens), 2, 400, dk, dv, dtype, 6, lens=lens)
    check_training(cottn, x, dtype, lens=lens, segments=segments)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("N,padded", [(100, False), (97, True), (33, False)])
def test_many_wide_sequences(cottn, dtype, N, padded):   # noqa: F811
    """258 of 128 x 128: with a state and without one."""
    B, H = 6, 43
    lens = [N, N // 2, 32, 31, 0, N - 1] if padded else None
    x = draw(B, H, N, 128, 128, dtype, N, lens=lens, states=True)
    assert cottn.cottn_segments_dkdv(cottn.OP_FWD_DECAY, B, H, N, 128, 128, 0, cottn.COTTN_BF16) == 1
    check_training(cottn, x, dtype, lens=lens)


# (B, H) = (1, 2): totals are carried from some 19 segments of 64 x 64 on
@pytest.mark.parametrize("dtype,dk,dv,N,segments", [("bf16", 64, 64, 1600, 25), ("f16", 64, 64, 1590, 25), ("f32", 64, 64, 800, 25),
                                                    ("f32", 32, 64, 1300, 41), ("bf16", 128, 32, 1500, 24), ("bf16", 32, 128, 1500, 24),
                                                    ("bf16", 64, 128, 900, 15), ("f32", 128, 128, 700, 22), ("bf16", 128, 128, 1000, 16)])
@pytest.mark.parametrize("padded", [False, True])
def test_carried(cottn, dtype, dk, dv, N, segments, padded):   # noqa: F811
    lens = [N - 3, N // 3] if padded else None
    x = draw(2 if padded else 1, 2, N, dk, dv, dtype, N, lens=lens, states=True)
    cottn.cottn_tune_segments(segments)
    try:
        cottn.profile_start()
        try:
            out = run(cottn, x, lens=lens)
        finally:
            launched = cottn.profile_stop()
        assert sum(n for name, (n, _) in launched.items() if "decay_carry" in name) == 2, launched
        alone = train(cottn, x, lens, share=False)
    finally:
        cottn.cottn_tune_segments(0)
    check(out, x, dtype, lens=lens)
    check({**out, **alone}, x, dtype, lens=lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_forward_alone_of_many_sequences(cottn, dtype):   # noqa: F811
    """Sequences enough to be whole: no parts of columns or rows."""
    B, H, N = 2, 129, 130
    for dk, dv in ((64, 64), (32, 128), (128, 64)):
        x = draw(B, H, N, dk, dv, dtype, dk, states=True)
        d, f = {k: v.cuda() for k, v in x.items()}, {k: v.double() for k, v in x.items()}
        state = torch.full((B, H, dk, dv), float("nan"), device="cuda")
        O = cottn.cottn_fwd_causal_decay(d["Q"], d["K"], d["V"], d["s"], d["log_decay"], state_in=d["state_in"], state=state)
        want, S, M, MS = ref.forward(f["Q"], f["K"], f["V"], x["s"], x["log_decay"], None, f["state_in"])
        assert worst(O, want, M, U[dtype], N + 168) <= 1.0 and worst(state, S, MS, U[dtype], N + 168, in_fp32=True) <= 1.0
        assert norm_error(O, want) <= NORM * U[dtype] + 2e-6
