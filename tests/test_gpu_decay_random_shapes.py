"""Seeded random calls with a decay against 64 bits: any widths, types, numbers of sequences and rows, splits, lengths, states, decays and
what is asked for."""
import random

import pytest
import torch

import decay_reference as ref
from decay_reference import U, worst
from test_gpu_decay import check, cottn, draw, run   # noqa: F401
from test_gpu_decay_launches import train

pytestmark = pytest.mark.gpu

SEEDS = range(80)


@pytest.mark.parametrize("seed", SEEDS)
def test_call(cottn, seed):   # noqa: F811
    rng = random.Random(seed)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    dk, dv = rng.choice([32, 64, 128]), rng.choice([32, 64, 128])
    B, H = rng.choice([1, 1, 2, 3, 7, 20]), rng.choice([1, 2, 5, 8, 13])
    N = int(2 ** rng.uniform(0, 10.5))
    N = max(1, min(N, int(2.0e7 / (B * H * (N + 64)))))   # (the 64-bit form is quadratic)
    lens = [rng.randint(-2, N + 2) for _ in range(B)] if rng.random() < 0.4 else None
    x = draw(B, H, N, dk, dv, dtype, seed, lens=lens, states=rng.random() < 0.5)
    if rng.random() < 0.3:
        x["log_decay"] = torch.tensor([rng.choice([0.0, -1e-6, -0.01, -0.3, -4.0, -60.0, float("-inf"), 0.2]) for _ in range(H)])
    segments, share = rng.choice([0, 0, 0, 1, 2, 3, 7, 50]), rng.random() < 0.7
    print(dict(dtype=dtype, dk=dk, dv=dv, B=B, H=H, N=N, lens=lens, segments=segments, share=share, states="state_in" in x))
    cottn.cottn_tune_segments(segments)
    try:
        out = run(cottn, x, lens=lens, share=share)
        mine = train(cottn, x, lens, share)
        d = {k: v.cuda() for k, v in x.items()}
        alone, state = torch.full_like(d["V"], float("nan")), torch.full((B, H, dk, dv), float("nan"), device="cuda")
        cottn.cottn_fwd_causal_decay(d["Q"], d["K"], d["V"], d["s"], d["log_decay"], state_in=d.get("state_in"), O=alone, state=state,
                                     seq_len=None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda())
    finally:
        cottn.cottn_tune_segments(0)
    there = None if lens is None else [min(N, max(0, n)) for n in lens]
    for o in (out, {**out, **mine}):
        check(o, x, dtype, lens=there, norms=False)
    f = {k: v.double() for k, v in x.items()}
    O, S, M, MS = ref.forward(f["Q"], f["K"], f["V"], x["s"], x["log_decay"], there, f.get("state_in"))
    n = N + max(dk, dv) + 40
    floor = ref.f16_floor(x["s"], x["V"], dk) if dtype == "f16" else 0.0
    assert worst(alone, O, M, U[dtype], n, floor=floor) <= 1.0 and worst(state, S, MS, U[dtype], n, in_fp32=True) <= 1.0
