"""States, reverse-time states and ds come out to fp32's accuracy whatever the element type (decay_accuracy derives the bounds;
test_decay_accuracy_cpu shows that operands in one part fewer would not meet them)."""
import pytest
import torch

import decay_accuracy as acc
import decay_reference as ref
from decay_reference import TYPES
from test_gpu_decay import cottn, run   # noqa: F401

pytestmark = pytest.mark.gpu

B, H = 3, 6
CHUNK = {"bf16": 64, "f16": 64, "f32": 32}


def draw(N, dk, dv, dtype, seed, H=H):
    g = torch.Generator().manual_seed(seed)
    x = {k: torch.randn(B, H, N, d, generator=g).to(TYPES[dtype]) for k, d in (("Q", dk), ("K", dk), ("V", dv), ("dO", dv))}
    x["s"] = torch.rand(B, H, generator=g) + 0.5
    x["log_decay"] = -torch.exp(torch.linspace(-9.0, 0.0, H))
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (32, 128), (128, 32), (64, 128), (32, 32)])
@pytest.mark.parametrize("N", [64, 130, 260])
@pytest.mark.parametrize("segments", [1, 2])
def test_states_and_ds(cottn, dtype, dk, dv, N, segments):   # noqa: F811
    lens = [N] * B   # (ds of each sequence)
    x = draw(N, dk, dv, dtype, N + dk + dv)
    cottn.cottn_tune_segments(segments)
    try:
        out = run(cottn, x, lens=lens)
    finally:
        cottn.cottn_tune_segments(0)
    f = {k: v.double() for k, v in x.items()}
    state = ref.forward(f["Q"], f["K"], f["V"], x["s"], x["log_decay"], lens)[1]
    want = ref.backward(f["Q"], f["K"], f["V"], x["s"], x["log_decay"], f["dO"], lens)
    found = (acc.state_error(out["state"], state) / acc.state_bound(N), acc.state_error(out["rev"], want["rev"][0]) / acc.state_bound(N),
             acc.ds_error(out["ds"], want["ds"][0], acc.ds_terms(x, x["log_decay"])) / acc.ds_bound(N, dk, dv, CHUNK[dtype]))
    print(found)
    assert all(e <= 1.0 for e in found), found


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv,H", [(64, 64, 6), (128, 128, 6), (128, 64, 30), (64, 128, 60), (128, 128, 90)])
@pytest.mark.parametrize("N", [64, 260])
def test_states_of_a_forward_alone(cottn, dtype, dk, dv, H, N):   # noqa: F811
    """In parts of the value columns and of the rows, where sequences are few, and in one piece."""
    x = draw(N, dk, dv, dtype, N + dk + H, H)
    d = {k: v.cuda() for k, v in x.items()}
    state = torch.full((B, H, dk, dv), float("nan"), device="cuda")
    cottn.cottn_fwd_causal_decay(d["Q"], d["K"], d["V"], d["s"][0].contiguous(), d["log_decay"], state=state)
    f = {k: v.double() for k, v in x.items()}
    want = ref.forward(f["Q"], f["K"], f["V"], x["s"][0], x["log_decay"])[1]
    found = acc.state_error(state, want) / acc.state_bound(N)
    print(found)
    assert found <= 1.0
