"""fp16 backward with a decay: the products dO . v, which the kernels keep in 16 bits, may be anything that fp16 holds, as in the
backward without a decay.  (They were kept times a row's factor between 2 and 4, which overflowed from 16 400 on.)"""
import pytest
import torch

import decay_reference as ref
from test_gpu_decay import check, cottn, draw, run   # noqa: F401

pytestmark = pytest.mark.gpu


def large_products(dk, dv, N, most, seed):
    """Rows whose largest |dO_i . v_j|, j <= i, is `most`; q and k are long, so that no gradient is beyond fp16."""
    x = draw(2, 3, N, dk, dv, "f16", seed)
    for k, by in (("Q", 8.0), ("K", 8.0), ("V", 16.0)):
        x[k] = x[k] * by   # (powers of two)
    dots = lambda: (x["dO"].double() @ x["V"].double().transpose(-1, -2)).tril().abs().max()   # noqa: E731
    for _ in range(4):   # (the roundings of dO move the largest product by 2^-11)
        x["dO"] = (x["dO"].double() * (most / float(dots()))).half()
    assert 0.99 * most < float(dots()) < 65504
    return x


@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (32, 64), (128, 32), (64, 128)])
@pytest.mark.parametrize("most", [16000.0, 30000.0, 65000.0])
@pytest.mark.parametrize("segments", [0, 1])
def test_largest_products(cottn, dk, dv, most, segments):   # noqa: F811
    x = large_products(dk, dv, 150, most, dk + dv)
    cottn.cottn_tune_segments(segments)
    try:
        out = run(cottn, x)
    finally:
        cottn.cottn_tune_segments(0)
    check(out, x, "f16")


def test_as_without_a_decay(cottn):   # noqa: F811
    x = large_products(64, 64, 150, 60000.0, 5)
    x["log_decay"] = torch.zeros(3)
    out = run(cottn, x)
    d = {k: v.cuda() for k, v in x.items()}
    for a, b in zip((out["dQ"], out["dK"], out["dV"]), cottn.cottn_bwd_causal(d["Q"], d["K"], d["V"], d["s"], d["dO"])):
        assert torch.isfinite(b).all()
        assert ref.norm_error(a, b.cpu().double()) <= 4 * ref.U["f16"]   # (that call rounds the normalised rows too)
