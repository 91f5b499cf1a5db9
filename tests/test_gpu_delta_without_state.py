"""A 16-bit forward by the gated delta rule that is asked for no state has the recurrence of one that is: the same results, also where
nothing contracts and errors add up over a long sequence."""
import pytest
import torch

import delta_reference as ref
from delta_reference import TYPES, U
from test_gpu_delta import cottn, cuda, double, draw   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", [(32, 64), (64, 64), (64, 32), (128, 128)])
@pytest.mark.parametrize("G", [1, 4])
def test_the_same_results(cottn, dtype, dk, dv, G):   # noqa: F811
    x, more = draw(2, 3, 500, dk, dv, dtype, dk + dv)
    x["beta"] *= 2.0
    x["log_decay"] /= 16.0
    d, m = cuda(x), cuda(more)
    cottn.cottn_tune_segments(G)
    try:
        for from_ in (None, m["state_in"]):
            O = cottn.cottn_fwd_causal_delta(**d, state_in=from_, state=torch.empty_like(m["state_in"]))
            assert torch.equal(cottn.cottn_fwd_causal_delta(**d, state_in=from_), O)
    finally:
        cottn.cottn_tune_segments(0)


def test_nothing_contracts(cottn):   # noqa: F811
    """beta 2, no decay, 256 chunks.  A result is off by its rounding, and by what it is rounded from: 768 roundings of 2^-24 a chunk,
    whose signs are as good as random, and the last products' operands in two parts, 2^-15 of a product."""
    N = 16384
    x, _ = draw(1, 2, N, 64, 32, "f16", 4)
    x["beta"].fill_(2.0)
    x["log_decay"].zero_()
    want, _ = ref.forward(**double(x))
    got = cottn.cottn_fwd_causal_delta(**cuda(x)).double().cpu()
    norm = float(want.norm())
    rounding = float((want.to(TYPES["f16"]).double() - want).norm()) / norm
    off = float((got - want).norm()) / norm
    print("rounding %.3g, off %.3g" % (rounding, off))
    assert off <= rounding + (N // 64 * 768) ** 0.5 * U["f32"] + 2.0 ** -15
