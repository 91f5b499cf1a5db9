"""Calls with a decay and trees where 1 / eps or the reciprocal norms are so large that two of them multiplied leave fp32: zero rows, rows
that do not exist (which are filled with zeros) and short ones.  The normalised product of two rows is 1 at most all the same."""
import pytest
import torch

import decay_reference as ref
from decay_reference import U, worst
from test_gpu_decay import check, cottn, draw, run   # noqa: F401
from test_gpu_decode_decay import draw as draw_tokens, random_tree

pytestmark = pytest.mark.gpu

EPS = 1e-25


def shorten(x, q, k):
    """Zero rows of q and k, the same one and different ones, and all others times 2^-57 (some 1e-16 long)."""
    for name, zero in ((q, (3, 40)), (k, (3, 17))):
        x[name] = (x[name].double() * 2.0 ** -57).to(x[name].dtype)
        for i in zero:
            if i < x[name].shape[2]:
                x[name][:, :, i] = 0
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv,segments", [(64, 64, 0), (64, 64, 1), (128, 128, 2), (32, 128, 0)])
def test_rows(cottn, dtype, dk, dv, segments):   # noqa: F811
    x = shorten(draw(2, 3, 150, dk, dv, dtype, dk + dv), "Q", "K")
    cottn.cottn_tune_segments(segments)
    try:
        out = run(cottn, x, eps=EPS)
    finally:
        cottn.cottn_tune_segments(0)
    check(out, x, dtype, eps=EPS, norms=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T", [(2, 13), (13, 20), (13, 50)])
def test_tree(cottn, dtype, B, T):   # noqa: F811
    x, parent = shorten(draw_tokens(B, 6, T, 64, 64, dtype, T), "q", "k"), random_tree(B, T, T)
    d = {k: v.cuda() for k, v in x.items()}
    o = cottn.cottn_tree(d["q"], d["k"], d["v"], d["s"], d["S"], parent.cuda(), log_decay=d["ld"], eps=EPS)
    want, M = ref.tree(x["q"][:2].double(), x["k"][:2].double(), x["v"][:2].double(), x["s"], x["ld"], parent[:2], x["S"][:2].double(), EPS)
    assert torch.isfinite(o).all()
    assert worst(o[:2], want, M, U[dtype], T + 104) <= 1.0
