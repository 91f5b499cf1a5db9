"""Pairs of an axis that there is not are not turned: their features stay bit for bit what they are, whatever the pair's other feature
is."""
import pytest
import torch

from test_gpu_delta_step import cottn   # noqa: F401

pytestmark = pytest.mark.gpu
KINDS = {"bf16": (torch.bfloat16, torch.int16), "f16": (torch.float16, torch.int16), "f32": (torch.float32, torch.int32)}


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,pairs,N", [(32, 16, 70), (64, 32, 130), (64, 15, 40), (128, 64, 1), (128, 24, 33)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_pairs_that_are_not_turned(cottn, dtype, d, pairs, N, neighbours):   # noqa: F811
    kind, bits = KINDS[dtype]
    g = torch.Generator().manual_seed(d + pairs)
    B, H, axes = 2, 3, 2
    X = torch.randn(B, H, N, d, generator=g)
    for value in (float("inf"), -float("inf"), float("nan"), -0.0, 0.0):
        X[torch.rand(X.shape, generator=g) < 0.1] = value
    X = X.to(kind)
    p = torch.arange(pairs)
    a, b = (2 * p, 2 * p + 1) if neighbours else (p, p + pairs)
    axis = torch.tensor([(0, 5, 1, -1, -2 ** 31, axes)[i % 6] for i in range(pairs)], dtype=torch.int32)
    still = (axis < 0) | (axis >= axes)
    at = torch.randint(1, 1000, (B, N, axes), generator=g).to(torch.int32)
    freq = torch.rand(pairs, generator=g) + 0.1
    for inverse in (False, True):
        got = cottn.cottn_rotary(X.cuda(), X.cuda(), at.cuda(), freq.cuda(), axis=axis.cuda(), neighbours=neighbours, inverse=inverse)
        for t in got:
            for f in (a[still], b[still], torch.arange(2 * pairs, d)):
                assert torch.equal(t.cpu().view(bits)[..., f], X.view(bits)[..., f])
        finite = torch.isfinite(X[..., a]) & torch.isfinite(X[..., b])
        for f in (a, b):
            assert torch.isfinite(got[0].cpu()[..., f][finite]).all()
