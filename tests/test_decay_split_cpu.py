"""The split of a call with a decay into segments, from the library itself, without a GPU."""
import ctypes
import itertools
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAIR, BACKWARD, ALONE = 5, 6, 8
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def segments():
    lib = ctypes.CDLL(os.path.join(ROOT, "paper_2409_18747_amd", "libcottn.so"))
    lib.cottn_tune_segments(0)
    return lambda op, units, rows, dk, dv, dtype: lib.cottn_segments_dkdv(op, 1, units, rows, dk, dv, 0, dtype)


@pytest.mark.parametrize("dk,dv", itertools.product((32, 64, 128), repeat=2))
def test_two_chunks(segments, dk, dv):
    """With a backward, 16-bit sequences of two chunks are cut up to 128 of them, whatever the model says; no others need the rule."""
    for dtype in (BF16, F16):
        assert all(segments(PAIR, units, rows, dk, dv, dtype) == 2 for units in (1, 16, 77, 128) for rows in (65, 100, 128))
        assert all(segments(PAIR, units, rows, dk, dv, dtype) == 1 for units in (129, 192, 300, 1000) for rows in (65, 128))
    assert segments(PAIR, 300, 64, dk, dv, F32) == 1


@pytest.mark.parametrize("dk,dv", itertools.product((32, 64, 128), repeat=2))
@pytest.mark.parametrize("dtype,chunk", [(F32, 32), (BF16, 64)])
def test_long_sequences_are_cut(segments, dk, dv, dtype, chunk):
    """Few sequences of more than four chunks in no fewer segments than keep the compute units busy, and no call in more than 1024
    workgroups or than it has chunks; the backward takes the forward's split, a forward alone no more."""
    for units in (1, 5, 40, 96, 160, 383, 800):
        for chunks in (1, 2, 3, 5, 9, 17, 64, 500):
            g, alone = segments(PAIR, units, chunks * chunk, dk, dv, dtype), segments(ALONE, units, chunks * chunk, dk, dv, dtype)
            assert 1 <= alone <= g <= chunks and (g == 1 or units * g <= 1024)
            assert segments(BACKWARD, units, chunks * chunk, dk, dv, dtype) == g
            if units <= 96 and chunks > 4:
                assert g > 1
