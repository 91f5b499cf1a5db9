"""Refusals of the calls with a decay and of the tree calls, before anything would be enqueued, without a GPU."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, HIP, ARG = range(8)
NO_SIZE = ctypes.c_size_t(-1).value
P, BIG = 1 << 20, 1 << 40   # places that are never read: the calls are refused


@pytest.fixture(scope="module")
def lib():
    lib = ctypes.CDLL(os.path.join(ROOT, "paper_2409_18747_amd", "libcottn.so"))
    vp, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.cottn_workspace_bytes_dkdv.restype = sz
    lib.cottn_workspace_bytes_dkdv.argtypes = [i] * 8
    lib.cottn_segments_dkdv.argtypes = [i] * 8
    lib.cottn_fwd_causal_decay.argtypes = [vp] * 10 + [sz] + [i] * 6 + [f, vp]
    lib.cottn_bwd_causal_decay.argtypes = [vp] * 15 + [sz, vp, sz] + [i] * 6 + [f, vp]
    lib.cottn_step_decay.argtypes = [vp] * 7 + [i, vp, vp] + [i] * 5 + [f, vp]
    lib.cottn_tree.argtypes = [vp] * 8 + [i] * 6 + [f, vp]
    lib.cottn_tree_accept.argtypes = [vp] * 6 + [i] * 6 + [f, vp]
    lib.cottn_tune_segments(0)
    yield lib
    lib.cottn_tune_segments(0)


FWD = dict(Q=P, K=P, V=P, s=P, log_decay=P, seq_len=None, state_in=None, O=P, state=None, ws=256 * P, ws_bytes=BIG, B=2, H=3, N=100,
           dk=64, dv=64, dtype=1, eps=1e-6, stream=None)
BWD = dict(Q=P, K=P, V=P, s=P, log_decay=P, seq_len=None, dO=P, state_in=None, rev_in=None, dQ=P, dK=P, dV=P, ds=P, rev_out=None,
           fws=None, fws_bytes=0, ws=256 * P, ws_bytes=BIG, B=2, H=3, N=100, dk=64, dv=64, dtype=1, eps=1e-6, stream=None)
STEP = dict(q=P, k=P, v=P, s=P, log_decay=P, state_in=P, parent=None, B_in=2, state=P, o=P, B=2, H=3, dk=64, dv=64, dtype=1,
            eps=1e-6, stream=None)
TREE = dict(q=P, k=P, v=P, s=P, log_decay=P, parent=P, state=P, o=P, B=2, H=3, T=8, dk=64, dv=64, dtype=1, eps=1e-6, stream=None)
ACCEPT = dict(k=P, v=P, log_decay=P, parent=P, last=P, state=P, B=2, H=3, T=8, dk=64, dv=64, dtype=1, eps=1e-6, stream=None)
COMMON = [({"dk": 48}, SHAPE), ({"dv": 256}, SHAPE), ({"B": 0}, SHAPE), ({"H": -1}, SHAPE), ({"dtype": 3}, DTYPE), ({"eps": 0.0}, ARG),
          ({"eps": float("nan")}, ARG), ({"B": 1 << 20, "H": 1 << 20}, SHAPE), ({"log_decay": P + 2}, ALIGN)]


def refused(lib, name, base, change, status):
    args = dict(base)
    args.update(change)
    return getattr(lib, name)(*args.values()) == status


@pytest.mark.parametrize("change,status", COMMON + [({k: None}, NULL) for k in ("Q", "K", "V", "s", "log_decay", "O")] + [
    ({"N": -1}, SHAPE), ({"Q": P + 8}, ALIGN), ({"state": P + 4}, ALIGN), ({"state_in": P + 8}, ALIGN), ({"seq_len": P + 1}, ALIGN),
    ({"state_in": P, "state": P}, ARG), ({"state_in": P, "state": P + 64}, ARG), ({"state_in": P + 6 * 64 * 64 * 4 - 16, "state": P}, ARG),
    ({"N": 5000, "ws": None}, WORKSPACE), ({"N": 5000, "ws_bytes": 16}, WORKSPACE), ({"N": 5000, "ws": 256 * P + 16}, ALIGN)])
def test_forward(lib, change, status):
    assert refused(lib, "cottn_fwd_causal_decay", FWD, change, status)


@pytest.mark.parametrize("change,status", COMMON + [({k: None}, NULL) for k in ("Q", "K", "V", "s", "log_decay", "dO", "dQ", "dK", "dV", "ds")] + [
    ({"N": -1}, SHAPE), ({"dV": P + 8}, ALIGN), ({"rev_in": P + 4}, ALIGN), ({"rev_out": P + 4}, ALIGN), ({"seq_len": P + 2}, ALIGN),
    ({"rev_in": P, "rev_out": P}, ARG), ({"rev_in": P, "rev_out": P + 16}, ARG), ({"state_in": P, "rev_out": P}, ARG),
    ({"ws": None}, WORKSPACE), ({"ws_bytes": 0}, WORKSPACE), ({"N": 5000, "fws": 256 * P, "fws_bytes": 16}, WORKSPACE),
    ({"N": 5000, "fws": 256 * P + 16, "fws_bytes": BIG}, ALIGN)])
def test_backward(lib, change, status):
    assert refused(lib, "cottn_bwd_causal_decay", BWD, change, status)


@pytest.mark.parametrize("change,status", COMMON + [({k: None}, NULL) for k in ("q", "k", "v", "s", "state_in", "state", "o")] + [
    ({"B_in": 3}, SHAPE), ({"B_in": 0, "parent": P}, SHAPE), ({"parent": P + 2}, ALIGN), ({"state_in": P + 8}, ALIGN),
    ({"parent": P}, ARG), ({"state_in": P + 16}, ARG), ({"parent": P, "B_in": 9, "state_in": P, "state": P + 8 * 3 * 64 * 64 * 4}, ARG)])
def test_step(lib, change, status):
    assert refused(lib, "cottn_step_decay", STEP, change, status)


@pytest.mark.parametrize("change,status", COMMON + [({k: None}, NULL) for k in ("q", "k", "v", "s", "parent", "state", "o")] + [
    ({"T": 65}, SHAPE), ({"T": -1}, SHAPE), ({"parent": P + 2}, ALIGN), ({"o": P + 2}, ALIGN), ({"T": 0}, OK)])
def test_tree(lib, change, status):
    assert refused(lib, "cottn_tree", TREE, change, status)


@pytest.mark.parametrize("change,status", COMMON + [({k: None}, NULL) for k in ("k", "v", "parent", "last", "state")] + [
    ({"T": 65}, SHAPE), ({"T": -1}, SHAPE), ({"last": P + 2}, ALIGN), ({"state": P + 4}, ALIGN), ({"T": 0}, OK)])
def test_accept(lib, change, status):
    assert refused(lib, "cottn_tree_accept", ACCEPT, change, status)


def test_sizes(lib):
    size, segments = lib.cottn_workspace_bytes_dkdv, lib.cottn_segments_dkdv
    for dtype, chunk in ((0, 32), (1, 64), (2, 64)):
        lib.cottn_tune_segments(1)
        assert size(5, 2, 3, 1000, 64, 32, 0, dtype) == 0
        assert size(6, 2, 3, 1000, 64, 32, 0, dtype) == 256     # one partial sum of ds each
        lib.cottn_tune_segments(5)
        assert segments(5, 2, 3, 1000, 64, 32, 0, dtype) == segments(6, 2, 3, 1000, 64, 32, chunk, dtype)
        g = segments(5, 2, 3, 1000, 64, 32, 0, dtype)
        assert size(5, 2, 3, 1000, 64, 32, 0, dtype) == 6 * g * 64 * 32 * 4
        assert size(6, 2, 3, 1000, 64, 32, chunk, dtype) == 2 * 6 * g * 64 * 32 * 4 + 256
        lib.cottn_tune_segments(0)
        assert size(5, 2, 3, 1000, 64, 32, 128, dtype) == NO_SIZE and segments(5, 2, 3, 1000, 64, 32, 128, dtype) == 0
        assert size(5, 2, 3, 0, 64, 32, 0, dtype) == 0
    assert size(7, 2, 3, 1000, 64, 32, 0, 1) == size(9, 2, 3, 1000, 64, 32, 0, 1) == NO_SIZE


def test_a_forward_alone_needs_no_more(lib):
    """It takes as many segments as with its backward, or fewer, as short prompts of few sequences and many sequences do."""
    size = lib.cottn_workspace_bytes_dkdv
    fewer = 0
    for dtype in (0, 1, 2):
        for B in (1, 4, 8, 16, 40):
            for N in (1, 64, 128, 192, 384, 385, 2048, 30000):
                for dk, dv in ((32, 32), (64, 64), (64, 128), (128, 128)):
                    pair, alone = size(5, B, 16, N, dk, dv, 0, dtype), size(8, B, 16, N, dk, dv, 0, dtype)
                    assert 0 <= alone <= pair
                    fewer += alone < pair
    assert fewer > 50
    # without room the forward takes that split; where neither fits it is refused
    assert refused(lib, "cottn_fwd_causal_decay", {**FWD, "B": 1, "H": 16, "N": 2048}, {"ws": None}, WORKSPACE)
    lib.cottn_tune_segments(4)
    assert size(8, 1, 16, 192, 128, 128, 0, 1) == size(5, 1, 16, 192, 128, 128, 0, 1) > 0
    lib.cottn_tune_segments(0)
