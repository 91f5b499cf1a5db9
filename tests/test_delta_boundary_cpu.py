"""Refusals of the calls by the gated delta rule and of rotary positions, before anything would be enqueued, and the sizes of their
workspaces, without a GPU."""
import ctypes
import os

import pytest

from test_decay_boundary_cpu import ALIGN, ARG, BIG, DTYPE, NO_SIZE, NULL, OK, P, ROOT, SHAPE, WORKSPACE, refused
import test_older_library_cpu as older

FWD_OP, ALONE_OP, BWD_OP, SAVED_OP = 16, 17, 18, 19
STATES = 2 * 3 * 64 * 64 * 4   # bytes of the states of the calls below


@pytest.fixture(scope="module")
def lib():
    lib = ctypes.CDLL(os.path.join(ROOT, "paper_2409_18747_amd", "libcottn.so"))
    vp, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.cottn_workspace_bytes_dkdv.restype = sz
    lib.cottn_workspace_bytes_dkdv.argtypes = [i] * 8
    lib.cottn_segments_dkdv.argtypes = [i] * 8
    lib.cottn_fwd_causal_delta.argtypes = [vp] * 11 + [sz] + [i] * 6 + [f, vp]
    lib.cottn_bwd_causal_delta.argtypes = [vp] * 18 + [sz, vp, sz] + [i] * 6 + [f, vp]
    lib.cottn_step_delta.argtypes = [vp] * 8 + [i, vp, vp] + [i] * 5 + [f, vp]
    lib.cottn_rotary.argtypes = [vp] * 7 + [i] * 9 + [vp]
    lib.cottn_tune_segments(0)
    yield lib
    lib.cottn_tune_segments(0)


FWD = dict(Q=P, K=P, V=P, s=P, log_decay=P, beta=P, seq_len=None, state_in=None, O=P, state=None, ws=256 * P, ws_bytes=BIG, B=2, H=3,
           N=100, dk=64, dv=64, dtype=1, eps=1e-6, stream=None)
BWD = dict(Q=P, K=P, V=P, s=P, log_decay=P, beta=P, seq_len=None, dO=P, state_in=None, dstate=None, dQ=P, dK=P, dV=P, ds=P,
           dlog_decay=P, dbeta=P, dstate_in=None, fws=None, fws_bytes=0, ws=256 * P, ws_bytes=BIG, B=2, H=3, N=100, dk=64, dv=64,
           dtype=1, eps=1e-6, stream=None)
STEP = dict(q=P, k=P, v=P, s=P, log_decay=P, beta=P, state_in=P, parent=None, B_in=2, state=P, o=P, B=2, H=3, dk=64, dv=64, dtype=1,
            eps=1e-6, stream=None)
ROTARY = dict(Q=P, K=2 * P, positions=P, freq=P, axis=None, Qr=3 * P, Kr=4 * P, B=2, H=3, N=100, d=64, pairs=32, axes=1, neighbours=0,
              inverse=0, dtype=1, stream=None)
COMMON = [({"dk": 48}, SHAPE), ({"dv": 256}, SHAPE), ({"B": 0}, SHAPE), ({"H": -1}, SHAPE), ({"dtype": 3}, DTYPE), ({"eps": 0.0}, ARG),
          ({"eps": float("nan")}, ARG), ({"B": 1 << 20, "H": 1 << 20}, SHAPE), ({"log_decay": P + 2}, ALIGN), ({"beta": P + 1}, ALIGN)]


@pytest.mark.parametrize("change,status", COMMON + [({k: None}, NULL) for k in ("Q", "K", "V", "s", "beta", "O")] + [
    ({"N": -1}, SHAPE), ({"Q": P + 8}, ALIGN), ({"state": P + 4}, ALIGN), ({"state_in": P + 8}, ALIGN), ({"seq_len": P + 1}, ALIGN),
    ({"state_in": P, "state": P + 64}, ARG), ({"state_in": P + STATES - 16, "state": P}, ARG), ({"ws": None}, WORKSPACE),
    ({"ws_bytes": 16}, WORKSPACE), ({"ws": 256 * P + 16}, ALIGN), ({"B": 1 << 11, "H": 1 << 12, "N": 64}, SHAPE), ({"B": 1 << 11, "H": 1 << 11, "N": 65}, SHAPE),
    ({"B": 1 << 11, "H": 1 << 11, "dv": 128}, SHAPE), ({"N": 0, "ws": None}, OK), ({"N": 0, "Q": None, "beta": None}, OK)])
def test_forward(lib, change, status):
    assert refused(lib, "cottn_fwd_causal_delta", FWD, change, status)


@pytest.mark.parametrize("change,status", COMMON + [({k: None}, NULL) for k in
                                                    ("Q", "K", "V", "s", "beta", "dO", "dQ", "dK", "dV", "ds", "dbeta")] + [
    ({"N": -1}, SHAPE), ({"dV": P + 8}, ALIGN), ({"dstate": P + 4}, ALIGN), ({"dstate_in": P + 4}, ALIGN), ({"dbeta": P + 2}, ALIGN),
    ({"dlog_decay": P + 2}, ALIGN), ({"seq_len": P + 2}, ALIGN), ({"log_decay": None}, ARG),
    ({"dstate": P, "dstate_in": P + 16}, ARG), ({"state_in": P, "dstate_in": P}, ARG), ({"state_in": P, "dstate_in": P + 16}, ARG),
    ({"ws": None}, WORKSPACE), ({"ws_bytes": 0}, WORKSPACE), ({"fws": 256 * P, "fws_bytes": 16}, WORKSPACE),
    ({"fws": 256 * P + 16, "fws_bytes": BIG}, ALIGN), ({"fws": 256 * P, "fws_bytes": BIG}, ARG),
    ({"fws": 256 * P + 256, "fws_bytes": BIG}, ARG)])
def test_backward(lib, change, status):
    assert refused(lib, "cottn_bwd_causal_delta", BWD, change, status)


def test_a_forward_alones_workspace_is_no_backwards(lib):
    size = lib.cottn_workspace_bytes_dkdv
    alone, whole = (size(op, 2, 3, 100, 64, 64, 0, 1) for op in (ALONE_OP, FWD_OP))
    assert 0 < alone < whole
    assert refused(lib, "cottn_bwd_causal_delta", BWD, {"fws": 512 * P, "fws_bytes": alone}, WORKSPACE)
    # up to the end of the forward's workspace the two must not share a byte
    assert refused(lib, "cottn_bwd_causal_delta", BWD, {"fws": 256 * P - whole + 256, "fws_bytes": whole}, ARG)


@pytest.mark.parametrize("change,status", COMMON + [({k: None}, NULL) for k in ("q", "k", "v", "s", "beta", "state_in", "state", "o")] + [
    ({"B_in": 3}, SHAPE), ({"B_in": 0, "parent": P}, SHAPE), ({"parent": P + 2}, ALIGN), ({"state_in": P + 8}, ALIGN),
    ({"parent": P}, ARG), ({"state_in": P + 16}, ARG), ({"parent": P, "B_in": 9, "state_in": P, "state": P + 8 * 3 * 64 * 64 * 4}, ARG),
    ({"B": 1 << 12, "H": 1 << 12, "B_in": 1 << 12}, SHAPE)])
def test_step(lib, change, status):
    assert refused(lib, "cottn_step_delta", STEP, change, status)


ROWS = 2 * 3 * 100 * 64 * 2


@pytest.mark.parametrize("change,status", [({k: None}, NULL) for k in ("Q", "K", "Kr", "Qr", "positions", "freq")] + [
    ({"d": 48}, SHAPE), ({"B": 0}, SHAPE), ({"H": -1}, SHAPE), ({"N": -1}, SHAPE), ({"dtype": 3}, DTYPE), ({"pairs": 0}, SHAPE),
    ({"pairs": 33}, SHAPE), ({"axes": 0}, SHAPE), ({"Q": P + 8}, ALIGN), ({"Kr": 4 * P + 2}, ALIGN), ({"positions": P + 2}, ALIGN),
    ({"freq": P + 1}, ALIGN), ({"axis": P + 2}, ALIGN),
    ({"Qr": 2 * P}, ARG), ({"Kr": P}, ARG), ({"Kr": 3 * P}, ARG), ({"Qr": P + 16}, ARG), ({"Qr": P + ROWS - 16}, ARG),
    ({"Kr": 3 * P + ROWS - 16}, ARG), ({"K": P, "Qr": P}, ARG), ({"B": 1 << 24, "H": 1, "N": 1}, SHAPE),
    ({"N": 0}, OK), ({"N": 0, "Q": None, "K": None, "Qr": None, "Kr": None, "positions": None}, OK)])
def test_rotary(lib, change, status):
    assert refused(lib, "cottn_rotary", ROTARY, change, status)


def test_sizes(lib):
    size, segments = lib.cottn_workspace_bytes_dkdv, lib.cottn_segments_dkdv
    record, w = 2384, 6 * 3 * 1024
    for dtype in (0, 1, 2):
        chunks = 16
        lib.cottn_tune_segments(1)
        per = 6 * chunks   # chunks of all units
        alone = per * (record + w)
        assert alone % 256 == 0
        whole = alone + per * (w + 64 * 32 * 4 + 64 * 32 * 4)
        saved = per * (64 * 32 * 4 + 64 * 32 * 4) + 512   # (one partial sum of ds to a chunk, 384 bytes)
        assert [size(op, 2, 3, 1000, 64, 32, 0, dtype) for op in (ALONE_OP, FWD_OP, SAVED_OP, BWD_OP)] == [alone, whole, saved, whole + saved]
        lib.cottn_tune_segments(5)
        assert segments(FWD_OP, 2, 3, 1000, 64, 32, 0, dtype) == 4   # of 4 chunks each
        more = 6 * 4 * 64 * 32 * 4
        assert size(ALONE_OP, 2, 3, 1000, 64, 32, 0, dtype) == alone + more + 6 * 4 * 64 * 64 * 4
        assert size(SAVED_OP, 2, 3, 1000, 64, 32, 0, dtype) == saved + more
        lib.cottn_tune_segments(0)
        for op in (FWD_OP, ALONE_OP, BWD_OP, SAVED_OP):
            assert size(op, 2, 3, 1000, 64, 32, 128, dtype) == size(op, 2, 3, 1000, 64, 48, 0, dtype) == NO_SIZE
            assert size(op, 2, 3, 1000, 64, 32, 64, dtype) == size(op, 2, 3, 1000, 64, 32, 0, dtype)
            assert segments(op, 2, 3, 1000, 64, 32, 128, dtype) == 0
            assert size(op, 2, 3, 0, 64, 32, 0, dtype) == 0
            assert size(op, 1 << 12, 1 << 12, 65, 64, 32, 0, dtype) == NO_SIZE
            assert size(op, 2, 3, 1000, 64, 32, 0, 3) == NO_SIZE
    # one sequence of few heads is cut, a full chip is not
    assert segments(FWD_OP, 1, 8, 32768, 64, 64, 0, 1) > 1
    assert segments(FWD_OP, 1, 8, 32768, 128, 64, 0, 0) > 1 and segments(FWD_OP, 32, 16, 2048, 64, 64, 0, 1) == 1


def test_a_library_without_them(tmp_path):
    """binding.py beside a libcottn.so that was built before these calls."""
    names = ["cottn_fwd_causal_delta", "cottn_bwd_causal_delta", "cottn_step_delta", "cottn_rotary"]
    before, older.LATER = older.LATER, names
    try:
        older.test_it_imports_and_makes_the_calls_that_are_there(tmp_path)
    finally:
        older.LATER = before


def test_arguments_are_checked_first():
    """By binding.py, on host tensors: the wrong ones are named before the GPU is asked for."""
    import torch
    import paper_2409_18747_amd.binding as b
    x = torch.zeros(2, 3, 8, 64)
    at, freq = torch.zeros(2, 8, dtype=torch.int32), torch.ones(32)
    for wrong, says in ((dict(positions=at[:, :7].contiguous()), "positions"), (dict(positions=at.long()), "positions"),
                        (dict(positions=at[0]), "positions"), (dict(freq=freq[None]), "freq"), (dict(freq=freq.double()), "freq"),
                        (dict(axis=torch.zeros(31, dtype=torch.int32)), "axis"), (dict(K=x[:, :2]), "K"), (dict(Qr=x.half()), "Qr"),
                        (dict(K=None, Kr=x), "Kr needs K"), (dict(Q=x[0]), "rows must be"), ({}, "must live on the GPU")):
        with pytest.raises((ValueError, TypeError), match=says):
            b.cottn_rotary(**{**dict(Q=x, K=x, positions=at, freq=freq), **wrong})
    t, gate, S = torch.zeros(2, 3, 64), torch.zeros(2, 3), torch.zeros(2, 3, 64, 64)
    for wrong, says in ((dict(beta=gate[:1]), "beta"), (dict(log_decay=gate.double()), "log_decay"), (dict(state=S[:1]), "state"),
                        (dict(parent=torch.zeros(2, dtype=torch.int32)), "parent needs state_in"), (dict(k=t[:, :2]), "k"),
                        (dict(s=torch.ones(2)), "s"), ({}, "must live on the GPU")):
        with pytest.raises((ValueError, TypeError), match=says):
            b.cottn_step_delta(**{**dict(q=t, k=t, v=t, s=torch.ones(3), log_decay=gate, beta=gate, state=S), **wrong})
    gates = torch.zeros(2, 3, 8)
    base = dict(Q=x, K=x, V=x, s=torch.ones(3), log_decay=gates, beta=gates)
    for wrong, says in ((dict(beta=gates[:, :2]), "beta"), (dict(log_decay=gates.half()), "log_decay"), (dict(V=x[:, :, :7]), "V"),
                        (dict(state=S[:1]), "state"), (dict(seq_len=torch.zeros(2, dtype=torch.int32)), "s must"),
                        ({}, "must live on the GPU")):
        with pytest.raises((ValueError, TypeError), match=says):
            b.cottn_fwd_causal_delta(**{**base, **wrong})
        with pytest.raises((ValueError, TypeError), match=says.replace("state", "state_in")):
            b.cottn_bwd_causal_delta(**{**base, **{("state_in" if n == "state" else n): t for n, t in wrong.items()}, "dO": wrong.get("V", x)})
