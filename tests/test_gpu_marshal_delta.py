"""The C++ marshalling of the calls by the gated delta rule and of rotary positions, as test_gpu_marshal_decay has it of the calls
with a decay: what it must not take, that it lets other threads run, that it gives what the ctypes calls give, and that a library
without these functions leaves them to ctypes."""
import pytest

import test_gpu_marshal_decay as others
from test_gpu_marshal_refusals import BYTES, LENGTHS, NARROW, PER_HEAD, PER_UNIT, ROW, STATE_DKDV, TAKEN, TOKEN, WIDE, good, wrong_alike, wrongs
from test_gpu_marshal_threads import LAUNCHES

pytestmark = pytest.mark.gpu

MORE = others.MORE + ["fwd_causal_delta", "bwd_causal_delta", "step_delta", "rotary"]
B, H, N = ROW[1][:3]
GATES = ("floats", (B, H, N))
cottn = others.cottn


def calls():
    first = {"Q": ROW, "K": ROW, "V": WIDE}
    gates = {"log_decay": GATES, "beta": GATES}
    grads = {"dQ": ROW, "dK": ROW, "dV": WIDE}
    tokens = {"q": TOKEN, "k": TOKEN, "v": NARROW, "s": PER_HEAD, "log_decay": PER_UNIT, "beta": PER_UNIT, "state": STATE_DKDV, "o": NARROW}
    turned = {"Q": ROW, "K": ROW, "positions": ("lengths", (B, N, 2)), "freq": ("floats", (20,)), "axis": ("lengths", (20,))}
    return {
        "cottn_fwd_causal_delta": ("fwd_delta", {**first, "s": PER_HEAD, **gates, "state_in": STATE_DKDV, "O": WIDE, "state": STATE_DKDV,
                                                 "workspace": BYTES}),
        "cottn_fwd_causal_delta padded": ("fwd_delta", {**first, "s": PER_UNIT, **gates, "seq_len": LENGTHS, "O": WIDE}),
        "cottn_bwd_causal_delta": ("bwd_delta", {**first, "s": PER_HEAD, **gates, "dO": WIDE, "state_in": STATE_DKDV, "dstate": STATE_DKDV,
                                                 "dstate_in": STATE_DKDV, **grads, "ds": PER_HEAD, "dlog_decay": GATES, "dbeta": GATES,
                                                 "fwd_workspace": BYTES, "workspace": BYTES}),
        "cottn_bwd_causal_delta padded": ("bwd_delta", {**first, "s": PER_UNIT, **gates, "seq_len": LENGTHS, "dO": WIDE, "ds": PER_UNIT}),
        "cottn_step_delta": ("step_delta", tokens),
        "cottn_step_delta beams": ("step_delta", {**tokens, "state_in": STATE_DKDV, "parent": LENGTHS}),
        "cottn_rotary": ("rotary", {**turned, "Qr": ROW, "Kr": ROW}),
        "cottn_rotary of one": ("rotary", {"Q": ROW, "positions": ("lengths", (B, N)), "freq": ("floats", (32,))}),
    }


GIVEN = {"cottn_rotary of one": {"K": None}}


@pytest.fixture(scope="module")
def stand_ins(tmp_path_factory):
    return others.library(tmp_path_factory.mktemp("stand_ins"), LAUNCHES + MORE, TAKEN)


@pytest.mark.parametrize("call", sorted(calls()))
def test_refused(cottn, call):
    import torch
    function, specs = calls()[call]
    name = call.split()[0]
    arguments = {n: good(torch, spec) for n, spec in specs.items()}
    more = GIVEN.get(call, {})
    with pytest.raises(cottn.CottnError) as e:
        getattr(cottn, name)(**arguments, **more)
    assert e.value.status == TAKEN   # all right: the C++ half makes the call
    tries = [("%s: %s" % (n, what), {**arguments, n: wrong})
             for n, spec in specs.items() for what, wrong in wrongs(torch, "_dkdv", n, spec)
             if not (n == "freq" and "element" in what)]   # (its length is the number of pairs; where it should not fit axis, axis is tried)
    if "V" in specs or "v" in specs:
        tries += wrong_alike(torch, "_dkdv", arguments, specs)
    taken = []
    for what, wrong in tries:
        del cottn.answers[:]
        try:
            getattr(cottn, name)(**wrong, **more)
        except (ValueError, TypeError):
            if cottn.answers == [(function, False)]:
                continue
        except (cottn.CottnError, AssertionError):
            pass
        taken.append(what)
    assert not taken


def test_what_needs_another(cottn):
    import torch
    function, specs = calls()["cottn_step_delta beams"]
    with pytest.raises(ValueError):
        cottn.cottn_step_delta(**{n: good(torch, spec) for n, spec in specs.items() if n != "state_in"})
    function, specs = calls()["cottn_rotary"]
    with pytest.raises(ValueError):
        cottn.cottn_rotary(**{n: good(torch, spec) for n, spec in specs.items() if n != "K"}, K=None)
    assert cottn.answers == [("step_delta", False), ("rotary", False)]


def real_arguments(torch, call):
    g = torch.Generator(device="cuda").manual_seed(3)
    out = dict(GIVEN.get(call, {}))
    for n, (kind, shape) in calls()[call][1].items():
        if n in ("O", "o", "dQ", "dK", "dV", "ds", "dlog_decay", "dbeta", "workspace", "fwd_workspace", "Qr", "Kr"):
            continue
        if n == "seq_len":
            out[n] = torch.tensor([5, 8], dtype=torch.int32, device="cuda")
        elif kind == "lengths":
            out[n] = torch.randint(0, 2, shape, generator=g, device="cuda", dtype=torch.int32)
        else:
            out[n] = torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16 if kind == "rows" else torch.float32)
    if "log_decay" in out:
        out["log_decay"] = -out["log_decay"].abs()
    return out


@pytest.mark.parametrize("decays", [True, False])
@pytest.mark.parametrize("call", sorted(calls()))
def test_same_as_ctypes(call, decays, monkeypatch):
    import torch
    import paper_2409_18747_amd.binding as b
    name = call.split()[0]

    def results():
        arguments = real_arguments(torch, call)
        if not decays and "log_decay" in arguments:
            arguments["log_decay"] = None
        r = getattr(b, name)(**arguments)
        torch.cuda.synchronize()
        r = list(r) if isinstance(r, tuple) else [r]
        return r + [arguments[n] for n in ("state", "dstate_in") if n in arguments]

    mine = results()
    monkeypatch.setattr(b, "_marshal", b._NoMarshal)
    for x, y in zip(mine, results()):
        assert (x is None and y is None) or (x.shape == y.shape and x.dtype == y.dtype and torch.equal(x, y))


def test_lock_is_released(tmp_path):
    import torch
    import paper_2409_18747_amd.binding as b
    so = others.library(tmp_path, LAUNCHES + MORE, "PyGILState_Check() ? 5 : 0")
    b._marshal.bind(so, b.CottnError)
    try:
        for call in calls():
            getattr(b, call.split()[0])(**real_arguments(torch, call))
    finally:
        b._marshal.bind(b.library_path, b.CottnError)


def test_a_library_without_them(tmp_path):
    import torch
    import paper_2409_18747_amd.binding as b
    so = others.library(tmp_path, LAUNCHES + others.MORE, TAKEN)
    b._marshal.bind(so, b.CottnError)
    try:
        for call in calls():
            assert getattr(b, call.split()[0])(**real_arguments(torch, call)) is not None   # over ctypes, by the real library
            with pytest.raises(b.CottnError):
                b.cottn_scale_from_m_varlen(torch.ones(3, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda"))
    finally:
        b._marshal.bind(b.library_path, b.CottnError)
    torch.cuda.synchronize()
