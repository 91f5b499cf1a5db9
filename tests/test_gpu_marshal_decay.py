"""The C++ marshalling of the calls with a decay and of the tree calls: what it must not take (as in test_gpu_marshal_refusals, with
stand-ins for the library, so that nothing is launched), that it lets other threads run, that it gives what the ctypes calls
give, and that a library without these functions leaves them to ctypes."""
import subprocess

import pytest

from test_gpu_marshal_refusals import BYTES, LENGTHS, NARROW, PER_HEAD, PER_UNIT, ROW, STATE_DKDV, TAKEN, TOKEN, WIDE, good, wrong_alike, wrongs
from test_gpu_marshal_threads import LAUNCHES

pytestmark = pytest.mark.gpu

MORE = ["fwd_causal_decay", "bwd_causal_decay", "step_decay", "tree", "tree_accept"]
B, H, N = ROW[1][:3]
TREE = ("lengths", (B, N))


def calls():
    first = {"Q": ROW, "K": ROW, "V": WIDE}
    grads = {"dQ": ROW, "dK": ROW, "dV": WIDE}
    states = {"state_in": STATE_DKDV, "rev_state_in": STATE_DKDV, "rev_state_out": STATE_DKDV}
    shared = {"fwd_workspace": BYTES, "workspace": BYTES}
    tokens = {"q": TOKEN, "k": TOKEN, "v": NARROW, "s": PER_HEAD, "log_decay": PER_HEAD, "state": STATE_DKDV, "o": NARROW}
    return {
        "cottn_fwd_causal_decay": ("fwd_decay", {**first, "s": PER_HEAD, "log_decay": PER_HEAD, "state_in": STATE_DKDV, "O": WIDE,
                                                 "state": STATE_DKDV, "workspace": BYTES}),
        "cottn_fwd_causal_decay padded": ("fwd_decay", {**first, "s": PER_UNIT, "log_decay": PER_HEAD, "seq_len": LENGTHS, "O": WIDE}),
        "cottn_bwd_causal_decay": ("bwd_decay", {**first, "s": PER_HEAD, "log_decay": PER_HEAD, "dO": WIDE, **states, **grads,
                                                 "ds": PER_HEAD, **shared}),
        "cottn_bwd_causal_decay padded": ("bwd_decay", {**first, "s": PER_UNIT, "log_decay": PER_HEAD, "seq_len": LENGTHS, "dO": WIDE,
                                                        "ds": PER_UNIT}),
        "cottn_step_decay": ("step_decay", tokens),
        "cottn_step_decay beams": ("step_decay", {**tokens, "state_in": STATE_DKDV, "parent": LENGTHS}),
        "cottn_tree": ("tree", {"q": ROW, "k": ROW, "v": WIDE, "s": PER_HEAD, "state": STATE_DKDV, "parent": TREE, "log_decay": PER_HEAD,
                                "o": WIDE}),
        "cottn_tree_accept": ("tree_accept", {"k": ROW, "v": WIDE, "state": STATE_DKDV, "parent": TREE, "last": LENGTHS,
                                              "log_decay": PER_HEAD}),
    }


def library(where, names, answer):
    src, so = where / "stand_ins.cpp", where / "stand_ins.so"
    src.write_text('#include <cstddef>\nextern "C" {\nint PyGILState_Check(void);\nsize_t cottn_workspace_bytes_dkdv() { return 256; }\n'
                   + "".join("int cottn_%s() { return %s; }\n" % (n, answer) for n in names) + "}\n")
    subprocess.run(["g++", "-shared", "-fPIC", str(src), "-o", str(so)], check=True)
    return str(so)


@pytest.fixture(scope="module")
def stand_ins(tmp_path_factory):
    return library(tmp_path_factory.mktemp("stand_ins"), LAUNCHES + MORE, TAKEN)


@pytest.fixture
def cottn(stand_ins, monkeypatch):
    import paper_2409_18747_amd.binding as b
    real, marshal = b.lib, b._marshal
    answers = []

    class SizesOnly:
        def __getattr__(self, name):
            if "workspace_bytes" in name or name == "cottn_status_string":
                return getattr(real, name)

            def called(*_):
                raise AssertionError("%s was called" % name)
            return called

    class Watch:
        def __getattr__(self, what):
            def through(*a):
                r = getattr(marshal, what)(*a)
                answers.append((what, r is not None))
                return r
            return through
    monkeypatch.setattr(b, "lib", SizesOnly())
    monkeypatch.setattr(b, "_marshal", Watch())
    b.answers = answers
    marshal.bind(stand_ins, b.CottnError)
    yield b
    marshal.bind(b.library_path, b.CottnError)
    del b.answers


@pytest.mark.parametrize("call", sorted(calls()))
def test_refused(cottn, call):
    import torch
    function, specs = calls()[call]
    name = call.split()[0]
    arguments = {n: good(torch, spec) for n, spec in specs.items()}
    with pytest.raises(cottn.CottnError) as e:
        getattr(cottn, name)(**arguments)
    assert e.value.status == TAKEN   # all right: the C++ half makes the call
    # ("_dkdv": widths of values are their own)
    tries = [("%s: %s" % (n, what), {**arguments, n: wrong})
             for n, spec in specs.items() for what, wrong in wrongs(torch, "_dkdv", n, spec)]
    taken = []
    for what, wrong in tries + list(wrong_alike(torch, "_dkdv", arguments, specs)):
        del cottn.answers[:]
        try:
            getattr(cottn, name)(**wrong)
        except (ValueError, TypeError):
            if cottn.answers == [(function, False)]:
                continue
        except (cottn.CottnError, AssertionError):
            pass
        taken.append(what)
    assert not taken


def test_parent_needs_states(cottn):
    import torch
    function, specs = calls()["cottn_step_decay beams"]
    arguments = {n: good(torch, spec) for n, spec in specs.items() if n != "state_in"}
    with pytest.raises(ValueError):
        cottn.cottn_step_decay(**arguments)
    assert cottn.answers == [(function, False)]


def real_arguments(torch, call):
    g = torch.Generator(device="cuda").manual_seed(3)
    out = {}
    for n, (kind, shape) in calls()[call][1].items():
        if n in ("O", "o", "dQ", "dK", "dV", "ds", "workspace", "fwd_workspace"):
            continue
        if n == "seq_len":
            out[n] = torch.tensor([5, 8], dtype=torch.int32, device="cuda")
        elif kind == "lengths":
            out[n] = torch.randint(0, 2, shape, generator=g, device="cuda", dtype=torch.int32)
        else:
            out[n] = torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16 if kind == "rows" else torch.float32)
    out["log_decay"] = -out["log_decay"].abs()
    return out


@pytest.mark.parametrize("call", sorted(calls()))
def test_same_as_ctypes(call, monkeypatch):
    import torch
    import paper_2409_18747_amd.binding as b
    name = call.split()[0]

    def results():
        arguments = real_arguments(torch, call)
        r = getattr(b, name)(**arguments)
        torch.cuda.synchronize()
        r = list(r) if isinstance(r, tuple) else [r]
        return r + [arguments[n] for n in ("state", "rev_state_out") if n in arguments]

    mine = results()
    monkeypatch.setattr(b, "_marshal", b._NoMarshal)
    for x, y in zip(mine, results()):
        assert x.shape == y.shape and x.dtype == y.dtype and torch.equal(x, y)


def test_lock_is_released(tmp_path):
    import torch
    import paper_2409_18747_amd.binding as b
    so = library(tmp_path, LAUNCHES + MORE, "PyGILState_Check() ? 5 : 0")
    b._marshal.bind(so, b.CottnError)
    try:
        for call in calls():
            getattr(b, call.split()[0])(**real_arguments(torch, call))
    finally:
        b._marshal.bind(b.library_path, b.CottnError)


def test_a_library_without_them(tmp_path):
    import torch
    import paper_2409_18747_amd.binding as b
    so = library(tmp_path, LAUNCHES, TAKEN)
    b._marshal.bind(so, b.CottnError)
    try:
        for call, (function, _) in calls().items():
            a = real_arguments(torch, call)
            assert getattr(b, call.split()[0])(**a) is not None   # over ctypes, by the real library
            with pytest.raises(b.CottnError):
                b.cottn_scale_from_m_varlen(torch.ones(3, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda"))
    finally:
        b._marshal.bind(b.library_path, b.CottnError)
    torch.cuda.synchronize()
