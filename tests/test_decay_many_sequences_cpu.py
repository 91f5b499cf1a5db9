"""How many sequences the calls with a decay and the tree calls take: one too many is refused before anything is enqueued, without a
GPU."""
import pytest

from test_decay_boundary_cpu import ACCEPT, BWD, FWD, SHAPE, STEP, TREE, lib, refused   # noqa: F401

CALLS = [("cottn_fwd_causal_decay", FWD, 1 << 23), ("cottn_bwd_causal_decay", BWD, 1 << 23), ("cottn_step_decay", STEP, 1 << 24),
         ("cottn_tree", TREE, 1 << 23), ("cottn_tree_accept", ACCEPT, 1 << 24)]


@pytest.mark.parametrize("name,base,units", CALLS)
def test_one_too_many(lib, name, base, units):   # noqa: F811
    change = {"B": units // 4, "H": 4, "dk": 32, "dv": 32}
    if "N" in base:
        change["N"] = 1
    if "B_in" in base:
        change["B_in"] = change["B"]
    assert refused(lib, name, base, change, SHAPE)


@pytest.mark.parametrize("op", [5, 6, 8])
def test_sizes_of_workspaces(lib, op):   # noqa: F811
    size = lib.cottn_workspace_bytes_dkdv
    assert size(op, 1 << 21, 4, 1, 32, 32, 0, 1) == (1 << 64) - 1
    assert size(op, (1 << 21) - 1, 4, 1, 32, 32, 0, 1) < 1 << 63
