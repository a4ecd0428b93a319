"""The operators' plans and the package's names, on the host."""
import copy
import ctypes
import pickle
import subprocess
import sys

import pytest

from conftest import ROOT


def plan(r):
    """What the library would read at the address that a call passes."""
    from paper_2511_22009_amd import binding
    s = r._struct
    assert r._address == ctypes.addressof(s)
    at = binding._Rope.from_address(ctypes.addressof(s))
    return at.axes, tuple(at.dims), at.layout, at.spread, at.theta


@pytest.mark.parametrize("way", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r)),
                                 lambda r: copy.deepcopy({"rotary": [r]})["rotary"][0]], ids=["copy", "deepcopy", "pickle", "nested"])
def test_copies_of_a_plan_have_memory_of_their_own(way):
    """A plan's address goes to the library, so a copy passes its own, which lives as long as it."""
    pytest.importorskip("torch")
    from paper_2511_22009_amd import Rotary
    r = Rotary((16, 24, 0), theta=500.0, layout="axis_halves", spread=True)
    c = way(r)
    assert (c.dims, c.theta, c.layout, c.spread) == (r.dims, r.theta, r.layout, r.spread)
    want = plan(r)
    assert c._address != r._address
    del r
    assert plan(c) == want
