"""Calls too large for the rotation and append (no GPU): nothing is launched."""
import pytest

import paper_2605_20104_amd as graft
from test_mx_refusals import APPEND, MX, _call, lib  # noqa: F401

SHAPE = graft.GRAFT_ERR_SHAPE


@pytest.mark.parametrize("D,T", [(128, (1 << 26) - 3), (128, 1 << 26), (64, (1 << 27) - 7), (64, 1 << 30)])
def test_more_tokens_than_a_launch_has_lanes_for(lib, D, T):  # noqa: F811
    """D / 2 lanes have a token, and a launch has fewer than 2^32 lanes."""
    none = {"a0": None, "a3": 0}                           # keys and values alone: spans of queries are another refusal
    assert _call(lib.graft_kv_append, APPEND, **none, a4=256, a5=256, a13=4096, a14=128, a15=2048, a21=T, a22=0, a24=D, a27=None) == SHAPE
    assert _call(lib.graft_kv_append_mx, MX, **none, a4=256, a5=256, a13=2 * 1088, a14=1088, a20=T, a21=0, a23=D, a26=None) == SHAPE
