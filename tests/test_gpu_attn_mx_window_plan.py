"""graft_tree_attn_mx with a window over a table of much more room: keys are split by what the window leaves."""
import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from test_gpu_attn_mx import _case, _check, _run

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 8, 2, 128, (9000,)), (2, 17, 6, 2, 64, (6000, 33)), (8, 100, 12, 4, 128, (900, 64, 0, 300, 301, 302, 303, 500))]


def _wide(*args):
    c = _case(*args)
    return dict(c, table=np.pad(c["table"], ((0, 0), (0, 2048 - c["table"].shape[1]))))


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P", SHAPES)
@pytest.mark.parametrize("window", [1, 350, 600, 4000])
def test_a_window_over_a_wide_table(B, K, Hq, Hkv, D, P, window):
    c = _wide(window + K, B, K, Hq, Hkv, D, P)
    out = _run(c, window=window)
    _check(c, out, window=window)


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P", SHAPES[:2])
def test_no_more_splits_than_the_window_has_pages_for(B, K, Hq, Hkv, D, P):
    """A split has at least 32 pages: a window of fewer has one, and one split needs no workspace.  Many nodes' positions may lie further apart
    than there are nodes: the pages of all of them are read all the same."""
    c = _wide(3, B, K, Hq, Hkv, D, P)
    assert graft.graft_tree_attn_mx_workspace_bytes(B, K, Hq, Hkv, D, 2048) > 0
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    want = _run(c, window=400)
    assert torch.equal(_run(c, window=400, workspace=none), want)
    _check(c, want, window=400)
    with pytest.raises(graft.GraftError):
        _run(c, window=4000, workspace=none)
    if K > 1:
        c["pos"][0, 1] -= 4000
        _check(c, _run(c, window=400, workspace=none), window=400)
