"""graft_tree_attn_mx: a row's result depends on its own query and on what it sees, not on the rows that share its wavefront: neither on
what padding nodes hold nor on its neighbours' scores.  Bit for bit, since a row's rounding is to depend on nothing else either."""
import numpy as np
import pytest
import torch

from test_gpu_attn_mx import _case, _run

pytestmark = pytest.mark.gpu

# B, K, Hq, Hkv, D, P, nodes: single rows, one and two blocks of 16 rows a wavefront, keys split and not, many rows a head; blocks with
# padding rows beside live ones in each
SHAPES = [
    (2, 4, 8, 2, 64, (700, 33), (1, 3)), (2, 2, 16, 2, 128, (1500, 64), (1, 1)), (3, 40, 12, 3, 128, (900, 0, 300), (33, 7, 39)), (2, 24, 8, 2, 128, (400, 90), (24, 19)),
    (8, 100, 12, 4, 128, (700, 64, 0, 300, 301, 302, 303, 900), (99, 44, 2, 100, 6, 37, 51, 85)), (4, 128, 16, 8, 64, (600, 33, 500, 0), (127, 60, 3, 101)),
]


def _widened(c, pages):
    """The same case with a block table of more pages (the launch is planned from its width)."""
    return dict(c, table=np.pad(c["table"], ((0, 0), (0, max(0, pages - c["table"].shape[1])))))


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P,n", SHAPES)
@pytest.mark.parametrize("cap,window", [(0.0, 0), (5.0, 0), (0.0, 100), (30.0, 70)])
@pytest.mark.parametrize("wide", [0, 600, 60000])
def test_padding_queries_do_not_matter(B, K, Hq, Hkv, D, P, n, cap, window, wide):
    c = _widened(_case(B + K, B, K, Hq, Hkv, D, P, n=n, spread=1.5), wide)
    live = torch.arange(K)[None, :] < torch.tensor(n)[:, None]
    outs = []
    for filler in (0.0, 1.0, -1e30, 1e30, float("inf"), float("nan")):
        q = c["q"].clone()
        q[~live] = filler
        outs.append(_run(dict(c, q=q), cap=cap, window=window))
    for out in outs[1:]:
        assert torch.equal(out, outs[0])


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P,n", SHAPES)
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_other_rows_queries_do_not_matter(B, K, Hq, Hkv, D, P, n, cap):
    """Every third row's query is another, larger by far, or no number: the others' results stay as they are."""
    c = _case(B + K + 1, B, K, Hq, Hkv, D, P, n=n)
    clean = _run(c, cap=cap)
    rows = torch.arange(K * Hq).view(K, Hq) % 3 == 1
    for factor in (40.0, -1000.0, float("nan")):
        q = c["q"].clone()
        q[:, rows] = q[:, rows] * factor
        out = _run(dict(c, q=q), cap=cap)
        assert torch.equal(out[:, ~rows], clean[:, ~rows])
        assert not torch.equal(out, clean)
