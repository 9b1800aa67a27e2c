"""graft_tree_attn_mx where a row's scores rise by so much that what was summed before is almost nothing, but a number."""
import math

import numpy as np
import pytest
import torch

from mx_util import GRID, write_row
from test_gpu_attn_mx import _case, _check, _run

pytestmark = pytest.mark.gpu


def _keys_of(score, D):
    """Codes of a key whose first 32 elements add up to `score` halves."""
    code, grid = np.zeros(D, np.uint8), [int(2 * x) for x in GRID]
    for i in range(32):
        code[i] = max(j for j in range(8) if grid[j] <= score)
        score -= grid[code[i]]
    assert score == 0
    return code


@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 128, (2000,)), (2, 1, 8, 8, 64, (640, 3)), (2, 33, 8, 2, 128, (2100, 640)), (8, 100, 12, 4, 128, (640, 0, 64, 300, 301, 128, 303, 500))])
@pytest.mark.parametrize("wide", [0, 600])
@pytest.mark.parametrize("rise", [100, 115, 118, 120])
def test_a_maximum_that_rises_by_many_powers_of_two(shape, wide, rise):
    """Tokens of 2^11 times the first tile's maximum, too little for a lane to take another one, and behind them one of 2^rise times theirs
    whose value is zero in every other element: there the first ones' share is the result, 2^-rise and a normal number."""
    B, K, Hq, Hkv, D, P = shape
    c = _case(5, *shape, n=(K,) * B, chain=True)
    c["k"][:] = 0
    c["k"][..., 8 * D:] = 127
    c["scale"] = math.log(2.0)                             # scores in powers of two are sums of keys
    q = np.zeros((B, K, Hq, D), np.float32)
    q[..., :32] = 1
    c["q"] = torch.from_numpy(q).bfloat16()
    ones = np.full(D // 32, 127, np.uint8)
    for b in range(B):
        if P[b] < 200:
            continue
        for t, score in {70: 22, 75: 23, 97: 22, 110: 23, 130 + b: 23 + 2 * rise}.items():         # (one in each quarter of the pages)
            for g in range(Hkv):
                write_row(c["k"][c["table"][b, t // 16], g], D, False, t % 16, _keys_of(score, D), ones)
        for g in range(Hkv):
            write_row(c["v"][c["table"][b, (130 + b) // 16], g], D, True, (130 + b) % 16, np.where(np.arange(D) % 2, 0, 2).astype(np.uint8), ones)
    out = _run(dict(c, table=np.pad(c["table"], ((0, 0), (0, max(0, wide - c["table"].shape[1]))))))
    _check(c, out)
    assert bool((out[0, :, :, 1::2] != 0).any())
