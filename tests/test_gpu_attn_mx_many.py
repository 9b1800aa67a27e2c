"""graft_tree_attn_mx with many rows of many heads, which go another way than few: the same properties at sizes that take it."""
import math

import numpy as np
import pytest
import torch

from mx_util import attention, dequantise, read_runs
from test_gpu_attn_mx import _case, _check, _run, _sees

pytestmark = pytest.mark.gpu

SHAPES = [  # B, K, Hq, Hkv, D, P: more than 192 rows a head, and 256 tiles of 32 rows or more
    (4, 128, 16, 8, 64, (130, 33, 0, 500)), (8, 100, 12, 4, 128, (1, 15, 16, 63, 64, 65, 200, 0)), (1, 125, 65, 13, 128, (700,)), (32, 17, 16, 1, 128, tuple(range(20, 52))),
]


def _tiles(B, K, Hq, Hkv):
    rows = K * (Hq // Hkv)
    return rows > 192 and B * Hkv * ((rows + 31) // 32) >= 256


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P", SHAPES)
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_trees(B, K, Hq, Hkv, D, P, cap):
    assert _tiles(B, K, Hq, Hkv)
    c = _case(B * K + Hq, B, K, Hq, Hkv, D, P, order="head" if K % 2 else "page")
    _check(c, _run(c, cap=cap), cap=cap)


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P", SHAPES[:2])
def test_split_keys_agree(B, K, Hq, Hkv, D, P):
    c = _case(9, B, K, Hq, Hkv, D, P, capacity=320)
    _check(c, _run(c))


@pytest.mark.parametrize("window", [1, 17, 100, 1000])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_windows(window, cap):
    c = _case(window % 97, 8, 100, 12, 4, 128, (300, 0, 37, 64, 80, 129, 500, 16), capacity=300)
    _check(c, _run(c, cap=cap, window=window), cap=cap, window=window)


@pytest.mark.parametrize("window", [0, 33])
def test_chains_need_no_mask(window):
    c = _case(3, 8, 100, 12, 4, 128, (77, 0, 1500, 1, 2, 3, 4, 64), chain=True)
    one = _run(c, window=window)
    two = _run(c, window=window, mask=False, pos=False)
    assert torch.equal(one, two)
    _check(c, two, window=window)


def test_rows_without_tokens_and_few_nodes():
    """Masks of zeros, no nodes, one node, a tile of rows and one more, lengths that do not fit."""
    c = _case(4, 8, 100, 12, 4, 64, (0, 40, 0, 10, 16, 64, 300, 5), n=(100, 12, 0, 1, 33, 43, 42, 5))
    c["mask"][0, 3] = 0
    c["mask"][0, 70] = 0
    _check(c, _run(c))
    c["pos"][1, 4] += 1000
    c["mask"][1, 4] = 0
    out = _run(c, window=8)
    assert bool((out[1, 4] == 0).all())
    _check(c, out, window=8)
    for P, n in ((-1, 5), (10, 101), (10, -1), (c["table"].shape[1] * 16 - 4, 5)):
        c["P"][3], c["n"][3] = P, n
        out = _run(c)
        assert bool((out[3] == 0).all()) and bool(torch.isfinite(out).all())


def test_what_nobody_sees_does_not_matter():
    c = _case(6, 8, 100, 12, 4, 128, (100, 5, 64, 0, 1, 15, 16, 17))
    clean = _run(c)
    for b in range(8):
        P, n = int(c["P"][b]), int(c["n"][b])
        for x in (c["k"], c["v"]):
            for t in list(range(P + n, c["table"].shape[1] * 16)) + [P + n - 1]:
                x[c["table"][b, t // 16], :, 8 * 128 + np.arange(4) * 16 + t % 16] = 255
    out = _run(c)
    for b in range(8):
        n = int(c["n"][b])
        assert torch.equal(out[b, :n - 1], clean[b, :n - 1]) and bool(torch.isnan(out[b, n - 1]).all())


def test_nan_in_the_prefix_and_in_queries():
    c = _case(7, 8, 100, 12, 4, 128, (200,) * 8, n=(100,) * 8)
    clean = _run(c)
    page, at = c["table"][0, 3], 3
    c["v"][page, 1, 8 * 128 + 2 * 16 + at] = 255           # elements 64..96 of head 1's value of one token
    out = _run(c)
    bad = torch.isnan(out)
    assert bool(bad[0, :, 3:6, 64:96].all()) and int(bad.sum()) == 100 * 3 * 32
    assert torch.equal(out[~bad], clean[~bad])
    c["q"][1, 2, 1, 5] = float("inf")
    c["q"][1, 99, 3, 127] = float("nan")
    out = _run(c)
    assert bool(torch.isnan(out[1, 2, 1]).all()) and bool(torch.isnan(out[1, 99, 3]).all()) and int(torch.isnan(out[1]).sum()) == 2 * 128


@pytest.mark.parametrize("scale", [3.0, -0.5, 0.0])
def test_scales(scale):
    """Scores that leave one token, negative scales, equal weights; the running maximum moves by hundreds."""
    c = _case(11, 8, 100, 12, 4, 128, (900, 31, 0, 400, 401, 402, 3, 64), spread=3.0)
    c["scale"] = scale
    _check(c, _run(c))


@pytest.mark.parametrize("cap", [1024.0, 0.05])
@pytest.mark.parametrize("shape", [(8, 100, 12, 4, 128, (200,) * 8), (2, 5, 8, 2, 64, (700, 3))])
def test_largest_and_small_caps(shape, cap):
    c = _case(23, *shape, spread=2.0)
    _check(c, _run(c, cap=cap), cap=cap)


@pytest.mark.parametrize("K,Hq,D", [(1, 8, 128), (1, 32, 64), (8, 8, 128), (7, 6, 64), (2, 2, 128)])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_tables_with_room_for_more_than_the_caches_hold(K, Hq, D, cap):
    """Few rows a head over what may be more than 208 MB are read another way."""
    c = _case(31, 4, K, Hq, 2, D, (700, 3, 64, 1500))
    c["table"] = np.pad(c["table"], ((0, 0), (0, 26000 - c["table"].shape[1])))
    assert 2 * 26000 * 4 * 2 * (17 * D // 2) > 208 << 20
    _check(c, _run(c, cap=cap), cap=cap)
    _check(c, _run(c, cap=cap, window=50), cap=cap, window=50)


def test_error_is_that_of_two_roundings():
    """As with few rows: 2^-8 sqrt(1 / (8 ln 2)) for either of two roundings, 2.35e-3 for both."""
    c = _case(21, 1, 128, 65, 13, 128, (2048,), n=(128,))
    assert _tiles(1, 128, 65, 13)
    out = _run(c).double().cpu().numpy()
    off = size = 0.0
    for g in range(13):
        used = c["table"][0, :(2048 + 128 + 15) // 16]
        k, v = (dequantise(*read_runs(x[used, g], 128, i)).reshape(-1, 128)[:2048 + 128] for i, x in enumerate((c["k"], c["v"])))
        want, _ = attention(c["q"][0, :, g * 5:(g + 1) * 5].double().numpy(), k, v, _sees(c, 0, 0), c["scale"], 0.0)
        off += ((out[0, :, g * 5:(g + 1) * 5] - want) ** 2).sum()
        size += (want ** 2).sum()
    assert math.sqrt(off / size) < 1.06 * 2.35e-3
