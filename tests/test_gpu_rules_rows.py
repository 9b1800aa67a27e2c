"""graft_logits_adjust where a workgroup takes several rows of a sequence (2, 4 and 8 of them), and where the logits pass the caches: bit for bit
against plain numpy.  What a workgroup takes follows from the constants in the kernel's source, which are read here."""
import os
import re

import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from rules_util import adjusted
from test_gpu_rules import _case, _gpu, same, up

pytestmark = pytest.mark.gpu

SOURCE = open(os.path.join(os.path.dirname(graft.__file__), "csrc", "logits_adjust.hip")).read()
THREADS, QUADS, ROWS, FILL = (int(re.search(x + r" = (\d+)", SOURCE).group(1)) for x in ("LA_THREADS", "LA_QUADS", "LA_ROWS", "LA_FILL"))


def plan(B, K, V):
    """(columns of a block, rows of a workgroup)."""
    quads = QUADS
    blocks = -(-V // (4 * THREADS * quads))
    if blocks * B * K < FILL:
        quads, blocks = 1, -(-V // (4 * THREADS))
    rows = 1
    while rows < ROWS and 2 * rows <= K and blocks * B * K // (2 * rows) >= FILL:
        rows *= 2
    return 4 * THREADS * quads, rows


ENDS = [48, 47, 33, 1, 8, 9, 17, 16, 7, 15, 2, 40]                # trees that end at, in front of and behind a workgroup's rows


def _check(c, rows_per, special=()):
    B, K, V = c["logits"].shape
    assert plan(B, K, V) == (4 * THREADS * QUADS, rows_per)
    want, ids, st = adjusted(**c)
    gpu = _gpu(c)
    for write in ("none", "apart", "in place"):
        result = None if write == "none" else gpu["logits"] if write == "in place" else gpu["logits"].clone()
        got = graft.graft_logits_adjust(**gpu, result=result)
        assert (got["status"].cpu().numpy() == st).all() and (got["target_ids"].cpu().numpy() == ids).all(), write
        if write == "apart":
            assert same(gpu["logits"].cpu().numpy(), c["logits"])              # (as they were)
        if result is not None:
            assert same(result.cpu().numpy(), want), write


@pytest.mark.parametrize("B,K,V,rows_per,options", [
    (12, 48, 9001, 2, dict(bias=1, states=5)), (12, 48, 20480, 4, dict(bias=2, states=7)), (12, 48, 30011, 8, dict(bias=1)),
    (12, 48, 30011, 8, dict(states=40, params="r")), (12, 48, 30010, 8, dict(bias=2, states=3, params="fp")), (12, 48, 30009, 8, dict(params="", bias=1, states=9)),
    (12, 48, 30012, 8, dict(paths=False, states=6)), (12, 48, 32768, 8, dict(counts=False, bias=1)),
])
def test_several_rows_a_workgroup(B, K, V, rows_per, options):
    c = _case(V + rows_per, B, K, V, n=ENDS, **options)
    _check(c, rows_per)


def test_trees_of_128_nodes_and_three():
    _check(_case(61, 5, 128, 30011, n=[128, 127, 121, 65, 3], bias=1, states=11), 8)
    _check(_case(62, 300, 3, 9001, n=[1 + i % 3 for i in range(300)], bias=1, states=4), 2)     # no more rows than a tree has


def test_values_that_are_no_numbers_among_several_rows():
    """Rows of NaN, infinities, equal maxima and the like beside ordinary ones of the same workgroup; trees that are none."""
    c = _case(63, 12, 48, 30011, n=ENDS[:9] + [0, 49, 40], bias=1, states=5, special=True)
    c["allow_index"][0, 9], c["allow_index"][1, 30], c["allow_index"][2, 40] = 5, -2, 99            # (the last one is padding)
    c["repetition"][5], c["frequency"][6], c["presence"][7], c["repetition"][8] = 0.0, np.inf, np.nan, np.nan
    c["tokens"][0, 4], c["tokens"][1, 5] = -1, 30011
    _check(c, 8)
    assert list(adjusted(**c)[2][:2]) == [1, 1]


def test_rows_of_any_address_among_several():
    c = _case(64, 12, 48, 30011, n=ENDS, bias=2, states=3)
    want, ids, _ = adjusted(**c)
    gpu = _gpu(c)
    for x in ("logits", "counts", "bias", "allow"):
        base = torch.empty(gpu[x].numel() + 1, dtype=gpu[x].dtype, device="cuda")
        base[1:] = gpu[x].flatten()
        gpu[x] = base[1:].view(gpu[x].shape)
    for shift in (1, 2, 3):
        result = torch.empty(want.size + shift, device="cuda")[shift:].view(want.shape)
        result.copy_(gpu["logits"])
        got = graft.graft_logits_adjust(**gpu, result=result)
        assert same(result.cpu().numpy(), want) and (got["target_ids"].cpu().numpy() == ids).all()


@pytest.mark.parametrize("params", ["rfp", ""])
def test_logits_past_the_caches(params):
    """233 MB of logits, which are read past the caches; the rows are the same few, so that the reference takes no longer than they do."""
    B, K, V = 8, 48, 151937
    assert B * K * V * 4 > 208 << 20 and plan(B, K, V)[1] == 8
    small = _case(65, 1, 48, V, n=[48], bias=1, states=5, params=params)
    want, ids, _ = adjusted(**small)
    n = [48, 48, 41, 40, 39, 8, 1, 48]
    big = {k: (x if k in ("bias", "allow") else np.repeat(x, B, 0)) for k, x in small.items()}
    big["n_nodes"] = np.array(n, np.int32)
    gpu = {k: up(x.view(np.int64) if k == "mask" else x) for k, x in big.items()}
    for write in ("none", "apart", "in place"):
        result = None if write == "none" else gpu["logits"] if write == "in place" else gpu["logits"].clone()
        got = graft.graft_logits_adjust(**gpu, result=result)
        for b in range(B):
            # (a node's history is its own path: what lies behind a tree's end changes nothing in front)
            live = [i for i in range(n[b])]
            assert (got["target_ids"][b].cpu().numpy() == np.where(np.arange(K) < n[b], ids[0], -1)).all()
            if result is not None:
                out = result[b].cpu().numpy()
                assert same(out[live], want[0, live]) and same(out[n[b]:], big["logits"][b, n[b]:])
