"""Scale bytes of the 4-bit cache that appends do not write: the smallest, and those whose elements pass what bfloat16 holds."""
import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from gpu_util import dev, host
from mx_util import GRID, pack_runs, run_bytes
from test_gpu_attn_mx import _case, _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_as_numbers(D, dtype):
    """Every element under every scale byte that the format has finite numbers for, exactly; 255 is NaN."""
    pages, run = 16, run_bytes(D)                          # token t has scale byte t, elements 0, 1, .., 15 over and over
    code = np.arange(D) % 16
    elements = np.zeros((pages, 16, D), np.uint8) + code.astype(np.uint8)
    byte = np.broadcast_to(np.arange(256, dtype=np.uint8).reshape(16, 16, 1), (16, 16, D // 32))
    k, v = (torch.from_numpy(pack_runs(elements, byte, values)[:, None]).cuda() for values in (False, True))
    out = graft.graft_kv_gather_mx(k, v, 0, 1, {"page": run, "head": run}, dev(np.arange(pages)[None]), None, dev([256]), 256, 1, D, dtype=dtype)
    assert host(out["status"]).tolist() == [0]
    number = np.where(code & 8, -GRID[code & 7], GRID[code & 7])
    for name in ("k", "v"):
        got = out[name][0, 0, :, 0].double().cpu().numpy()
        want = number[None] * np.exp2(np.arange(253.0) - 127)[:, None]
        wrong = np.argwhere(got[:253] != want)
        assert len(wrong) == 0, (wrong[:8], sorted(set(wrong[:, 0])))
        assert np.isnan(got[255]).all()


SHAPES = [(2, 24, 6, 2, 128, (100, 5), (24, 20)), (2, 5, 8, 2, 64, (100, 37), (5, 4)), (2, 1, 8, 2, 128, (100, 64), (1, 1)),
          (8, 100, 12, 4, 128, (100, 5, 64, 0, 1, 15, 16, 17), (100,) * 8)]


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P,n", SHAPES)
@pytest.mark.parametrize("byte", [0, 1, 253, 254, 255])
def test_what_a_row_does_not_see(B, K, Hq, Hkv, D, P, n, byte):
    """Behind the last token, in a leaf that its own row alone sees, and in front of the windows: blocks of the largest elements under any
    scale byte leave every other row as it was."""
    c = _case(6, B, K, Hq, Hkv, D, P, n=n)
    clean, windowed = _run(c), _run(c, window=30)
    keep = [x.copy() for x in (c["k"], c["v"])]

    def spoil(b, t, scales):
        for x in (c["k"], c["v"]):
            x[c["table"][b, t // 16], :, 8 * D + np.arange(D // 32) * 16 + t % 16] = scales

    for b in range(B):
        last = P[b] + n[b] - 1
        for t in list(range(last + 1, c["table"].shape[1] * 16)) + ([last] if n[b] > 1 else []):
            spoil(b, t, byte)
    out = _run(c)
    for b in range(B):
        rows = n[b] - 1 if n[b] > 1 else 1
        assert torch.equal(out[b, :rows], clean[b, :rows]), (b, byte)
    c["k"][:], c["v"][:] = keep
    for t in range(100 - 30 + 1):                          # in front of every window of sequence 0
        spoil(0, t, byte)
    assert torch.equal(_run(c, window=30)[0, :n[0]], windowed[0, :n[0]])


@pytest.mark.parametrize("shape", [(2, 9, 8, 2, 128, (900, 31)), (2, 1, 8, 2, 64, (3000, 31)), (8, 100, 12, 4, 128, (900, 31, 0, 400, 401, 402, 3, 64))])
def test_large_values(shape):
    """Values of nearly 2^97 everywhere: sums of them over a prefix stay finite, whatever the scores."""
    c = _case(41, *shape, spread=3.0)
    D = shape[4]
    c["v"][..., 8 * D:] += 92
    assert c["v"][..., 8 * D:].max() == 221                # 6 * 2^(221 - 127) = 1.5 * 2^96
    out = _run(c)
    assert bool(torch.isfinite(out).all())
    _check(c, out)
