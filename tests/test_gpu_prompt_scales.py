"""graft_prompt_attn with scales of zero and next to it: every score is 0 (or nearly), a row the mean of the values that it sees."""
import numpy as np
import pytest
import torch

from prompt_util import call, check, make

pytestmark = pytest.mark.gpu

# Tiles of 32, 64 and 256 rows in bf16, of 16, 32 and 128 in fp32; keys in splits and not; groups of three; a sequence without tokens.
SHAPES = [
    ("bf16", 1, 1, 8, 2, 128, 0, None), ("bf16", 2, 1, 16, 1, 64, [777, 64], None), ("bf16", 1, 7, 8, 2, 128, 3000, None), ("bf16", 2, 40, 8, 2, 128, [333, 20], [40, 0]),
    ("bf16", 1, 12, 6, 2, 64, 100, None), ("bf16", 1, 300, 6, 2, 128, 100, None), ("bf16", 2, 300, 4, 2, 64, [700, 31], [300, 77]),
    ("f32", 1, 1, 8, 2, 64, 255, None), ("f32", 2, 3, 8, 2, 128, [700, 0], None), ("f32", 1, 9, 6, 2, 64, 300, None), ("f32", 2, 90, 8, 2, 128, [77, 300], [90, 50]),
]


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,P,n", SHAPES)
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45, 1e-40, -1e-40])
@pytest.mark.parametrize("window,cap", [(0, 0.0), (70, 0.0), (1, 0.0), (0, 5.0), (70, 1024.0)])
def test_scales_of_nothing(dtype, B, T, Hq, Hkv, D, P, n, scale, window, cap):
    c = dict(make(B + T, dtype, B, T, Hq, Hkv, D, P, n), scale=scale)
    check(c, call(c, window, cap), window, cap)


# 0 times an infinite or undefined product is no number for the rows that see the key, and nothing to the others.
@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,P,n", [x for x in SHAPES if x[1] == 1])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("window", [0, 70])
def test_scale_of_zero_and_keys_that_are_no_numbers(dtype, B, T, Hq, Hkv, D, P, n, bad, window):
    c = dict(make(B + T, dtype, B, T, Hq, Hkv, D, P, n), scale=0.0)
    clean = call(c, window).float().cpu()
    G, at = Hq // Hkv, sorted({P // 2, P + T // 2})
    d = dict(c, k=c["k"].clone())
    for t in at:
        d["k"][d["table"][0, t // 16], 1, t % 16, 5] = bad
    got = call(d, window).float().cpu()
    assert torch.equal(got[:, :, :G], clean[:, :, :G])
    for i in range(T):
        sees = any(t <= P + i and (not window or t > P + i - window) for t in at)
        row = got[0, i, G:]
        assert bool(torch.isnan(row).all()) if sees else torch.equal(row, clean[0, i, G:]), i
