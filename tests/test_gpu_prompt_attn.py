"""graft_prompt_attn against the same attention in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from prompt_util import call, check, exact, make, rows

pytestmark = pytest.mark.gpu

# (dtype, B, T, Hq, Hkv, D, P, n, layout, window, cap)
CASES = [
    ("bf16", 1, 1, 8, 2, 128, 0, None, "head", 0, 0.0),                     # the first token: sees itself
    ("bf16", 1, 1, 1, 1, 64, 0, None, "token", 0, 0.0),
    ("f32", 1, 1, 8, 2, 64, 255, None, "head", 0, 0.0),
    ("f32", 1, 1, 1, 1, 128, 0, None, "head", 0, 0.0),
    ("bf16", 2, 1, 16, 1, 128, [777, 64], None, "token", 0, 0.0),           # 16 heads a KV head, single tokens
    ("bf16", 3, 33, 4, 4, 128, [0, 15, 100], [33, 1, 0], "head", 0, 0.0),   # groups of one; a sequence without tokens
    ("bf16", 1, 257, 6, 2, 128, 0, None, "head", 0, 0.0),                   # groups of three; tiles that end inside a token
    ("bf16", 2, 130, 5, 1, 64, [31, 500], [130, 77], "gap", 0, 0.0),
    ("bf16", 1, 300, 8, 8, 64, 1000, None, "head", 0, 0.0),
    ("bf16", 1, 64, 40, 8, 128, 2048, None, "token", 0, 0.0),               # splits
    ("bf16", 2, 90, 8, 4, 128, [600, 3], [90, 64], "head", 17, 0.0),        # windows shorter than a stage, longer than all
    ("bf16", 1, 200, 4, 2, 128, 333, None, "head", 1, 0.0),
    ("bf16", 1, 200, 4, 2, 64, 333, None, "token", 2 ** 31 - 1, 0.0),
    ("bf16", 1, 400, 2, 2, 128, 100, None, "head", 128, 0.0),
    ("bf16", 1, 100, 4, 2, 128, 333, None, "head", 0, 20.0),
    ("bf16", 2, 100, 4, 2, 64, [333, 64], [100, 50], "token", 70, 50.0),
    ("bf16", 1, 300, 4, 2, 128, 1200, None, "head", 0, 8.0),                # many stages with a cap, behind and in front of partly hidden ones
    ("bf16", 1, 300, 4, 2, 64, 1200, None, "head", 640, 8.0),
    ("bf16", 1, 260, 2, 2, 128, 700, None, "head", 449, 100.0),
    ("f32", 2, 130, 6, 2, 128, [0, 77], [130, 60], "token", 0, 0.0),
    ("f32", 1, 200, 4, 1, 64, 500, None, "gap", 0, 0.0),
    ("f32", 1, 100, 4, 4, 128, 200, None, "head", 33, 0.0),
    ("f32", 1, 70, 4, 2, 64, 200, None, "head", 64, 30.0),
    ("f32", 1, 40, 16, 1, 128, 1500, None, "head", 0, 5.0),
]


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,P,n,layout,window,cap", CASES)
def test_against_64_bits(dtype, B, T, Hq, Hkv, D, P, n, layout, window, cap):
    c = make(B * 7 + T, dtype, B, T, Hq, Hkv, D, P, n, layout)
    check(c, call(c, window, cap), window, cap)


# Scores that rise as the keys go on: in steps that references follow, by more than probabilities hold, in one place, in the last stage.
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("T,P", [(1, 900), (300, 700)])
@pytest.mark.parametrize("kind", ["slow", "steps", "jump", "end", "fall", "negative scale"])
def test_rising_scores(dtype, D, T, P, kind):
    c = make(5, dtype, 1, T, 4, 2, D, P)
    n = P + T
    t = torch.arange(n, dtype=torch.float64)
    height = {"slow": t / 40, "steps": (t // 64) * 30, "jump": (t > 500) * 300.0, "end": (t > n - 20) * 200.0, "fall": -t, "negative scale": t / 10}[kind]
    # the first dim carries the height: q = 1 there, so x = scale * height + noise
    c["q"][..., 0] = 1.0
    keys = c["k"].float() * 0.1
    for s in range(c["pages"]):
        for o in range(16):
            if 16 * s + o < n:
                keys[c["table"][0, s], :, o, 0] = float(height[16 * s + o]) / c["scale"]
    c["k"] = keys.to(c["k"].dtype)
    if kind == "negative scale":
        c["scale"] = -c["scale"]
    check(c, call(c))


# What a token does not see does not reach it, whatever it is.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,window", [(1, 40), (3, 40), (100, 0), (200, 70), (200, 1)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_infinities_in_hidden_places(dtype, T, window, bad):
    P = 150
    c = make(9, dtype, 1, T, 6, 2, 128, P, T, extra_pages=1)
    clean = call(c, window).float().cpu()
    n = P + T
    at = sorted({10, P + T // 2, n - 1} if T > 3 else {10, 50})
    for which in "kv":
        d = dict(c, k=c["k"].clone(), v=c["v"].clone())
        for t in at:
            d[which][d["table"][0, t // 16], 1, t % 16, 5] = bad
        # slots behind the last token, and pages that nobody has
        d[which][d["table"][0, n // 16], :, n % 16:] = bad
        got = call(d, window).float().cpu()
        assert torch.equal(got[:, :, :3], clean[:, :, :3])                     # the other KV head
        for i in range(T):
            seen = [t for t in at if t <= P + i and (not window or t > P + i - window)]
            row = got[0, i, 3:]
            if not seen:
                assert torch.equal(row, clean[0, i, 3:]), (which, i)
            elif which == "v":
                assert not torch.isfinite(row[:, 5]).any()
                assert torch.isfinite(torch.cat([row[:, :5], row[:, 6:]], 1)).all()


# What a token does see of infinite values, in the stage of its row's first scores as elsewhere: a positive share of an infinity.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,T,window", [(0, 1, 0), (0, 3, 0), (0, 20, 0), (0, 300, 0), (150, 3, 0), (150, 3, 40), (150, 200, 70), (3000, 2, 0), (3000, 100, 0)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_infinities_in_seen_places(dtype, P, T, window, bad):
    c = make(11, dtype, 1, T, 6, 2, 128, P, T)
    clean = call(c, window).float().cpu()
    at = sorted({0, P, P + T // 2})
    d = dict(c, v=c["v"].clone())
    for t in at:
        d["v"][d["table"][0, t // 16], 1, t % 16, 5] = bad
    got = call(d, window).float().cpu()
    for i in range(T):
        if any(t <= P + i and (not window or t > P + i - window) for t in at):
            row = got[0, i, 3:, 5]
            assert bool((torch.isnan(row) if bad != bad else row == bad).all()), (i, row)
            got[0, i, 3:, 5] = clean[0, i, 3:, 5]
    check(c, got, window)


# ... and where its share is below fp32's smallest number, it is 0 times an infinity: no number, whichever split it lies in.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 20, 100])
@pytest.mark.parametrize("at", [3, 700, 1900])
@pytest.mark.parametrize("low", [1, 2000])
def test_infinities_without_weight(dtype, T, at, low):
    c = make(12, dtype, 1, T, 6, 2, 128, 3000, T)
    c["q"] = c["q"].abs()
    for t in [at] if low == 1 else range(low):                 # one token, or all of the first splits': scores of some -360, the others within 20 of 0
        c["k"][c["table"][0, t // 16], :, t % 16] = -40.0
    tok = (c["table"][0, at // 16], slice(None), at % 16)
    c["v"][tok] = 0.0
    check(c, call(c))
    c["v"][tok] = float("inf")
    assert not bool(torch.isfinite(call(c)).any())


# fp32 with few rows: on either side of 16 and 32 of a KV head, on pages that end inside a step.
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 2, 2), (1, 16, 1), (5, 6, 2), (8, 4, 2), (16, 1, 1), (17, 1, 1), (4, 32, 4), (11, 6, 2), (33, 2, 2)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P,window,cap,layout", [(0, 0, 0.0, "head"), (50, 0, 0.0, "gap"), (1001, 300, 0.0, "token"), (4000, 0, 30.0, "head"), (700, 13, 5.0, "token")])
def test_few_rows_in_fp32(T, Hq, Hkv, D, P, window, cap, layout):
    c = make(T + P, "f32", 2, T, Hq, Hkv, D, [P, P // 3], [T, max(1, T - 2)], layout)
    check(c, call(c, window, cap), window, cap)
