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
