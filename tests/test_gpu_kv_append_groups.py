"""graft_kv_append and graft_kv_append_mx of large batches of one to a few tokens, which fill a wavefront's groups of lanes or do not."""
import pytest

import test_gpu_kv_append as few

pytestmark = pytest.mark.gpu

BATCHES = [  # dtype, B, T, Hq, Hkv, D, R, P, interleaved, layout
    ("bf16", 1100, 1, 6, 2, 128, 128, 7, False, "head"), ("f32", 800, 1, 2, 1, 64, 32, 15, True, "token"), ("bf16", 1600, 1, 3, 1, 64, 64, 16, False, "gap"),
    ("bf16", 400, 2, 5, 2, 128, 64, 3, False, "head"), ("bf16", 530, 3, 1, 3, 64, 16, 1, False, "head"), ("f32", 400, 4, 3, 1, 64, 64, 30, False, "token"),
]


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,R,P,interleaved,layout", BATCHES)
def test_append(dtype, B, T, Hq, Hkv, D, R, P, interleaved, layout):
    few.test_append(dtype, B, T, Hq, Hkv, D, R, P, interleaved, layout, True)


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,R,P,interleaved", [x[:9] for x in BATCHES])
def test_append_mx(dtype, B, T, Hq, Hkv, D, R, P, interleaved):
    few.test_append_mx(dtype, B, T, Hq, Hkv, D, R, P, interleaved, False)
