"""graft_kv_append and graft_kv_append_mx with many tokens (768 and more of D = 128, 1536 of D = 64), which are dealt out another way than few."""
import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
import test_gpu_kv_append as few
from gpu_util import dev, host
from mx_util import read_runs

pytestmark = pytest.mark.gpu

APPENDS = [  # dtype, B, T, Hq, Hkv, D, R, P, interleaved, layout: odd numbers of tokens and of rows, every rotation, one token of many sequences
    ("f32", 3, 515, 3, 2, 64, 64, 5, False, "head"), ("bf16", 1, 771, 32, 8, 128, 128, 100, False, "head"), ("bf16", 97, 17, 16, 1, 64, 16, 31, False, "token"),
    ("f32", 2, 389, 3, 3, 128, 64, 15, True, "gap"), ("bf16", 780, 1, 7, 2, 128, 96, 9, False, "head"), ("bf16", 2, 801, 1, 1, 64, 0, 0, True, "token"),
    ("bf16", 195, 4, 5, 5, 128, 48, 3, True, "head"),
]


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,R,P,interleaved,layout", APPENDS)
@pytest.mark.parametrize("fused", [True, False])
def test_append(dtype, B, T, Hq, Hkv, D, R, P, interleaved, layout, fused):
    assert B * T * D >= 768 * 128
    few.test_append(dtype, B, T, Hq, Hkv, D, R, P, interleaved, layout, fused)


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,R,P,interleaved", [x[:9] for x in APPENDS])
def test_append_mx(dtype, B, T, Hq, Hkv, D, R, P, interleaved):
    few.test_append_mx(dtype, B, T, Hq, Hkv, D, R, P, interleaved, T >= 7)


def test_q_in_place():
    c = few._case(3, "bf16", 2, 401, 20, 2, 128, 128, 9, fused=False, tree=False)
    strides = {"page": 16 * 2 * 128, "token": 128, "head": 16 * 128}
    q, k, v = (x.contiguous() for x in c["gpu"])
    angles, place = dev(c["cos_sin"], "f32"), (dev(c["table"]), dev(c["P"]), dev(c["n"]))
    a, b = ([torch.zeros((c["total"], 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2))
    one = graft.graft_kv_append(q, k, v, angles, dev(c["pos"]), *a, strides, *place)
    keep = q.clone()
    graft.graft_kv_append(q, k, v, angles, None, *b, strides, *place, out={"q": q, "status": torch.zeros(2, dtype=torch.int32, device="cuda")})
    for i in range(2):
        n = c["n"][i]
        assert torch.equal(one["q"][i, :n], q[i, :n]) and torch.equal(q[i, n:], keep[i, n:])
    for x, y in zip(a, b):
        assert torch.equal(x, y)


@pytest.mark.parametrize("mx", [False, True])
def test_lengths_and_positions_out_of_range(mx):
    """A bad sequence stays as it was; tokens whose positions are not in the table stay out, their neighbours do not."""
    B, T, D = 4, 200, 128
    c = few._case(5, "f32", B, T, 2, 2, D, 64, [0, 1, 10, 20], lengths=[200, 4, 200, 0], tree=False)
    c["P"][1], c["n"][2] = -1, 201
    wrong = [3, 5, 64, 199]
    c["pos"][0, wrong] = [-1, c["cos_sin"].shape[0], 1 << 30, -(1 << 31)]
    if mx:
        strides, caches = {"page": 2176, "head": 1088}, [torch.full((c["total"], 2, 1088), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2)]
    else:
        strides, caches = {"page": 4096, "token": 128, "head": 2048}, [torch.full((c["total"], 2, 16, 128), -7.0, device="cuda") for _ in range(2)]
    out = {"q": torch.full((B, T, 2, D), -7.0, device="cuda"), "status": torch.full((B,), -7, dtype=torch.int32, device="cuda")}
    f = graft.graft_kv_append_mx if mx else graft.graft_kv_append
    before = [x.clone() for x in caches]
    got = f(*c["gpu"], dev(c["cos_sin"], "f32"), dev(c["pos"]), *caches, strides, dev(c["table"]), dev(c["P"]), dev(c["n"]), out=out)
    assert host(got["status"]).tolist() == [1, 1, 1, 0]
    written = [i for i in range(T) if i not in wrong]
    assert bool((got["q"][0, wrong] == -7).all()) and bool((got["q"][1:] == -7).all()) and not bool((got["q"][0, written] == -7).any())
    pages = torch.from_numpy(c["table"][0].astype(np.int64)).cuda()
    rest = torch.ones(c["total"], dtype=torch.bool, device="cuda")
    rest[pages] = False
    stay = wrong + list(range(T, len(pages) * 16))
    for cache, old, values in zip(caches, before, (False, True)):
        assert torch.equal(cache[rest], old[rest])
        for h in range(2):
            if mx:
                (code, byte), (was, _) = ([y.reshape(-1, y.shape[-1]) for y in read_runs(x[pages, h].cpu().numpy(), D, values)] for x in (cache, old))
                assert (code[stay] == was[stay]).all() and (byte[stay] == 0x5A).all() and not (byte[written] == 0x5A).any()
            else:
                rows = cache[pages, h].reshape(-1, D)
                assert bool((rows[stay] == -7).all()) and not bool((rows[written] == -7).any())
