"""graft_kv_compact_mx and graft_kv_gather_mx: bytes of a 4-bit cache, against plain numpy (bit for bit)."""
import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from gpu_util import dev, host
from mx_util import dequantise, element_at, read_runs, run_bytes

pytestmark = pytest.mark.gpu


def _cache(rng, layers, total, Hkv, D, gap=0):
    run = run_bytes(D) + gap
    x = rng.integers(0, 256, (layers, total, Hkv, run)).astype(np.uint8)
    return x, {"page": Hkv * run, "head": run}, total * Hkv * run


def _moved(x, D, values, table, P, path, acc):
    """The cache after the rows of each sequence's path have moved."""
    y = x.copy()
    e = element_at(D, values)
    for b in range(len(P)):
        rows = []
        for k in range(1, acc[b] + 1):
            t = P[b] + path[b, k]
            rows.append((x[:, table[b, t // 16]], t % 16))
        for k, (run, t) in enumerate(rows, 1):
            to = P[b] + k
            dst = y[:, table[b, to // 16]]
            for d in range(0, D, 2):                       # two elements to a byte, of one token in either order
                dst[..., e[to % 16, d] // 2] = run[..., e[t, d] // 2]
            for c in range(D // 32):
                dst[..., 8 * D + 16 * c + to % 16] = run[..., 8 * D + 16 * c + t]
            y[:, table[b, to // 16]] = dst
    return y


@pytest.mark.parametrize("layers,Hkv,D,P,K,accept,gap", [
    (1, 1, 64, (0,), 16, (5,), 0), (3, 8, 128, (5, 300, 17), 64, (4, 0, 9), 0), (2, 3, 128, (1000, 33), 96, (40, 1), 32), (4, 2, 64, (31, 32, 47, 48), 128, (63, 127, 17, 8), 16),
    (94, 4, 128, (100,) * 3, 48, (6, 7, 8), 0),
])
def test_compact(layers, Hkv, D, P, K, accept, gap):
    rng = np.random.default_rng(layers + D)
    B, cap = len(P), 127
    pages = (max(P) + K + 15) // 16
    total = B * pages + 2
    table = rng.permutation(total)[:B * pages].reshape(B, pages).astype(np.int32)
    k, strides, layer = _cache(rng, layers, total, Hkv, D, gap)
    v = _cache(rng, layers, total, Hkv, D, gap)[0]
    path = np.full((B, cap + 1), -1, np.int32)
    for b in range(B):
        path[b, 0] = 0
        path[b, 1:accept[b] + 1] = np.sort(rng.choice(np.arange(1, K), accept[b], replace=False))
    kd, vd = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    out = graft.graft_kv_compact_mx(kd, vd, layer, layers, strides, dev(table), dev(P), dev(path), dev(accept), K, Hkv, D)
    assert (host(out["status"]) == 0).all() and (host(out["new_prefix_len"]) == np.array(P) + accept + 1).all()
    assert (kd.cpu().numpy() == _moved(k, D, False, table, P, path, accept)).all()
    assert (vd.cpu().numpy() == _moved(v, D, True, table, P, path, accept)).all()


def test_compact_refuses_a_sequence():
    rng = np.random.default_rng(1)
    B, K, Hkv, D, pages = 6, 24, 2, 128, 3
    table = rng.permutation(B * pages).reshape(B, pages).astype(np.int32)
    k, strides, layer = _cache(rng, 2, B * pages, Hkv, D)
    kd, vd = torch.from_numpy(k).cuda(), torch.from_numpy(k).cuda()
    path = np.tile(np.array([0, 5, 9, 11, -1], np.int32), (B, 1))
    P, acc = np.array([9, 9, 9, -1, 40, 9], np.int32), np.array([3, 3, 5, 1, 3, -1], np.int32)
    path[0, 2], path[1, 0] = 5, 1
    out = graft.graft_kv_compact_mx(kd, vd, layer, 2, strides, dev(table), dev(P), dev(path), dev(acc), K, Hkv, D)
    assert host(out["status"]).tolist() == [2, 2, 1, 1, 1, 1] and (host(out["new_prefix_len"]) == P).all()
    assert (kd.cpu().numpy() == k).all() and (vd.cpu().numpy() == k).all()


@pytest.mark.parametrize("layers,B,T,Hkv,D", [(1, 1, 1, 1, 64), (3, 4, 33, 3, 128), (2, 3, 130, 8, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gather(layers, B, T, Hkv, D, dtype):
    rng = np.random.default_rng(T)
    pages = 12
    table = rng.permutation(B * pages + 1)[:B * pages].reshape(B, pages).astype(np.int32)
    k, strides, layer = _cache(rng, layers, B * pages + 1, Hkv, D, 16)
    k[..., 8 * D:] = np.where(rng.random(k[..., 8 * D:].shape) < 0.02, 255, 2 + k[..., 8 * D:] % 251)
    v = k[::-1, ::-1].copy()
    start, count = rng.integers(0, 40, B).astype(np.int32), rng.integers(0, T + 1, B).astype(np.int32)
    count[0] = T
    kd, vd = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    for s in (start, None):
        out = graft.graft_kv_gather_mx(kd, vd, layer, layers, strides, dev(table), dev(s), dev(count), T, Hkv, D, dtype=dtype)
        assert (host(out["status"]) == 0).all()
        for name, x in (("k", k), ("v", v)):
            got = out[name].double().cpu().numpy()
            for b in range(B):
                t = np.arange(count[b]) + (s[b] if s is not None else 0)
                code, byte = read_runs(x[..., :17 * D // 2], D, name == "v")
                want = dequantise(code, byte)[:, table[b, t // 16], :, t % 16]         # [count, layers, Hkv, D]
                assert np.array_equal(got[:, b, :count[b]], np.moveaxis(want, 0, 1), equal_nan=True)
                assert (got[:, b, count[b]:] == 0).all()


def test_gather_out_of_range():
    cache = torch.full((8, 1, 544), 0x77, dtype=torch.uint8, device="cuda")
    table = dev(np.arange(8).reshape(4, 2))
    out = graft.graft_kv_gather_mx(cache, cache, 0, 1, {"page": 544, "head": 544}, table, dev([-1, 30, 0, 0]), dev([1, 3, 5, -1]), 4, 1, 64)
    assert host(out["status"]).tolist() == [1, 1, 1, 1] and bool((out["k"] == 0).all()) and bool((out["v"] == 0).all())
