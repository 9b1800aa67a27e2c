"""graft_tree_attn_mx against attention in 64 bits over the numbers that the cache's elements stand for."""
import math

import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from gpu_util import dev, host
from mx_util import attention, dequantise, pack_runs, quantise, random_tree, read_runs, run_bytes, tree_mask

pytestmark = pytest.mark.gpu


def _case(seed, B, K, Hq, Hkv, D, P, n=None, capacity=None, order="page", spread=1.0, chain=False):
    rng = np.random.default_rng(seed)
    P = np.array(P, np.int32)
    n = np.array(n if n is not None else [K - (3 * b) % K for b in range(B)], np.int32)
    pages = max(capacity or 0, int((P + K).max() + 15) // 16)
    total = B * pages + 1
    table = rng.permutation(total)[:B * pages].reshape(B, pages).astype(np.int32)
    shape = (total, Hkv) if order == "page" else (Hkv, total)
    runs = [pack_runs(*quantise(spread * rng.standard_normal((*shape, 16, D)).astype(np.float32)), values) for values in (False, True)]
    run = run_bytes(D)
    strides = {"page": Hkv * run, "head": run} if order == "page" else {"page": run, "head": total * run}
    q = torch.from_numpy(rng.standard_normal((B, K, Hq, D)).astype(np.float32) * spread).bfloat16()
    mask, pos = np.zeros((B, K, 2), np.uint64), np.full((B, K), -1, np.int32)
    for b in range(B):
        parent, depth = (np.arange(n[b]) - 1, np.arange(n[b])) if chain else random_tree(rng, n[b])
        mask[b, :n[b]] = tree_mask(parent, n[b])
        pos[b, :n[b]] = P[b] + depth
    return dict(B=B, K=K, Hq=Hq, Hkv=Hkv, D=D, P=P, n=n, table=table, k=runs[0], v=runs[1], strides=strides, q=q, mask=mask, pos=pos, order=order,
                scale=1 / math.sqrt(D))


def _run(c, cap=0.0, window=0, mask=True, pos=True, **kw):
    return graft.graft_tree_attn_mx(c["q"].cuda(), torch.from_numpy(c["k"]).cuda(), torch.from_numpy(c["v"]).cuda(), c["strides"], dev(c["table"]), dev(c["P"]),
                                    dev(c["n"]), torch.from_numpy(c["mask"].view(np.int64)).cuda() if mask else None, c["Hkv"], c["scale"], softcap=cap, window=window,
                                    pos=dev(c["pos"]) if pos else None, **kw)


def _sees(c, b, window):
    P, n = int(c["P"][b]), int(c["n"][b])
    bits = (c["mask"][b, :n, np.arange(n) // 64].T >> (np.arange(n) % 64).astype(np.uint64)) & np.uint64(1)
    see = np.concatenate([np.ones((n, P), bool), bits.astype(bool)], 1)
    if window:
        place = np.concatenate([np.arange(P), c["pos"][b, :n]])
        see &= c["pos"][b, :n, None].astype(np.int64) - place[None] < window
    return see


def _check(c, out, cap=0.0, window=0):
    got = out.double().cpu().numpy()
    G = c["Hq"] // c["Hkv"]
    worst = 0.0
    for b in range(c["B"]):
        P, n = int(c["P"][b]), int(c["n"][b])
        assert (got[b, n:] == 0).all()
        if n == 0:
            continue
        used, see = c["table"][b, :(P + n + 15) // 16], _sees(c, b, window)
        for g in range(c["Hkv"]):
            k, v = (dequantise(*read_runs(x[used, g] if c["order"] == "page" else x[g, used], c["D"], i)).reshape(-1, c["D"])[:P + n]
                    for i, x in enumerate((c["k"], c["v"])))
            want, tol = attention(c["q"][b, :n, g * G:(g + 1) * G].double().numpy(), k, v, see, c["scale"], cap)
            off = abs(got[b, :n, g * G:(g + 1) * G] - want)
            assert np.array_equal(np.isnan(got[b, :n, g * G:(g + 1) * G]), np.isnan(want))
            ok = np.isnan(want) | (off <= tol)
            assert ok.all(), (b, g, np.argwhere(~ok)[:4], off[~ok][:4], tol[~ok][:4])
            worst = max(worst, float(np.nanmax(off / tol)))
    return worst


SHAPES = [  # B, K, Hq, Hkv, D, P
    (1, 1, 8, 2, 64, (0,)), (1, 1, 1, 1, 128, (1,)), (2, 1, 8, 1, 128, (255, 16)), (3, 5, 6, 2, 64, (15, 16, 17)), (2, 16, 4, 4, 128, (63, 64)), (1, 17, 16, 1, 128, (500,)),
    (4, 40, 12, 3, 128, (48, 0, 47, 1000)), (2, 128, 10, 2, 64, (130, 33)), (1, 128, 16, 1, 64, (257,)), (2, 33, 16, 8, 128, (700, 650)), (1, 96, 15, 3, 128, (2000,)),
    (1, 2, 4, 2, 128, (6000,)), (3, 64, 5, 1, 128, (320, 321, 0)),
]


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P", SHAPES)
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_trees(B, K, Hq, Hkv, D, P, cap):
    c = _case(B * K + Hq, B, K, Hq, Hkv, D, P, order="head" if K % 2 else "page")
    _check(c, _run(c, cap=cap), cap=cap)


@pytest.mark.parametrize("B,K,Hq,Hkv,D,P", [SHAPES[i] for i in (0, 2, 6, 7, 10)])
def test_split_keys_agree(B, K, Hq, Hkv, D, P):
    """A block table of much more room has the keys split over workgroups, most of which find none."""
    c = _case(9, B, K, Hq, Hkv, D, P, capacity=2048)
    assert graft.graft_tree_attn_mx_workspace_bytes(B, K, Hq, Hkv, D, 2048) > 0
    _check(c, _run(c))


@pytest.mark.parametrize("window", [1, 2, 16, 17, 100, 1000, 1 << 30])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_windows(window, cap):
    c = _case(window % 97, 3, 20, 8, 2, 128, (300, 0, 37), capacity=300)
    _check(c, _run(c, cap=cap, window=window), cap=cap, window=window)


@pytest.mark.parametrize("K,window", [(1, 0), (1, 5), (7, 0), (64, 33), (128, 0)])
def test_chains_need_no_mask(K, window):
    c = _case(K, 3, K, 8, 4, 128, (77, 0, 1500), chain=True)
    one = _run(c, window=window)
    two = _run(c, window=window, mask=False, pos=False)
    assert torch.equal(one, two)
    _check(c, two, window=window)


def test_rows_without_tokens():
    """A mask of zeros without a prefix, a window that leaves nothing, no nodes, lengths that do not fit: rows of zeros."""
    c = _case(4, 4, 12, 4, 2, 64, (0, 40, 0, 10), n=(12, 12, 0, 5))
    c["mask"][0, 3] = 0
    c["mask"][0, 7] = 0
    _check(c, _run(c))
    c["pos"][1, 4] += 1000                                 # far behind everything it could see
    c["mask"][1, 4] = 0
    out = _run(c, window=8)
    assert bool((out[1, 4] == 0).all())
    _check(c, out, window=8)
    for P, n in ((-1, 5), (10, 13), (10, -1), (c["table"].shape[1] * 16 - 4, 5)):
        c["P"][3], c["n"][3] = P, n
        out = _run(c)
        assert bool((out[3] == 0).all()) and bool(torch.isfinite(out).all())


def test_what_nobody_sees_does_not_matter():
    """NaN blocks and garbage behind the last token, in tree slots that only some nodes see, and in front of the window."""
    c = _case(6, 2, 24, 6, 2, 128, (100, 5), n=(24, 20))
    clean = _run(c)
    windowed = _run(c, window=30)
    for b in range(2):
        P, n = int(c["P"][b]), int(c["n"][b])
        last = P + n - 1                                   # the last node of a tree is a leaf: seen by itself alone
        for x in (c["k"], c["v"]):
            for t in list(range(P + n, c["table"].shape[1] * 16)) + [last]:
                x[c["table"][b, t // 16], :, 8 * 128 + np.arange(4) * 16 + t % 16] = 255
    out = _run(c)
    for b in range(2):
        n = int(c["n"][b])
        assert torch.equal(out[b, :n - 1], clean[b, :n - 1]) and bool(torch.isnan(out[b, n - 1]).all())
    for t in range(100 - 30 + 1):                          # in front of every window of sequence 0
        for x in (c["k"], c["v"]):
            x[c["table"][0, t // 16], :, 8 * 128 + np.arange(4) * 16 + t % 16] = 255
    out = _run(c, window=30)
    assert torch.equal(out[0, :23], windowed[0, :23])


def test_nan_in_the_prefix_and_in_queries():
    c = _case(7, 2, 4, 4, 2, 128, (200, 200), n=(4, 4))
    clean = _run(c)
    page, at = c["table"][0, 3], 3
    c["v"][page, 1, 8 * 128 + 2 * 16 + at] = 255           # elements 64..96 of head 1's value of one token
    out = _run(c)
    bad = torch.isnan(out)
    assert bool(bad[0, :, 2:, 64:96].all()) and int(bad.sum()) == 4 * 2 * 32
    assert torch.equal(out[~bad], clean[~bad])
    c["q"][1, 2, 1, 5] = float("inf")
    c["q"][1, 3, 3, 127] = float("nan")
    out = _run(c)
    assert bool(torch.isnan(out[1, 2, 1]).all()) and bool(torch.isnan(out[1, 3, 3]).all()) and int(torch.isnan(out[1]).sum()) == 2 * 128


@pytest.mark.parametrize("scale", [3.0, -0.5, 0.0, 1e-6])
@pytest.mark.parametrize("spread", [1.0, 3.0])
def test_scales(scale, spread):
    """Scores that leave one token, negative scales, equal weights; the running maximum moves by hundreds."""
    c = _case(11, 2, 9, 8, 2, 128, (900, 31), spread=spread)
    c["scale"] = scale
    _check(c, _run(c))


def test_small_and_large_numbers():
    """Blocks of queries and cache that differ by 2^40 within a row."""
    c = _case(12, 1, 8, 4, 2, 128, (150,))
    c["q"][..., 32:64] *= 2.0 ** 20
    c["q"][..., 64:96] *= 2.0 ** -20
    for x in (c["k"], c["v"]):
        x[..., 8 * 128 + 16:8 * 128 + 32] -= 20
        x[..., 8 * 128 + 32:8 * 128 + 48] += 20
    _check(c, _run(c))


def test_long_and_far_apart():
    """A cache of more than 4 GiB, the pages at its end, and a long prefix in many splits."""
    D, Hkv = 128, 1
    c = _case(13, 1, 3, 4, 1, D, (20000,))
    pages = c["table"].shape[1]
    stride = (5 << 30) // pages // 16 * 16
    big = [torch.zeros(stride * (pages + 1) + 1088, dtype=torch.uint8, device="cuda") for _ in range(2)]
    for x, runs in zip(big, (c["k"], c["v"])):
        x[:stride * (pages + 1)].view(pages + 1, stride)[:, :1088] = torch.from_numpy(runs[:, 0]).cuda()
    out = graft.graft_tree_attn_mx(c["q"].cuda(), *big, {"page": stride, "head": 1088}, dev(c["table"]), dev(c["P"]), dev(c["n"]),
                                   torch.from_numpy(c["mask"].view(np.int64)).cuda(), 1, c["scale"])
    _check(c, out)
    assert torch.equal(out, _run(c))
    # the same rows through the other calls: read, appended again, read
    start = dev([c["table"].shape[1] * 16 - 40])
    small = [torch.from_numpy(x).cuda() for x in (c["k"], c["v"])]
    a = graft.graft_kv_gather_mx(*big, 0, 1, {"page": stride, "head": 1088}, dev(c["table"]), start, dev([40]), 40, Hkv, D)
    b = graft.graft_kv_gather_mx(*small, 0, 1, c["strides"], dev(c["table"]), start, dev([40]), 40, Hkv, D)
    assert torch.equal(a["k"], b["k"]) and torch.equal(a["v"], b["v"]) and bool((a["k"] != 0).any())
    rows = torch.randn((1, 40, 1, D), device="cuda", dtype=torch.bfloat16)
    for caches, st in ((big, {"page": stride, "head": 1088}), (small, c["strides"])):
        graft.graft_kv_append_mx(None, rows, rows, None, None, *caches, st, dev(c["table"]), start, dev([40]))
    a = graft.graft_kv_gather_mx(*big, 0, 1, {"page": stride, "head": 1088}, dev(c["table"]), start, dev([40]), 40, Hkv, D)
    b = graft.graft_kv_gather_mx(*small, 0, 1, c["strides"], dev(c["table"]), start, dev([40]), 40, Hkv, D)
    assert torch.equal(a["k"], b["k"]) and torch.equal(a["v"], b["v"])


def test_streams_and_repeats():
    """Two streams at once with a workspace each, twenty times: the same bits."""
    c = _case(14, 2, 40, 16, 4, 128, (3000, 2500))
    d = _case(15, 1, 1, 8, 8, 128, (9000,))
    want = [_run(c), _run(d)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    args = []
    for x in (c, d):
        args.append((x["q"].cuda(), torch.from_numpy(x["k"]).cuda(), torch.from_numpy(x["v"]).cuda(), x["strides"], dev(x["table"]), dev(x["P"]), dev(x["n"]),
                     torch.from_numpy(x["mask"].view(np.int64)).cuda(), x["Hkv"], x["scale"]))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i in range(2):
            outs[i].append(graft.graft_tree_attn_mx(*args[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert torch.equal(o, want[i])


@pytest.mark.parametrize("K,G", [(1, 4), (8, 4), (40, 2), (128, 5)])
def test_error_is_that_of_two_roundings(K, G):
    """Over many elements the error is that of rounding probabilities and results to bfloat16, and no more: half a step is 2^-8 / m of a
    number of mantissa m, evenly spread errors have an rms of 1 / sqrt(3) of it, and over mantissas as they occur (log-uniform) m^-2 is
    3 / (8 ln 2) on average: 2^-8 sqrt(1/3 * 3 / (8 ln 2)) = 1.66e-3 for either, 2.35e-3 for both.  A query's third part left out would
    be 3.1e-3."""
    c = _case(21, 1, K, 2 * G, 2, 128, (2048,), n=(K,))
    out = _run(c).double().cpu().numpy()
    off = size = 0.0
    for g in range(2):
        used = c["table"][0, :(2048 + K + 15) // 16]
        k, v = (dequantise(*read_runs(x[used, g], 128, i)).reshape(-1, 128)[:2048 + K] for i, x in enumerate((c["k"], c["v"])))
        want, _ = attention(c["q"][0, :, g * G:(g + 1) * G].double().numpy(), k, v, _sees(c, 0, 0), c["scale"], 0.0)
        off += ((out[0, :, g * G:(g + 1) * G] - want) ** 2).sum()
        size += (want ** 2).sum()
    assert math.sqrt(off / size) < 1.06 * 2.35e-3
