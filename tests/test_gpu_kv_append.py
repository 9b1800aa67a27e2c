"""graft_kv_append and graft_kv_append_mx: rotated queries, and caches bit for bit, against plain numpy."""
import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from gpu_util import dev, host
from mx_util import dequantise, quantise, random_tree, read_runs, rotate32, rotate64, run_bytes, write_row

pytestmark = pytest.mark.gpu


def _case(seed, dtype, B, T, Hq, Hkv, D, R, P, lengths=None, fused=True, tree=True, special=False):
    rng = np.random.default_rng(seed)
    tt = torch.float32 if dtype == "f32" else torch.bfloat16
    lengths = np.array(lengths if lengths is not None else [T - b % (T // 2 + 1) for b in range(B)], np.int32)
    P = np.array([P + 3 * b for b in range(B)] if np.isscalar(P) else P, np.int32)
    max_pages = int((P + T).max() + 15) // 16
    total = B * max_pages + 2
    rows = torch.from_numpy(rng.standard_normal((B, T, Hq + 2 * Hkv, D)).astype(np.float32)).to(tt)
    if special:                                            # blocks with an infinity or NaN, all zeros, tiny, at rounding borders
        rows[0, 0, Hq:, 3] = float("inf")
        rows[0, 1, Hq:, 40] = float("nan")
        rows[0, 2, Hq:, :32] = 0
        rows[0, 3, Hq:, 32:] *= 2.0 ** -124
        rows[0, 4, Hq:, :32] = torch.tensor([1.75, 7, 0.25, 0.75, 1.25, 2.5, 3.5, 5] * 4)
        rows[0, 5, Hq:, :32] *= 2.0 ** 100
        rows[0, 6, Hq:, 5] = 3e38
    cut = [rows[:, :, :Hq], rows[:, :, Hq:Hq + Hkv], rows[:, :, Hq + Hkv:]]
    pos = np.full((B, T), -1, np.int32)
    for b in range(B):
        pos[b, :lengths[b]] = P[b] + (random_tree(rng, lengths[b])[1] if tree else np.arange(lengths[b]))
    n_pos = int((P + T).max())
    angle = rng.uniform(0, 6.28, (n_pos, R // 2))
    cos_sin = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    return dict(dtype=dtype, tt=tt, B=B, T=T, Hq=Hq, Hkv=Hkv, D=D, R=R, P=P, n=lengths, rows=rows, pos=pos, cos_sin=cos_sin, total=total, max_pages=max_pages,
                table=rng.permutation(total)[:B * max_pages].reshape(B, max_pages).astype(np.int32),
                gpu=[x.cuda() for x in cut] if not fused else [rows.cuda()[:, :, a:b] for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv))])


def _turned(c, b, part, interleaved, bits=32):
    """Rows [n,H,D] of sequence b: part 0 queries, 1 keys, 2 values."""
    lo, hi = (0, c["Hq"]) if part == 0 else (c["Hq"], c["Hq"] + c["Hkv"]) if part == 1 else (c["Hq"] + c["Hkv"], c["Hq"] + 2 * c["Hkv"])
    x = c["rows"][b, :c["n"][b], lo:hi].float().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        if part == 2 or c["R"] == 0:
            return (x, np.zeros_like(x)) if bits == 64 else x
        return (rotate64 if bits == 64 else rotate32)(x, c["cos_sin"], c["pos"][b, :c["n"][b]], interleaved)


def _same_bits(a, b):
    """Equal, NaN where NaN is."""
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


def _round(x, tt):
    return torch.from_numpy(np.ascontiguousarray(x)).to(tt)


def _check_q(c, q, interleaved):
    half = 2.0 ** -24 if c["dtype"] == "f32" else 2.0 ** -8
    for b in range(c["B"]):
        n = c["n"][b]
        assert _same_bits(q[b, :n].cpu(), _round(_turned(c, b, 0, interleaved), c["tt"]))
        # two products and a sum of half a step each, and the type's own
        exact, size = _turned(c, b, 0, interleaved, 64)
        got = q[b, :n].double().cpu().numpy()
        assert (abs(got - exact) <= (half + 2.0 ** -24) * abs(exact) + 2.0 ** -24 * (1 + 2.0 ** -20) * size + 1e-38).all()
        assert bool((q[b, n:] == -7).all())                # padding stays as it was


APPENDS = [
    ("f32", 1, 1, 8, 2, 64, 64, 0, False, "head"), ("f32", 3, 5, 3, 3, 128, 64, 15, True, "token"), ("bf16", 2, 40, 32, 8, 128, 128, 100, False, "head"),
    ("bf16", 5, 17, 16, 1, 64, 16, 31, False, "token"), ("bf16", 4, 128, 8, 4, 128, 48, 7, True, "head"), ("f32", 2, 33, 4, 2, 64, 0, 16, False, "head"),
    ("bf16", 1, 300, 7, 7, 64, 32, 5, True, "head"), ("bf16", 2, 9, 48, 3, 128, 112, 1000, False, "gap"),
]


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,R,P,interleaved,layout", APPENDS)
@pytest.mark.parametrize("fused", [True, False])
def test_append(dtype, B, T, Hq, Hkv, D, R, P, interleaved, layout, fused):
    c = _case(B * 100 + T, dtype, B, T, Hq, Hkv, D, R, P, fused=fused, tree=T <= 128)
    if layout == "token":
        strides, size = {"page": 16 * Hkv * D, "token": Hkv * D, "head": D}, 16 * Hkv * D
    elif layout == "head":
        strides, size = {"page": 16 * Hkv * D, "token": D, "head": 16 * D}, 16 * Hkv * D
    else:                                                  # a hole behind every token and page
        strides, size = {"page": 16 * Hkv * (D + 8) + 64, "token": D + 8, "head": 16 * (D + 8)}, 16 * Hkv * (D + 8) + 64
    caches = [torch.full((c["total"] * size,), -7.0, dtype=c["tt"], device="cuda") for _ in range(2)]
    want = [torch.full((c["total"] * size,), -7.0, dtype=c["tt"]) for _ in range(2)]
    out = {"q": torch.full((B, T, Hq, D), -7.0, dtype=c["tt"], device="cuda"), "status": torch.full((B,), -7, dtype=torch.int32, device="cuda")}
    got = graft.graft_kv_append(*c["gpu"], dev(c["cos_sin"], "f32") if R else None, dev(c["pos"]), *caches, strides, dev(c["table"]), dev(c["P"]),
                                dev(c["n"]), interleaved=interleaved, out=out)
    assert got["q"] is out["q"] and (host(got["status"]) == 0).all()
    _check_q(c, got["q"], interleaved)
    for b in range(B):
        for cache, part in zip(want, (1, 2)):
            x = _round(_turned(c, b, part, interleaved), c["tt"])
            for i in range(c["n"][b]):
                t = int(c["P"][b]) + i
                at = int(c["table"][b, t // 16]) * strides["page"] + t % 16 * strides["token"]
                for h in range(Hkv):
                    cache[at + h * strides["head"]:at + h * strides["head"] + D] = x[i, h]
    for cache, w in zip(caches, want):                     # every element, the untouched ones too
        assert _same_bits(cache.cpu(), w)


MXS = [("f32", 1, 1, 8, 2, 64, 64, 0, False), ("bf16", 2, 40, 32, 8, 128, 128, 100, False), ("bf16", 5, 17, 16, 1, 64, 16, 31, False), ("f32", 3, 9, 4, 3, 128, 48, 15, True),
       ("bf16", 4, 128, 8, 4, 128, 64, 7, True), ("bf16", 1, 300, 6, 2, 64, 0, 3, False), ("bf16", 2, 16, 5, 5, 128, 16, 16, True)]


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,D,R,P,interleaved", MXS)
@pytest.mark.parametrize("special", [False, True])
def test_append_mx(dtype, B, T, Hq, Hkv, D, R, P, interleaved, special):
    if special and T < 7:
        pytest.skip("seven special rows")
    c = _case(B * 100 + T + 1, dtype, B, T, Hq, Hkv, D, R, P, tree=T <= 128, special=special)
    run = run_bytes(D)
    strides = {"page": Hkv * (run + 48) + 32 if D == 64 else Hkv * run, "head": run + 48 if D == 64 else run}
    strides["page"] += -strides["page"] % 16
    caches = [torch.full((c["total"] * strides["page"],), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = {"q": torch.full((B, T, Hq, D), -7.0, dtype=c["tt"], device="cuda"), "status": torch.full((B,), -7, dtype=torch.int32, device="cuda")}
    place = (dev(c["table"]), dev(c["P"]), dev(c["n"]))
    got = graft.graft_kv_append_mx(*c["gpu"], dev(c["cos_sin"], "f32") if R else None, dev(c["pos"]), *caches, strides, *place, interleaved=interleaved, out=out)
    assert (host(got["status"]) == 0).all()
    _check_q(c, got["q"], interleaved)
    for cache, part in zip(caches, (1, 2)):
        want = np.full(c["total"] * strides["page"], 0xA5, np.uint8)
        for b in range(B):
            code, byte = quantise(_turned(c, b, part, interleaved))
            for i in range(c["n"][b]):
                t = int(c["P"][b]) + i
                for h in range(Hkv):
                    at = int(c["table"][b, t // 16]) * strides["page"] + h * strides["head"]
                    write_row(want[at:at + run], D, part == 2, t % 16, code[i, h], byte[i, h])
        assert (cache.cpu().numpy() == want).all()
    # and back as numbers, in both types
    for tt in (torch.bfloat16, torch.float32):
        back = graft.graft_kv_gather_mx(*caches, 0, 1, strides, *place, T, Hkv, D, dtype=tt)
        assert (host(back["status"]) == 0).all() and back["k"].dtype == tt
        for name, part in (("k", 1), ("v", 2)):
            for b in range(B):
                x = back[name][0, b].double().cpu().numpy()
                assert np.array_equal(x[:c["n"][b]], dequantise(*quantise(_turned(c, b, part, interleaved))), equal_nan=True)
                assert (x[c["n"][b]:] == 0).all()


def test_positions_without_a_tree_and_q_in_place():
    """pos None is prefix + i; q_out may be q; no queries at all."""
    c = _case(3, "bf16", 2, 21, 4, 2, 128, 128, 9, fused=False, tree=False)
    strides = {"page": 16 * 2 * 128, "token": 128, "head": 16 * 128}
    q, k, v = (x.contiguous() for x in c["gpu"])
    angles, place = dev(c["cos_sin"], "f32"), (dev(c["table"]), dev(c["P"]), dev(c["n"]))
    new = lambda: [torch.zeros((c["total"], 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    a, b, d = new(), new(), new()
    one = graft.graft_kv_append(q, k, v, angles, dev(c["pos"]), *a, strides, *place)
    keep = q.clone()
    two = graft.graft_kv_append(q, k, v, angles, None, *b, strides, *place, out={"q": q, "status": torch.zeros(2, dtype=torch.int32, device="cuda")})
    three = graft.graft_kv_append(None, k, v, angles, None, *d, strides, *place)
    assert "q" not in three
    for i in range(2):
        n = c["n"][i]
        assert torch.equal(one["q"][i, :n], two["q"][i, :n]) and torch.equal(q[i, n:], keep[i, n:])
    for x, y, z in zip(a, b, d):
        assert torch.equal(x, y) and torch.equal(x, z)


@pytest.mark.parametrize("mx", [False, True])
def test_lengths_and_positions_out_of_range(mx):
    """Sequences whose lengths do not fit stay as they were; a token whose position is not in the table stays out."""
    B, T, D = 6, 8, 64
    c = _case(5, "f32", B, T, 2, 2, D, 64, [0, 1, 10, 100, 4, 20], lengths=[8, 4, 8, 8, 0, 0], tree=False)
    c["P"][1], c["n"][2], c["n"][4] = -1, 9, -1
    c["pos"][0] = np.arange(T)
    c["pos"][0, 3], c["pos"][0, 5] = -1, c["cos_sin"].shape[0]
    c["P"][3] = c["max_pages"] * 16 - 7                    # one token too many
    if mx:
        strides, caches = {"page": 1088, "head": 544}, [torch.full((c["total"], 2, 544), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2)]
    else:
        strides, caches = {"page": 2048, "token": 64, "head": 1024}, [torch.full((c["total"], 2, 16, 64), -7.0, device="cuda") for _ in range(2)]
    out = {"q": torch.full((B, T, 2, D), -7.0, device="cuda"), "status": torch.full((B,), -7, dtype=torch.int32, device="cuda")}
    f = graft.graft_kv_append_mx if mx else graft.graft_kv_append
    before = [x.clone() for x in caches]
    got = f(*c["gpu"], dev(c["cos_sin"], "f32"), dev(c["pos"]), *caches, strides, dev(c["table"]), dev(c["P"]), dev(c["n"]), out=out)
    assert host(got["status"]).tolist() == [1, 1, 1, 1, 1, 0]
    written = [i for i in range(8) if i not in (3, 5)]
    assert bool((got["q"][0, [3, 5]] == -7).all()) and bool((got["q"][1:] == -7).all()) and not bool((got["q"][0, written] == -7).any())
    page = int(c["table"][0, 0])
    for cache, old in zip(caches, before):
        rest = torch.arange(c["total"], device="cuda") != page
        assert torch.equal(cache[rest], old[rest])
        if not mx:
            assert torch.equal(cache[page][:, [3, 5] + list(range(8, 16))], old[page][:, [3, 5] + list(range(8, 16))])
            assert not bool((cache[page][:, written] == -7).any())
    if mx:
        for cache, values in zip(caches, (False, True)):
            code, byte = read_runs(cache[page].cpu().numpy(), D, values)
            stay = [3, 5] + list(range(8, 16))
            old = read_runs(before[0][page].cpu().numpy(), D, values)
            assert (code[:, stay] == old[0][:, stay]).all() and (byte[:, stay] == 0x5A).all() and not (byte[:, written] == 0x5A).any()


def test_long_prompt():
    """4099 tokens: more than a tree, the last page half full."""
    c = _case(8, "bf16", 1, 4099, 2, 1, 128, 128, 30, lengths=[4099], tree=False)
    cache = [torch.zeros((c["total"], 1, 1088), dtype=torch.uint8, device="cuda") for _ in range(2)]
    graft.graft_kv_append_mx(*c["gpu"], dev(c["cos_sin"], "f32"), None, *cache, {"page": 1088, "head": 1088}, dev(c["table"]), dev(c["P"]), dev(c["n"]))
    for x, part in zip(cache, (1, 2)):
        runs = x[torch.from_numpy(c["table"][0].astype(np.int64)).cuda(), 0].cpu().numpy()
        code, byte = (y.reshape(-1, y.shape[-1])[30:30 + 4099] for y in read_runs(runs, 128, part == 2))
        want = quantise(_turned(c, 0, part, False)[:, 0])
        assert (code == want[0]).all() and (byte == want[1]).all()
