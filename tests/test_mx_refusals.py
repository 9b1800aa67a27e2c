"""Arguments that the rotation, the 4-bit cache and the attention over it refuse (no GPU): nothing is launched."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from mx_util import GRID, dequantise, pack_runs, quantise, read_runs, write_row

P = 0x1000      # a non-NULL placeholder: validation must fail before any pointer is touched
NULL, SHAPE, DTYPE, WORKSPACE = graft.GRAFT_ERR_NULL, graft.GRAFT_ERR_SHAPE, graft.GRAFT_ERR_DTYPE, graft.GRAFT_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return graft.load_library()


def _call(f, ok, **kw):
    a = list(ok)
    for k, v in kw.items():
        a[int(k[1:])] = v
    return f(*a)


# q k v | strides | cos_sin n_pos R interleaved pos | caches | page token head | table max_pages P n | B T Hq Hkv D page dtype | q_out status stream
APPEND = [P, 0x200000, 0x300000, 512, 256, 256, P, 64, 64, 0, None, 0x400000, 0x500000, 2048, 64, 1024, P, 4, P, P, 1, 4, 8, 2, 64, 16, 1, 0x600000, P, None]


@pytest.mark.parametrize("change,code", [
    ({"a0": None}, NULL), ({"a1": None}, NULL), ({"a2": None}, NULL), ({"a6": None}, NULL), ({"a11": None}, NULL), ({"a12": None}, NULL),
    ({"a16": None}, NULL), ({"a18": None}, NULL), ({"a19": None}, NULL), ({"a27": None}, NULL), ({"a28": None}, NULL),
    ({"a26": 2}, DTYPE),
    ({"a3": 511}, SHAPE), ({"a3": 504}, SHAPE), ({"a4": 120}, SHAPE), ({"a5": 130}, SHAPE), ({"a7": 0}, SHAPE), ({"a8": 80}, SHAPE), ({"a8": 8}, SHAPE),
    ({"a8": -16}, SHAPE), ({"a9": 2}, SHAPE), ({"a13": 0}, SHAPE), ({"a13": 2044}, SHAPE), ({"a14": 63}, SHAPE), ({"a15": 32}, SHAPE), ({"a17": 0}, SHAPE),
    ({"a17": 262145}, SHAPE), ({"a20": 0}, SHAPE), ({"a20": 65536}, SHAPE), ({"a21": 0}, SHAPE), ({"a22": -1}, SHAPE), ({"a23": 0}, SHAPE), ({"a24": 96}, SHAPE),
    ({"a25": 32}, SHAPE), ({"a0": P + 8}, SHAPE), ({"a11": P + 4}, SHAPE), ({"a27": 0x600008}, SHAPE),
    ({"a27": 0x200100}, SHAPE),                            # q_out within k
    ({"a27": P + 1024}, SHAPE),                            # q_out one token behind q
    ({"a27": P, "a3": 1024}, SHAPE),                       # q_out is q, but q is not dense
])
def test_append(lib, change, code):
    assert _call(lib.graft_kv_append, APPEND, **change) == code


MX = APPEND[:13] + [2 * 544, 544] + APPEND[16:]


@pytest.mark.parametrize("change,code", [
    ({"a1": None}, NULL), ({"a12": None}, NULL), ({"a27": None}, NULL), ({"a25": 5}, DTYPE), ({"a13": 543}, SHAPE), ({"a14": 528}, SHAPE), ({"a14": 552}, SHAPE),
    ({"a23": 32}, SHAPE), ({"a24": 8}, SHAPE), ({"a19": -1}, SHAPE), ({"a20": 0}, SHAPE),
])
def test_append_mx(lib, change, code):
    assert _call(lib.graft_kv_append_mx, MX, **change) == code


# caches layer_stride layers page head table max_pages start count B T Hkv D dtype outs status stream
GATHER = [P, P, 8704, 2, 1088, 544, P, 4, P, P, 1, 4, 2, 64, 1, P, P, P, None]


@pytest.mark.parametrize("change,code", [
    ({"a0": None}, NULL), ({"a1": None}, NULL), ({"a6": None}, NULL), ({"a9": None}, NULL), ({"a15": None}, NULL), ({"a16": None}, NULL), ({"a17": None}, NULL),
    ({"a14": 3}, DTYPE), ({"a2": 0}, SHAPE), ({"a2": -16}, SHAPE), ({"a2": 8705}, SHAPE), ({"a3": 0}, SHAPE), ({"a4": 500}, SHAPE), ({"a5": 540}, SHAPE),
    ({"a7": 0}, SHAPE), ({"a10": 0}, SHAPE), ({"a11": 0}, SHAPE), ({"a12": 0}, SHAPE), ({"a13": 32}, SHAPE), ({"a15": P + 2}, SHAPE),
])
def test_gather(lib, change, code):
    assert _call(lib.graft_kv_gather_mx, GATHER, **change) == code


def test_gather_limits(lib):
    """More rows of a sequence than a launch has lanes for."""
    assert _call(lib.graft_kv_gather_mx, GATHER, a11=(1 << 31) - 1) == SHAPE


# q caches page head table max_pages P n mask pos B K Hq Hkv D page scale cap window out ws bytes stream
ATTN = [P, P, P, 1088, 544, P, 4, P, P, P, P, 1, 4, 8, 2, 64, 16, 0.125, 0.0, 0, P, None, 0, None]


@pytest.mark.parametrize("change,code", [
    ({"a0": None}, NULL), ({"a1": None}, NULL), ({"a2": None}, NULL), ({"a5": None}, NULL), ({"a7": None}, NULL), ({"a8": None}, NULL), ({"a20": None}, NULL),
    ({"a10": None, "a19": 5}, NULL),                       # a window over a tree needs positions
    ({"a3": 543}, SHAPE), ({"a4": 8}, SHAPE), ({"a6": 0}, SHAPE), ({"a6": 262145}, SHAPE), ({"a11": 0}, SHAPE), ({"a12": 0}, SHAPE), ({"a12": 129}, SHAPE),
    ({"a13": 7}, SHAPE), ({"a13": 34}, SHAPE), ({"a13": 0}, SHAPE), ({"a14": 0}, SHAPE), ({"a15": 96}, SHAPE), ({"a16": 32}, SHAPE), ({"a17": float("inf")}, SHAPE),
    ({"a17": float("nan")}, SHAPE), ({"a18": -1.0}, SHAPE), ({"a18": float("inf")}, SHAPE), ({"a18": float("nan")}, SHAPE), ({"a19": -1}, SHAPE), ({"a0": P + 2}, SHAPE), ({"a20": P + 8}, SHAPE),
    ({"a6": 4096}, WORKSPACE), ({"a6": 4096, "a21": P, "a22": 64}, WORKSPACE), ({"a6": 4096, "a21": P + 4, "a22": 1 << 40}, WORKSPACE),
])
def test_attention(lib, change, code):
    assert _call(lib.graft_tree_attn_mx, ATTN, **change) == code


@pytest.mark.parametrize("change,code", [
    ({"a3": 1 << 32}, SHAPE), ({"a11": 65536}, SHAPE), ({"a11": 65535, "a13": 8, "a14": 8}, SHAPE), ({"a11": 4, "a13": 65536, "a14": 65536}, SHAPE),
])
def test_attention_limits(lib, change, code):
    """Page strides of 2^32 bytes, and more heads of sequences than workgroups are counted in."""
    assert _call(lib.graft_tree_attn_mx, ATTN, **change) == code


@pytest.mark.parametrize("change", [{"a18": 1025.0}, {"a17": 3e38}, {"a18": 1e-39}, {"a17": -3e38, "a18": 0.5}])
def test_attention_scales(lib, change):
    """Caps that leave too little of a score, scales whose products with log2(e) do not fit a float."""
    assert _call(lib.graft_tree_attn_mx, ATTN, **change) == SHAPE


@pytest.mark.parametrize("f,args,T,out", [("graft_kv_append", APPEND, "a21", "a27"), ("graft_kv_append_mx", MX, "a20", "a26")])
def test_append_limits(lib, f, args, T, out):
    """q in place where keys or values lie in it, and more tokens than are counted in."""
    f = getattr(lib, f)
    assert _call(f, args, **{out: P, "a1": P + 1024}) == SHAPE
    assert _call(f, args, **{out: P, "a2": P + 1024}) == SHAPE
    assert _call(f, args, **{T: (1 << 30) + 1}) == SHAPE


def test_attention_workspace(lib):
    w = graft.graft_tree_attn_mx_workspace_bytes
    assert w(1, 4, 8, 2, 64, 4) == 0                       # one split
    assert w(1, 4, 8, 2, 64, 4096) > 0
    assert w(1, 129, 8, 2, 64, 4096) == 0 and w(1, 4, 8, 3, 64, 4096) == 0 and w(1, 4, 8, 2, 80, 4096) == 0


# caches layer_stride layers page head table max_pages P path accept B cap K Hkv D new status stream
COMPACT = [P, P, 8704, 2, 1088, 544, P, 4, 0x2000, P, 0x3000, 1, 8, 16, 2, 64, 0x4000, P, None]


@pytest.mark.parametrize("change,code", [
    ({"a0": None}, NULL), ({"a6": None}, NULL), ({"a8": None}, NULL), ({"a9": None}, NULL), ({"a10": None}, NULL), ({"a16": None}, NULL), ({"a17": None}, NULL),
    ({"a2": 0}, SHAPE), ({"a3": 0}, SHAPE), ({"a4": 528}, SHAPE), ({"a5": 545}, SHAPE), ({"a7": 0}, SHAPE), ({"a11": 0}, SHAPE), ({"a12": 128}, SHAPE), ({"a12": -1}, SHAPE),
    ({"a13": 0}, SHAPE), ({"a13": 129}, SHAPE), ({"a14": 0}, SHAPE), ({"a15": 100}, SHAPE), ({"a0": P + 8}, SHAPE), ({"a16": 0x2000}, SHAPE), ({"a16": 0x3000}, SHAPE),
])
def test_compact(lib, change, code):
    assert _call(lib.graft_kv_compact_mx, COMPACT, **change) == code


def _append_args(**kw):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    a = dict(q=torch.zeros((1, 2, 4, 64)), k=torch.zeros((1, 2, 2, 64)), v=torch.zeros((1, 2, 2, 64)), cos_sin=torch.zeros((8, 64)), pos=i32(1, 2),
             k_cache=torch.zeros((4, 2, 16, 64)), v_cache=torch.zeros((4, 2, 16, 64)), strides={"page": 2048, "token": 64, "head": 1024}, block_table=i32(1, 4),
             prefix_len=i32(1), n_nodes=i32(1))
    a.update(kw)
    return a


@pytest.mark.parametrize("change,error", [
    ({}, ValueError),                                                                   # not on the GPU
    ({"q": torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)}, AssertionError),
    ({"q": torch.zeros((1, 2, 4, 64), dtype=torch.float16), "k": torch.zeros((1, 2, 2, 64), dtype=torch.float16)}, AssertionError),
    ({"q": torch.zeros((1, 3, 4, 64))}, ValueError), ({"v": torch.zeros((1, 2, 1, 64))}, ValueError), ({"k": torch.zeros((2, 2, 64))}, ValueError),
    ({"k": torch.zeros((1, 2, 64, 2)).transpose(2, 3)}, ValueError),                    # elements not side by side
    ({"q": torch.zeros((1, 4, 2, 64)).transpose(1, 2)}, ValueError),                    # heads not dense
    ({"pos": torch.zeros((1, 2), dtype=torch.int64)}, ValueError), ({"pos": torch.zeros((1, 3), dtype=torch.int32)}, ValueError),
    ({"prefix_len": torch.zeros(2, dtype=torch.int32)}, ValueError), ({"cos_sin": torch.zeros((8, 64), dtype=torch.float64)}, ValueError),
    ({"k_cache": torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)}, AssertionError), ({"strides": {"page": 1}}, KeyError), ({"q": 3}, TypeError),
])
def test_append_binding(change, error):
    with pytest.raises(error):
        graft.graft_kv_append(**_append_args(**change))


def test_mx_bindings():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    u8 = torch.zeros((4, 2, 544), dtype=torch.uint8)
    st = {"page": 1088, "head": 544}
    with pytest.raises(ValueError):                                                     # not bytes
        graft.graft_kv_append_mx(**_append_args(strides=st))
    with pytest.raises(ValueError):                                                     # not on the GPU
        graft.graft_kv_append_mx(**_append_args(k_cache=u8, v_cache=u8, strides=st))
    with pytest.raises(ValueError):
        graft.graft_kv_gather_mx(u8, u8, 0, 1, st, i32(1, 4), i32(1), i32(1), 2, 2, 64, dtype=torch.float16)
    with pytest.raises(OverflowError):
        graft.graft_kv_gather_mx(u8, u8, 0, 1, st, i32(1, 4), i32(1), i32(1), 1 << 40, 2, 64)
    q, mask = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 2), dtype=torch.int64)
    attn = lambda **kw: graft.graft_tree_attn_mx(**{**dict(q=q, k_cache=u8, v_cache=u8, strides=st, block_table=i32(1, 4), prefix_len=i32(1), n_nodes=i32(1),
                                                           mask=mask, Hkv=2, scale=0.1), **kw})
    for kw, error in (({}, ValueError), ({"q": q.float()}, AssertionError), ({"mask": mask[:, :1]}, ValueError), ({"k_cache": u8.float()}, ValueError),
                      ({"scale": "x"}, TypeError), ({"window": 1.5}, TypeError), ({"window": 1 << 35}, OverflowError), ({"pos": i32(1, 3)}, ValueError)):
        with pytest.raises(error):
            attn(**kw)
    with pytest.raises(ValueError):
        graft.graft_kv_compact_mx(u8, u8, 0, 1, st, i32(1, 4), i32(1), i32(1, 3), i32(1), 8, 2, 64)


def test_run_bytes():
    assert graft.graft_mx_run_bytes(64) == 544 and graft.graft_mx_run_bytes(128) == 1088


def test_the_reference_of_the_format():
    """The tests' own packing is its own inverse, rounds to even and keeps magnitudes: by hand."""
    x = np.zeros((1, 32), np.float32)
    x[0, :12] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5.01, -0.26, 7, 0.2]
    code, byte = quantise(x)
    assert byte[0, 0] == 127 and list(dequantise(code, byte)[0, :12]) == [6, 0, 1, 1, 2, 2, 4, 4, -6, -0.5, 6, 0]
    x[0, 10] = 7.01
    assert quantise(x)[1][0, 0] == 128
    x[0, 3] = np.inf
    assert quantise(x)[1][0, 0] == 255 and np.isnan(dequantise(*quantise(x))).all()
    rng = np.random.default_rng(0)
    for D in (64, 128):
        for values in (False, True):
            code, byte = rng.integers(0, 16, (3, 16, D)).astype(np.uint8), rng.integers(0, 256, (3, 16, D // 32)).astype(np.uint8)
            runs = pack_runs(code, byte, values)
            assert runs.shape == (3, 17 * D // 2)
            back = read_runs(runs, D, values)
            assert (back[0] == code).all() and (back[1] == byte).all()
            other = np.zeros_like(runs[0])
            for t in range(16):
                write_row(other, D, values, t, code[0, t], byte[0, t])
            assert (other == runs[0]).all()
    assert len(GRID) == 8
