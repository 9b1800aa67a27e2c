"""Arguments that prompt attention, token counts and rules on logits refuse (no GPU): nothing is launched."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2605_20104_amd as graft
from paper_2605_20104_amd import build
from test_device_plans import STAND_IN

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


# q caches | page token head | table max_pages P n | B T Hq Hkv D page | scale cap window dtype | out ws bytes stream
PROMPT = [P, 0x200000, 0x300000, 2048, 64, 1024, P, 64, P, P, 2, 40, 8, 2, 64, 16, 0.125, 0.0, 0, 1, 0x400000, None, 0, None]
# one token behind a table of 64K: this one has splits, and wants a workspace
SPLIT = PROMPT[:7] + [4096, P, P, 1, 1] + PROMPT[12:]


@pytest.mark.parametrize("change,code", [
    ({"a0": None}, NULL), ({"a1": None}, NULL), ({"a2": None}, NULL), ({"a6": None}, NULL), ({"a8": None}, NULL), ({"a9": None}, NULL), ({"a20": None}, NULL),
    ({"a19": 2}, DTYPE), ({"a19": -1}, DTYPE),
    ({"a3": 0}, SHAPE), ({"a3": 2044}, SHAPE), ({"a4": 56}, SHAPE), ({"a4": 68}, SHAPE), ({"a4": 1 << 26}, SHAPE), ({"a5": 60}, SHAPE), ({"a5": 1028}, SHAPE),
    ({"a7": 0}, SHAPE), ({"a7": 262145}, SHAPE), ({"a10": 0}, SHAPE), ({"a10": 65536}, SHAPE), ({"a11": 0}, SHAPE), ({"a11": (1 << 22) + 1}, SHAPE),
    ({"a12": 0}, SHAPE), ({"a12": 7}, SHAPE), ({"a12": 34}, SHAPE), ({"a13": 0}, SHAPE), ({"a14": 96}, SHAPE), ({"a15": 32}, SHAPE),
    ({"a10": 65535, "a12": 16, "a13": 16}, SHAPE), ({"a10": 64, "a11": 1 << 22, "a12": 16, "a13": 1}, SHAPE),
    ({"a16": float("nan")}, SHAPE), ({"a16": float("inf")}, SHAPE), ({"a16": 3e38}, SHAPE), ({"a17": -1.0}, SHAPE), ({"a17": 1025.0}, SHAPE),
    ({"a17": float("nan")}, SHAPE), ({"a17": 1e-38, "a16": 10.0}, SHAPE), ({"a18": -1}, SHAPE),
    ({"a0": P + 8}, SHAPE), ({"a1": 0x200004}, SHAPE), ({"a20": 0x400002}, SHAPE), ({"a20": P + 16}, SHAPE),
])
def test_prompt_attn(lib, change, code):
    assert _call(lib.graft_prompt_attn, PROMPT, **change) == code


@pytest.mark.parametrize("change", [{}, {"a21": P, "a22": 100}, {"a21": P + 8, "a22": 1 << 30}])
def test_prompt_attn_workspace(lib, change):
    assert lib.graft_prompt_attn_workspace_bytes(1, 1, 8, 2, 64, 4096, 0, 1) > 0
    assert _call(lib.graft_prompt_attn, SPLIT, **change) == WORKSPACE


def test_prompt_attn_workspace_sizes(lib):
    w = lib.graft_prompt_attn_workspace_bytes
    assert w(1, 1, 8, 2, 64, 1, 0, 1) == 0                  # one page: no splits
    assert w(0, 1, 8, 2, 64, 64, 0, 1) == 0 and w(1, 1, 8, 2, 64, 64, 0, 3) == 0 and w(1, 1, 7, 2, 64, 64, 0, 1) == 0
    assert w(1, 1, 8, 2, 64, 262144, 0, 1) > 0
    assert w(1, 1, 8, 2, 64, 262144, 64, 1) == 0            # a short window leaves nothing to split
    assert w(4, 8192, 32, 8, 128, 512, 0, 1) == 0           # enough tiles for every compute unit


# The merge has a wavefront for each row: with rows for 2^32 lanes and more there would be no launch for it, so nothing is split there.
@pytest.mark.parametrize("B,T,Hq,Hkv,D,dtype", [(1, 2097665, 32, 2, 64, 0), (1, 1048577, 128, 8, 64, 0), (1, 1048577, 32, 2, 64, 0), (3, 1 << 22, 16, 1, 128, 1)])
def test_prompt_attn_splits_only_what_a_merge_can_take(B, T, Hq, Hkv, D, dtype):
    rows = B * Hq * T
    size = graft.graft_prompt_attn_workspace_bytes(B, T, Hq, Hkv, D, 262144, 0, dtype)
    assert size == 0 or rows * 64 < 1 << 31, size / (rows * (D + 2) * 4)


def test_prompt_workspaces_follow_the_current_device(tmp_path):
    (tmp_path / "stand_in.c").write_text(STAND_IN)
    so = str(tmp_path / "stand_in.so")
    subprocess.run([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-o", so, str(tmp_path / "stand_in.c")], check=True)
    program = ("import ctypes, sys\ns = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)\nf = ctypes.CDLL(sys.argv[2]).graft_prompt_attn_workspace_bytes\n"
               "f.restype = ctypes.c_size_t\nfor d in (0, 1, 0):\n    s.set_device(d)\n    print(f(4, 1, 32, 8, 128, 4096, 0, 1))\n")
    a, b, c = [int(x) for x in subprocess.run([sys.executable, "-c", program, so, build.LIB], check=True, stdout=subprocess.PIPE, text=True).stdout.split()]
    assert a == c and b > 0 and a != b                      # (256 compute units and 64)


# ctx len prompt start | B L V | counts status stream
COUNTS = [P, P, P, None, 2, 100, 1000, P, P, None]


@pytest.mark.parametrize("change,code", [
    ({"a0": None}, NULL), ({"a1": None}, NULL), ({"a7": None}, NULL), ({"a8": None}, NULL), ({"a4": 0}, SHAPE), ({"a4": 65536}, SHAPE), ({"a5": 0}, SHAPE),
    ({"a5": 1 << 30}, SHAPE), ({"a6": 0}, SHAPE), ({"a6": 1 << 30}, SHAPE),
])
def test_token_counts(lib, change, code):
    assert _call(lib.graft_token_counts, COUNTS, **change) == code
    assert _call(lib.graft_token_counts, COUNTS, **dict({"a3": P}, **change)) == code


# logits n tokens mask | B K V | counts rep freq pres bias rows | allow n index | out ids status | ws bytes stream
RULES = [P, P, P, P, 2, 8, 1000, P, P, P, P, P, 1, P, 3, P, 0x200000, P, P, P, 1 << 20, None]


@pytest.mark.parametrize("change,code", [
    ({"a0": None}, NULL), ({"a1": None}, NULL), ({"a2": None}, NULL), ({"a3": None}, NULL), ({"a13": None}, NULL), ({"a15": None}, NULL), ({"a18": None}, NULL),
    ({"a16": None, "a17": None}, NULL),
    ({"a4": 0}, SHAPE), ({"a4": 65536}, SHAPE), ({"a5": 0}, SHAPE), ({"a5": 129}, SHAPE), ({"a6": 0}, SHAPE), ({"a6": 1 << 30}, SHAPE), ({"a12": 0}, SHAPE),
    ({"a12": 3}, SHAPE), ({"a14": 0}, SHAPE), ({"a16": P + 4}, SHAPE), ({"a16": P + 2 * 8 * 1000 * 4 - 4}, SHAPE),
    ({"a19": None}, WORKSPACE), ({"a20": 15}, WORKSPACE), ({"a19": P + 4}, WORKSPACE),
])
def test_logits_adjust(lib, change, code):
    assert _call(lib.graft_logits_adjust, RULES, **change) == code


def test_rules_workspace(lib):
    w = lib.graft_logits_adjust_workspace_bytes
    assert w(0, 8, 1000) == 0 and w(2, 8, 0) == 0 and w(2, 8, 1000) > 0
    assert w(2, 8, 1 << 30) == 0


# ---- what the binding checks before the library sees a pointer
def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_prompt_attn_binding():
    q, c = torch.zeros((2, 5, 8, 64), dtype=torch.bfloat16), torch.zeros((9, 2, 16, 64), dtype=torch.bfloat16)
    st = {"page": 2048, "token": 64, "head": 1024}
    ok = [q, c, c, st, _i32(2, 4), _i32(2), _i32(2), 2, 0.125]

    def call(i, x, **kw):
        a = list(ok)
        a[i] = x
        return graft.graft_prompt_attn(*a, **kw)
    with pytest.raises(ValueError, match="GPU"):
        call(0, q)
    with pytest.raises(AssertionError):
        call(0, q.float())
    with pytest.raises(AssertionError):
        call(1, c.float())
    with pytest.raises(ValueError):
        call(0, q[0])
    with pytest.raises(AssertionError, match="dense"):
        call(0, q.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(KeyError):
        call(3, {"page": 1, "head": 1})
    with pytest.raises(ValueError, match="block_table"):
        call(4, _i32(3, 4))
    with pytest.raises(ValueError, match="prefix_len"):
        call(5, _i32(3))
    with pytest.raises(ValueError, match="n_nodes"):
        call(6, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError):
        call(8, "0.1")
    with pytest.raises(OverflowError):
        call(7, 2, window=1 << 40)


def test_counts_and_rules_binding():
    with pytest.raises(ValueError, match="GPU"):
        graft.graft_token_counts(_i32(2, 9), _i32(2), None, _i32(2, 50))
    with pytest.raises(ValueError, match="counts"):
        graft.graft_token_counts(_i32(2, 9), _i32(2), None, _i32(3, 50))
    with pytest.raises(ValueError, match="start"):
        graft.graft_token_counts(_i32(2, 9), _i32(2), None, _i32(2, 50), start=_i32(3))
    x = torch.zeros((2, 3, 70))
    with pytest.raises(ValueError, match="GPU"):
        graft.graft_logits_adjust(x, _i32(2))
    for kw, what in ((dict(tokens=_i32(2, 4)), "tokens"), (dict(mask=_i32(2, 3, 2)), "mask"), (dict(counts=_i32(2, 71)), "counts"),
                     (dict(repetition=torch.zeros(3)), "repetition"), (dict(bias=torch.zeros(69)), "bias"), (dict(bias=torch.zeros(3, 70)), "bias"),
                     (dict(allow=_i32(4, 2)), "allow"), (dict(allow_index=_i32(2, 2)), "allow_index"), (dict(result=x.double()), "result")):
        with pytest.raises(ValueError, match=what):
            graft.graft_logits_adjust(x, _i32(2), **kw)
    with pytest.raises(ValueError):
        graft.graft_logits_adjust(x[0], _i32(2))
    with pytest.raises(ValueError, match="logits"):
        graft.graft_logits_adjust(x.double(), _i32(2))
