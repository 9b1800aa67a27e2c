"""graft_prompt_attn in the ways that programs call it: in place, over far and wide caches, on streams, captured, in pieces."""
import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from prompt_util import call, check, exact, make

pytestmark = pytest.mark.gpu


def _args(c):
    up = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()                                            # noqa: E731
    return dict(q=c["q"].cuda(), k_cache=c["k"].cuda(), v_cache=c["v"].cuda(), strides=c["strides"], block_table=c["table"].cuda(), prefix_len=up(c["P"]),
                n_nodes=up(c["n"]), Hkv=c["Hkv"], scale=c["scale"])


SHAPES = [("bf16", 1, 3, 8, 2, 64, 700), ("bf16", 2, 40, 8, 2, 128, 700), ("bf16", 2, 300, 8, 2, 128, 100), ("f32", 1, 2, 8, 2, 128, 700), ("f32", 1, 90, 8, 2, 64, 300)]


@pytest.mark.parametrize("shape", SHAPES)
def test_in_place(shape):
    c = make(3, *shape)
    a = _args(c)
    want = graft.graft_prompt_attn(**a)
    got = graft.graft_prompt_attn(**a, out=a["q"])
    assert got is a["q"] and torch.equal(got, want)


@pytest.mark.parametrize("shape", SHAPES)
def test_padded_rows_and_a_wide_table(shape):
    """More pages than the lengths need, whose numbers mean nothing; padding tokens whose queries are no numbers; rows of the output
    that held something."""
    dtype, B, T, Hq, Hkv, D, P = shape
    c = make(4, dtype, B, T, Hq, Hkv, D, P, n=[T - 1] * B)
    want = call(c)
    wide = torch.full((B, 3000), 0, dtype=torch.int32)
    wide[:, :c["pages"]] = c["table"]
    used = -(-int(c["P"][0] + T - 1) // 16)
    wide[:, used:] = 2 ** 31 - 1
    d = dict(c, table=wide, q=c["q"].clone())
    d["q"][:, T - 1:] = float("nan")
    out = torch.full_like(c["q"], 7).cuda()
    got = call(d, out=out)
    check(c, got)
    assert bool((got[:, T - 1:] == 0).all())
    assert torch.allclose(got.float(), want.float(), atol=0.02)


@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 200), ("f32", 1), ("f32", 60)])
def test_bad_lengths_give_zeros(dtype, T):
    c = make(5, dtype, 5, T, 4, 2, 64, 30)
    c["P"], c["n"] = np.array([30, -1, 30, 30, 16 * c["pages"]], np.int32), np.array([T, T, T + 1, -1, T], np.int32)
    got = call(c).float().cpu()
    assert bool((got[1:] == 0).all()) and bool(torch.isfinite(got[0]).all()) and bool((got[0] != 0).any())


@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 100), ("f32", 1), ("f32", 50)])
def test_offsets_past_32_bits(dtype, T):
    """Pages 2^29 elements apart and heads 2^27: the last one's elements are past 2^32, their bytes past 2^33."""
    c = make(6, dtype, 1, T, 4, 2, 64, 100)
    es = 4 if dtype == "f32" else 2
    page, head, n_pages = 1 << 29, 1 << 27, c["k"].shape[0]
    far = {}
    for x in "kv":
        big = torch.empty((n_pages - 1) * page + head + 1024, dtype=c["k"].dtype, device="cuda")
        for p in range(n_pages):
            for h in range(2):
                big[p * page + h * head:p * page + h * head + 1024] = c[x][p, h].reshape(-1).cuda()
        far[x] = big
    assert far["k"].numel() > 1 << 32 and far["k"].numel() * es > 1 << 33
    a = dict(_args(c), k_cache=far["k"], v_cache=far["v"], strides={"page": page, "token": 64, "head": head})
    check(c, graft.graft_prompt_attn(**a))


@pytest.mark.parametrize("shape", SHAPES)
def test_streams_and_repeats(shape):
    """Two streams at once, on tensors of the current one, twenty times: the same bits."""
    cases = [_args(make(s, *shape)) for s in (7, 8)]
    want = [graft.graft_prompt_attn(**a) for a in cases]
    outs = [[torch.empty_like(want[0]) for _ in range(20)] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for rep in range(20):
        for i in range(2):
            graft.graft_prompt_attn(**cases[i], out=outs[i][rep], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in outs[i])


@pytest.mark.parametrize("shape", SHAPES)
def test_captured(shape):
    """A graph's replays, with new queries and lengths in the same tensors and eager calls in between, against eager calls."""
    c = make(9, *shape)
    a = _args(c)
    out = torch.empty_like(a["q"])
    dtype = graft.GRAFT_F32 if shape[0] == "f32" else graft.GRAFT_BF16
    n = graft.graft_prompt_attn_workspace_bytes(c["B"], c["T"], c["Hq"], c["Hkv"], c["D"], c["pages"], 0, dtype)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graft.graft_prompt_attn(**a, out=out, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        graft.graft_prompt_attn(**a, out=out, workspace=ws)
    for rep in range(4):
        a["q"].copy_(torch.randn_like(a["q"]))
        a["prefix_len"].fill_(int(c["P"][0]) - 13 * rep)
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, graft.graft_prompt_attn(**a)), rep
    with pytest.raises(graft.GraftError):
        if n == 0:
            raise graft.GraftError("no workspace", 4)
        graft.graft_prompt_attn(**a, workspace=ws[:n - 16])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_make_the_whole(dtype):
    """A prompt in one piece, and in pieces of 1 to 300 tokens: each piece against 64 bits."""
    whole = make(11, dtype, 1, 700, 6, 2, 128, 0)
    check(whole, call(whole))
    at = 0
    for n in (1, 15, 1, 64, 300, 130, 189):
        piece = dict(whole, T=n, P=np.array([at], np.int32), n=np.array([n], np.int32), q=whole["q"][:, at:at + n].contiguous())
        check(piece, call(piece))
        at += n
    assert at == 700


def test_beside_the_tree_attention():
    """Chains of nodes through graft_tree_attn and as tokens of a prompt: the same rows, as near as either is to 64 bits."""
    c = make(12, "bf16", 2, 100, 16, 4, 128, [512, 33], n=[100, 57])
    a = _args(c)
    mask = np.zeros((2, 100, 2), np.uint64)
    for i in range(100):
        mask[:, i, 0] = (1 << min(i + 1, 64)) - 1
        mask[:, i, 1] = (1 << max(i - 63, 0)) - 1
    tree = graft.graft_tree_attn(**a, mask=torch.from_numpy(mask.view(np.int64)).cuda())
    check(c, graft.graft_prompt_attn(**a))
    assert float((tree.float() - call(c).float()).abs().max()) <= 2e-2
