"""graft_token_counts and graft_logits_adjust, bit for bit, against plain numpy."""
import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from mx_util import random_tree
from rules_util import PROMPT, adjusted, counts_of

pytestmark = pytest.mark.gpu


def up(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def same(a, b):
    """Equal, NaN where NaN is."""
    return bool(((a == b) | (np.isnan(a) & np.isnan(b))).all())


# ---- counts
@pytest.mark.parametrize("B,L,V", [(1, 1, 1), (1, 5, 3), (3, 301, 1000), (2, 1023, 8192), (2, 700, 8193), (4, 2050, 50257), (1, 9000, 20000)])
@pytest.mark.parametrize("prompts", [True, False])
def test_counts_anew(B, L, V, prompts):
    rng = np.random.default_rng(L + V)
    ctx = rng.integers(-2, V + 2, (B, L)).astype(np.int32)
    ctx[:, ::3] = ctx[:, :1]                               # one token many times
    n = rng.integers(0, L + 1, B).astype(np.int32)
    n[0] = L
    prompt = rng.integers(-1, L + 2, B).astype(np.int32) if prompts else None
    got = torch.full((B, V), 77, dtype=torch.int32, device="cuda")
    status = graft.graft_token_counts(up(ctx), up(n), up(prompt), got)
    want, st = counts_of(ctx, n, prompt, V)
    assert (got.cpu().numpy() == want).all() and (status.cpu().numpy() == st).all()


def test_counts_added_round_by_round():
    rng = np.random.default_rng(3)
    B, L, V = 3, 400, 500
    ctx = rng.integers(0, V, (B, L)).astype(np.int32)
    prompt = np.array([100, 0, 50], np.int32)
    length = np.array([100, 10, 50], np.int32)
    counts = torch.zeros((B, V), dtype=torch.int32, device="cuda")
    graft.graft_token_counts(up(ctx), up(length), up(prompt), counts)
    for _ in range(12):
        start, length = length, np.minimum(length + rng.integers(0, 9, B), L).astype(np.int32)
        status = graft.graft_token_counts(up(ctx), up(length), up(prompt), counts, start=up(start))
        assert (status.cpu().numpy() == 0).all()
        assert (counts.cpu().numpy() == counts_of(ctx, length, prompt, V)[0]).all()


def test_counts_of_what_was_accepted():
    """out_tokens of graft_accept, with their padding of -1; a token that occurs more than once."""
    out_tokens = np.array([[5, 5, 9, -1, -1], [2, -1, -1, -1, -1]], np.int32)
    counts = np.zeros((2, 12), np.int32)
    counts[0, 5] = PROMPT
    counts[1, 2] = PROMPT + 3
    got = up(counts)
    graft.graft_token_counts(up(out_tokens), up(np.array([5, 5], np.int32)), None, got, start=up(np.zeros(2, np.int32)))
    counts[0, 5] += 2
    counts[0, 9] += 1
    counts[1, 2] += 1
    assert (got.cpu().numpy() == counts).all()


@pytest.mark.parametrize("added", [True, False])
def test_counts_of_bad_lengths(added):
    ctx = np.array([[1, 2, 3], [1, 2, 3], [1, 2, 3], [1, 2, 3]], np.int32)
    n, start = np.array([4, -1, 2, 3], np.int32), np.array([0, 0, 3, 1], np.int32)
    before = np.arange(20, dtype=np.int32).reshape(4, 5)
    got = up(before)
    status = graft.graft_token_counts(up(ctx), up(n), None, got, start=up(start) if added else None)
    want, st = counts_of(ctx, n, None, 5, start if added else None, before)
    assert (status.cpu().numpy() == st).all() and (got.cpu().numpy() == want).all()
    assert list(st) == ([1, 1, 1, 0] if added else [1, 1, 0, 0])


# ---- rules
def _case(seed, B, K, V, n=None, paths=True, counts=True, params="rfp", bias=0, states=0, special=False):
    rng = np.random.default_rng(seed)
    f = np.float32
    c = dict(logits=(rng.standard_normal((B, K, V)) * 4).astype(f), n_nodes=np.array([K] * B if n is None else n, np.int32))
    if paths:
        c["tokens"] = rng.integers(0, V, (B, K)).astype(np.int32)
        c["tokens"][:, 1::2] = c["tokens"][:, 1:2]         # the same token several times on a path
        if K > 3:
            c["tokens"][:, 2], c["tokens"][0, 3] = V - 1, 0
        mask = np.zeros((B, K, 2), np.uint64)
        for b in range(B):
            parent = np.asarray(random_tree(rng, K)[0])
            for i in range(K):
                if i:
                    mask[b, i] = mask[b, parent[i]]
                mask[b, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
        c["mask"] = mask
    if counts:
        x = rng.integers(0, 4, (B, V)).astype(np.int32)
        x[rng.random((B, V)) < 0.8] = 0
        x[rng.random((B, V)) < 0.1] |= PROMPT
        c["counts"] = x
    for key, name, lo, hi in (("r", "repetition", 0.7, 1.8), ("f", "frequency", -0.5, 1.5), ("p", "presence", -1.0, 1.0)):
        if key in params:
            c[name] = rng.uniform(lo, hi, B).astype(f)
    if bias:
        c["bias"] = (rng.standard_normal((V,) if bias == 1 else (B, V)) * 2).astype(f)
    if states:
        W = (V + 31) // 32
        allow = rng.integers(0, 2 ** 32, (states, W), dtype=np.uint64).astype(np.uint32)
        allow[0] = 0                                       # allows nothing
        if states > 1:
            allow[1] = 0
            allow[1, (V - 1) // 32] = np.uint32(1) << np.uint32((V - 1) % 32)      # the last token only
        c["allow"] = allow.view(np.int32)
        c["allow_index"] = rng.integers(-1, states, (B, K)).astype(np.int32)
        c["allow_index"].flat[:min(states, B * K)] = np.arange(min(states, B * K))
    if special:
        x = c["logits"]
        x[0, 0, :] = -np.inf
        x[0, 1, V // 2], x[0, 1, 0] = np.nan, np.nan
        x[0, 2, 1] = np.inf
        x[0, 3, :] = np.nan
        x[0, 4, V - 1], x[0, 4, V // 3], x[0, 4, : V // 3] = 9.0, 9.0, 0.0         # equal maxima
        x[0, 5, :] = np.where(np.arange(V) % 2 == 0, -0.0, 0.0)
        x[0, 6, :] = 1e-41                                 # below the normal numbers
        x[0, 7, :] = 3e38
    return c


def _check(c, write="apart"):
    want, ids, st = adjusted(**c)
    gpu = {k: up(v.view(np.int64) if k == "mask" else v) for k, v in c.items()}
    if write == "none":
        got = graft.graft_logits_adjust(**gpu)
        assert same(gpu["logits"].cpu().numpy(), c["logits"])
    else:
        result = gpu["logits"] if write == "in place" else gpu["logits"].clone()
        got = graft.graft_logits_adjust(**gpu, result=result)
        assert same(result.cpu().numpy(), want)
    assert (got["status"].cpu().numpy() == st).all()
    assert (got["target_ids"].cpu().numpy() == ids).all()


@pytest.mark.parametrize("write", ["none", "apart", "in place"])
@pytest.mark.parametrize("B,K,V,options", [
    (1, 1, 1, dict(paths=False)), (1, 1, 3, dict(paths=False, bias=1, states=1)), (2, 3, 7, dict(states=3)), (1, 8, 33, dict(bias=1, states=4)),
    (3, 5, 1000, dict(bias=2, states=6)), (2, 33, 1001, dict(n=[33, 20])), (1, 128, 4099, dict(states=9, bias=1)), (2, 4, 32000, dict(params="r")),
    (1, 2, 50257, dict(params="fp", bias=1, states=3)), (2, 6, 50257, dict(params="", bias=2, states=2)), (1, 5, 30011, dict(counts=False, bias=1)),
    (4, 1, 16384, dict(paths=False, states=5)), (1, 3, 151936, dict(states=5, bias=1)), (1, 1, 600001, dict(paths=False, bias=1, states=2)),
    (2, 9, 517, dict(params="", counts=False)), (1, 12, 2048, dict(special=True)), (1, 12, 2049, dict(special=True, bias=1, params="p")),
])
def test_rules(B, K, V, options, write):
    _check(_case(K + V, B, K, V, **options), write)


def test_padding_bad_trees_and_bad_states():
    c = _case(1, 4, 6, 1000, n=[6, 0, 7, 2], states=4)
    c["allow_index"][0, 2], c["allow_index"][0, 3], c["allow_index"][3, 4] = 4, -2, 99       # the last one is padding
    c["tokens"][0, 4] = -1                                 # a node that no vocabulary has
    c["tokens"][3, 1] = 1000
    _check(c, "apart")
    assert list(adjusted(**c)[2]) == [1, 2, 2, 0]


def _gpu(c):
    return {k: up(v.view(np.int64) if k == "mask" else v) for k, v in c.items()}


def test_odd_parameters():
    """Repetitions that a quotient by reciprocal does not take, zero, negative, no numbers; frequencies that are no numbers."""
    for r in (0.0, -2.0, 1e-30, 1e30, np.inf, np.nan, 1.0):
        c = _case(41, 2, 5, 3001, bias=1)
        c["repetition"][:] = r
        _check(c, "apart")
    for f in (np.inf, np.nan, 1e38):
        c = _case(42, 2, 5, 3001)
        c["frequency"][0], c["presence"][1] = f, f
        _check(c, "apart")


def test_counts_that_fill_their_bits():
    c = _case(43, 1, 4, 1000)
    c["counts"][0, :4] = [2 ** 31 - 1, -1, PROMPT, 2 ** 24 + 1]
    c["tokens"][0, 1:] = [0, 1, 5]
    c["counts"][0, 0] = 2 ** 31 - 2                        # one more on the path fits
    _check(c, "apart")


def test_rows_of_any_address():
    """Logits, results, counts and biases that start 4 bytes past a 16-byte boundary."""
    c = _case(44, 2, 3, 1003, bias=2, states=3)
    want, ids, st = adjusted(**c)
    gpu = _gpu(c)
    for x in ("logits", "counts", "bias", "allow"):
        base = torch.empty(gpu[x].numel() + 1, dtype=gpu[x].dtype, device="cuda")
        base[1:] = gpu[x].flatten()
        gpu[x] = base[1:].view(gpu[x].shape)
    result = torch.empty(want.size + 3, device="cuda")[3:].view(want.shape)
    result.copy_(gpu["logits"])
    got = graft.graft_logits_adjust(**gpu, result=result)
    assert same(result.cpu().numpy(), want) and (got["target_ids"].cpu().numpy() == ids).all()


def test_streams_repeats_and_graphs():
    """Two streams at once, and a graph's replays with eager calls in between: the bits of a single call."""
    cases = [_case(s, 2, 20, 20011, bias=1, states=4) for s in (45, 46)]
    wants, gpus = [adjusted(**c) for c in cases], [_gpu(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = [[torch.empty_like(g["logits"]) for _ in range(10)] for g in gpus]
    outs = [[None] * 10 for _ in range(2)]
    torch.cuda.synchronize()
    for rep in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                outs[i][rep] = graft.graft_logits_adjust(**gpus[i], result=results[i][rep], stream=streams[i])
    torch.cuda.synchronize()
    live = lambda x, c: np.concatenate([x[b, :n].ravel() for b, n in enumerate(c["n_nodes"])])              # noqa: E731
    for i in range(2):
        for rep in range(10):
            assert same(live(results[i][rep].cpu().numpy(), cases[i]), live(wants[i][0], cases[i]))
            assert (outs[i][rep]["target_ids"].cpu().numpy() == wants[i][1]).all()
    gpu, (B, K, V) = gpus[0], gpus[0]["logits"].shape
    out = {"target_ids": torch.zeros((B, K), dtype=torch.int32, device="cuda"), "status": torch.zeros(B, dtype=torch.int32, device="cuda")}
    ws = torch.empty(graft.graft_logits_adjust_workspace_bytes(B, K, V), dtype=torch.uint8, device="cuda")
    ctx, n, counts = up(np.arange(300, dtype=np.int32).reshape(2, 150)), up(np.array([150, 20], np.int32)), gpu["counts"]

    def step():
        graft.graft_token_counts(ctx, n, n, counts, status=out["status"])
        graft.graft_token_counts(ctx, n, None, counts, start=up0, status=out["status"])
        graft.graft_logits_adjust(**gpu, result=results[0][0], out=out, workspace=ws)
    up0 = up(np.zeros(2, np.int32))
    step()
    torch.cuda.synchronize()
    eager = [results[0][0].clone(), out["target_ids"].clone(), counts.clone()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=streams[0]):
        step()
    for _ in range(4):
        results[0][0].zero_()
        out["target_ids"].zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(results[0][0], eager[0]) and torch.equal(out["target_ids"], eager[1]) and torch.equal(counts, eager[2])
        step()
        torch.cuda.synchronize()


def test_many_rows():
    """Several rows a workgroup, in the last of them fewer; trees of every length."""
    c = _case(47, 8, 48, 9001, n=[48, 47, 33, 1, 8, 9, 17, 16], bias=1, states=5)
    _check(c, "apart")
    _check(c, "none")
