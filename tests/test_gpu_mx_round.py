"""A decoding loop over a 4-bit cache: append, masks, attention, acceptance, cache update, as a serving program chains them;
eagerly against plain numpy, and captured in a graph against the eager run."""
import math

import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from gpu_util import dev, host
from mx_util import attention, dequantise, quantise, random_tree, rotate32, run_bytes

pytestmark = pytest.mark.gpu

B, K, Hq, Hkv, D, R, LAYERS, CAP = 2, 24, 8, 2, 128, 128, 2, 12
PAGES, PROMPT = 24, (37, 100)


def _cos_sin():
    angle = np.arange(PAGES * 16)[:, None] * 10000.0 ** (-np.arange(0, R, 2) / R)
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)


class Loop:
    def __init__(self, seed):
        self.rng = np.random.default_rng(seed)
        run, total = run_bytes(D), B * PAGES + 1
        self.strides, self.layer_stride = {"page": Hkv * run, "head": run}, total * Hkv * run
        self.cache = [torch.zeros((LAYERS, total, Hkv, run), dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.table = dev(self.rng.permutation(total)[:B * PAGES].reshape(B, PAGES))
        self.angles = _cos_sin()
        self.cos_sin = dev(self.angles, "f32")
        self.prefix = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.rows = [[[] for _ in range(B)] for _ in range(LAYERS)]       # (key, value) numbers of every token kept, per head

    def qkv(self, T):
        return torch.from_numpy(self.rng.standard_normal((LAYERS, B, T, Hq + 2 * Hkv, D)).astype(np.float32)).bfloat16()

    def append(self, qkv, l, pos, n, out=None):
        x = qkv[l]
        return graft.graft_kv_append_mx(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], self.cos_sin, pos, self.cache[0][l], self.cache[1][l], self.strides,
                                        self.table, self.prefix, n, out=out)

    def plain_rows(self, qkv, l, b, pos):
        x = qkv[l, b, :len(pos)].float().numpy()
        turned = rotate32(x[:, :Hq + Hkv], self.angles, pos, False)
        q = torch.from_numpy(turned[:, :Hq]).bfloat16().double().numpy()
        return q, dequantise(*quantise(turned[:, Hq:])), dequantise(*quantise(x[:, Hq + Hkv:]))


def _step(loop, qkv, parent, n, targets, tokens):
    mk = graft.graft_build_tree_mask(parent, n, loop.prefix, CAP + 1, CAP)
    outs = []
    for l in range(LAYERS):
        app = loop.append(qkv, l, mk["pos"], n)
        outs.append(graft.graft_tree_attn_mx(app["q"], loop.cache[0][l], loop.cache[1][l], loop.strides, loop.table, loop.prefix, n, mk["mask"], Hkv, 1 / math.sqrt(D),
                                             window=48 if l else 0, softcap=30.0 if l else 0.0, pos=mk["pos"]))
    acc = graft.graft_accept(parent, tokens, n, CAP, target_ids=targets)
    com = graft.graft_kv_compact_mx(*loop.cache, loop.layer_stride, LAYERS, loop.strides, loop.table, loop.prefix, acc["path"], acc["accept_len"], K, Hkv, D)
    return mk, outs, acc, com


def _tree(rng):
    parent, tokens, targets, n = np.full((B, K), -1, np.int32), rng.integers(0, 50, (B, K)).astype(np.int32), np.full((B, K), 99, np.int32), np.array([K, K - 5], np.int32)
    for b in range(B):
        p, _ = random_tree(rng, n[b], CAP)
        parent[b, :n[b]] = p
        node = 0
        while True:                                        # one path is accepted, as deep as it goes
            kids = [i for i in range(1, n[b]) if p[i] == node]
            if not kids:
                break
            node2 = kids[-1]
            targets[b, node] = tokens[b, node2] = 60 + node2
            node = node2
    return parent, tokens, targets, n


def test_loop_against_plain_arithmetic():
    loop = Loop(0)
    T = max(PROMPT)
    qkv = loop.qkv(T)
    gpu, n = qkv.cuda(), dev(PROMPT)
    for l in range(LAYERS):
        assert (host(loop.append(gpu, l, None, n)["status"]) == 0).all()
        for b in range(B):
            _, k, v = loop.plain_rows(qkv, l, b, np.arange(PROMPT[b]))
            loop.rows[l][b] = [(k[i], v[i]) for i in range(PROMPT[b])]
    loop.prefix = n.clone()
    for step in range(4):
        parent, tokens, targets, n = _tree(loop.rng)
        qkv = loop.qkv(K)
        P = host(loop.prefix)
        mk, outs, acc, com = _step(loop, qkv.cuda(), dev(parent), dev(n), dev(targets), dev(tokens))
        pos, path, a = host(mk["pos"]), host(acc["path"]), host(acc["accept_len"])
        assert (a >= 1).all() and (host(com["status"]) == 0).all()
        bits = host(mk["mask"])
        for l in range(LAYERS):
            for b in range(B):
                q, k, v = loop.plain_rows(qkv, l, b, pos[b, :n[b]])
                see = np.concatenate([np.ones((n[b], P[b]), bool), ((bits[b, :n[b], 0][:, None] >> np.arange(n[b], dtype=np.uint64)) & np.uint64(1)).astype(bool)], 1)
                place = np.concatenate([np.arange(P[b]), pos[b, :n[b]]])
                if l:
                    see &= pos[b, :n[b], None] - place[None] < 48
                for g in range(Hkv):
                    keys = np.array([x[0][g] for x in loop.rows[l][b]] + list(k[:, g]))
                    vals = np.array([x[1][g] for x in loop.rows[l][b]] + list(v[:, g]))
                    G = Hq // Hkv
                    want, tol = attention(q[:, g * G:(g + 1) * G], keys, vals, see, 1 / math.sqrt(D), 30.0 if l else 0.0)
                    got = outs[l][b, :n[b], g * G:(g + 1) * G].double().cpu().numpy()
                    assert (abs(got - want) <= tol).all(), (step, l, b, g)
                kept = path[b, :a[b] + 1]
                loop.rows[l][b] += [(k[i], v[i]) for i in kept]
        assert (host(com["new_prefix_len"]) == P + a + 1).all()
        loop.prefix = com["new_prefix_len"]
    # what the cache holds at the end is what was kept
    n = loop.prefix
    back = graft.graft_kv_gather_mx(*loop.cache, loop.layer_stride, LAYERS, loop.strides, loop.table, None, n, int(n.max()), Hkv, D)
    for l in range(LAYERS):
        for b in range(B):
            for name, i in (("k", 0), ("v", 1)):
                want = np.array([x[i] for x in loop.rows[l][b]])
                assert np.array_equal(back[name][l, b, :len(want)].double().cpu().numpy(), want)


def test_captured_steps_replay():
    """The step in a graph, replayed with new rows and lengths in between eager work, against the same steps run eagerly."""
    eager, graphed = Loop(3), Loop(3)
    assert torch.equal(eager.table, graphed.table)
    trees = [_tree(eager.rng) for _ in range(4)]
    rows = [eager.qkv(K).cuda() for _ in range(4)]
    static = [torch.empty_like(rows[0])] + [torch.empty((B, K), dtype=torch.int32, device="cuda") for _ in range(3)] + [torch.empty(B, dtype=torch.int32, device="cuda")]

    def fill(i):
        parent, tokens, targets, n = trees[i]
        static[0].copy_(rows[i])
        for t, x in zip(static[1:], (parent, tokens, targets, n)):
            t.copy_(dev(x))
    fill(0)
    keep = [x.clone() for x in graphed.cache]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run = lambda: _step(graphed, static[0], static[1], static[4], static[3], static[2])
    with torch.cuda.stream(side):
        run()                                              # (warm up)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(graphed.cache, keep):
        x.copy_(y)
    graphed.prefix.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for i in range(4):
        parent, tokens, targets, n = trees[i]
        want = _step(eager, rows[i], dev(parent), dev(n), dev(targets), dev(tokens))
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want[1], captured[1]):
            assert torch.equal(x, y)
        assert torch.equal(want[3]["new_prefix_len"], captured[3]["new_prefix_len"])
        for x, y in zip(eager.cache, graphed.cache):
            assert torch.equal(x, y)
        eager.prefix = want[3]["new_prefix_len"]
        graphed.prefix.copy_(captured[3]["new_prefix_len"])
