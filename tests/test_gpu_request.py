"""A request from its prompt to its answer: prompt appended and attended in pieces, contexts counted, rules on the logits of every tree,
acceptance, counts of what was emitted; the answer is the one that decoding token by token under the same rules gives."""
import math

import numpy as np
import pytest
import torch

import paper_2605_20104_amd as graft
from gpu_util import dev
from mx_util import random_tree
from prompt_util import check, rows
from rules_util import adjusted, counts_of

pytestmark = pytest.mark.gpu

V, B, K, CAP, PROMPT, LONG = 611, 2, 17, 12, (29, 40), 110


class Model:
    """Logits that depend on the last two tokens, and a grammar of six states."""
    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.first, self.second = (rng.standard_normal((V, V)).astype(np.float32) * 3 for _ in range(2))
        self.bias = (rng.standard_normal(V) * (rng.random(V) < 0.05) * 3).astype(np.float32)
        self.next_state = rng.integers(0, 6, (6, V))
        allow = rng.random((6, V)) < np.array([1, 0.5, 0.02, 0.9, 0.1, 0.5])[:, None]
        allow[2, 7] = True                                 # (a state always allows something)
        words = np.zeros((6, (V + 31) // 32), np.uint32)
        for v in range(V):
            words[:, v // 32] |= allow[:, v].astype(np.uint32) << np.uint32(v % 32)
        self.allow = words.view(np.int32)
        self.params = {"repetition": np.array([1.3, 0.9], np.float32), "frequency": np.array([0.4, 0.7], np.float32),
                       "presence": np.array([0.2, -0.3], np.float32)}

    def logits(self, before, last):
        return self.first[last] + self.second[before]

    def state(self, tokens):
        s = 0
        for t in tokens:
            s = self.next_state[s, t]
        return s


def _greedy(model, b, context, prompt, count):
    """Token by token, on the host."""
    context, out = list(context), []
    for _ in range(count):
        c, _ = counts_of(np.array([context], np.int32), [len(context)], [prompt], V)
        state = model.state(context[prompt:])
        params = {k: v[b:b + 1] for k, v in model.params.items()}
        _, ids, _ = adjusted(model.logits(context[-2], context[-1])[None, None], [1], counts=c, bias=model.bias, allow=model.allow,
                             allow_index=np.array([[state]], np.int32), **params)
        context.append(int(ids[0, 0]))
        out.append(context[-1])
    return out


@pytest.mark.parametrize("in_place", [False, True])
def test_emitted_tokens_are_those_of_plain_decoding(in_place):
    model, rng = Model(3), np.random.default_rng(5)
    ctx = np.full((B, LONG + K), -1, np.int32)
    length = np.array(PROMPT, np.int32)
    for b in range(B):
        ctx[b, :length[b]] = rng.integers(0, V, length[b])
    want = [_greedy(model, b, ctx[b, :length[b]], PROMPT[b], LONG - max(PROMPT) + CAP + 1) for b in range(B)]
    prompt_len, counts = dev(np.array(PROMPT)), torch.empty((B, V), dtype=torch.int32, device="cuda")
    graft.graft_token_counts(dev(ctx), dev(length), prompt_len, counts)
    gpu = {k: torch.from_numpy(v).cuda() for k, v in model.params.items()}
    gpu.update(bias=torch.from_numpy(model.bias).cuda(), allow=torch.from_numpy(model.allow).cuda())
    accepted = 0
    while length.max() < LONG:
        # a draft tree: the root is the last token; children are often what greedy decoding will emit
        tokens, parent, n = np.zeros((B, K), np.int32), np.full((B, K), -1, np.int32), np.array([K, K - 5], np.int32)
        states, logits = np.full((B, K), -1, np.int32), np.zeros((B, K, V), np.float32)
        for b in range(B):
            up, depth = random_tree(rng, n[b])
            done = length[b] - PROMPT[b]
            tokens[b, 0], parent[b, :n[b]] = ctx[b, length[b] - 1], up
            paths = [[]]
            for i in range(1, n[b]):
                right = want[b][done + depth[i] - 1] if depth[i] <= len(want[b]) - done else 0
                tokens[b, i] = right if rng.random() < 0.8 else rng.integers(0, V)
                paths.append(paths[up[i]] + [int(tokens[b, i])])
            for i in range(n[b]):
                seq = list(ctx[b, :length[b]]) + paths[i]
                states[b, i] = model.state(seq[PROMPT[b]:])
                logits[b, i] = model.logits(seq[-2], seq[-1])
        mk = graft.graft_build_tree_mask(dev(parent), dev(n), dev(length - 1), 0, 0)
        x = torch.from_numpy(logits).cuda()
        adj = graft.graft_logits_adjust(x, dev(n), tokens=dev(tokens), mask=mk["mask"], counts=counts, allow_index=dev(states),
                                        result=x if in_place else None, **gpu)
        if in_place:                                       # the acceptance may scan the adjusted logits as well
            acc = graft.graft_accept(dev(parent), dev(tokens), dev(n), CAP, logits=x)
            assert torch.equal(acc["target_ids"], adj["target_ids"])
        else:
            acc = graft.graft_accept(dev(parent), dev(tokens), dev(n), CAP, target_ids=adj["target_ids"])
        graft.graft_token_counts(acc["out_tokens"], dev(np.full(B, CAP + 1)), None, counts, start=dev(np.zeros(B)))
        emitted, took = acc["out_tokens"].cpu().numpy(), acc["accept_len"].cpu().numpy()
        for b in range(B):
            new = emitted[b, :took[b] + 1]
            done = length[b] - PROMPT[b]
            assert list(new) == want[b][done:done + len(new)]
            ctx[b, length[b]:length[b] + len(new)] = new
            length[b] += len(new)
        accepted += int(took.sum())
        again, _ = counts_of(ctx, length, np.array(PROMPT), V)
        assert (counts.cpu().numpy() == again).all()
    assert accepted > 20                                   # the trees' paths were used


def test_prompt_in_pieces_then_a_tree():
    """Appends, prompt attention in pieces, then a tree over the same cache: the prompt's rows and a chain of the tree's against 64 bits."""
    g = torch.Generator().manual_seed(2)
    Hq, Hkv, D, T, pages = 8, 2, 128, 150, 12
    qkv = torch.randn((1, T, Hq + 2 * Hkv, D), generator=g).bfloat16().cuda()
    angle = np.arange(pages * 16)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    cos_sin = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).cuda()
    k, v = (torch.zeros((pages + 2, Hkv, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    strides, table = {"page": Hkv * 16 * D, "token": D, "head": 16 * D}, dev(np.random.default_rng(1).permutation(pages + 2)[None, :pages])
    queries, outs, at = [], [], 0
    for n in (70, 1, 59):                                  # a prompt, then a chain of 20 as a tree
        P, N = dev([at]), dev([n])
        x = qkv[:, at:at + n]
        app = graft.graft_kv_append(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], cos_sin, None, k, v, strides, table, P, N)
        queries.append(app["q"])
        outs.append(graft.graft_prompt_attn(app["q"], k, v, strides, table, P, N, Hkv, 1 / math.sqrt(D)))
        at += n
    n = T - at
    parent = np.arange(-1, n - 1, dtype=np.int32)[None]
    mk = graft.graft_build_tree_mask(dev(parent), dev([n]), dev([at]), 0, 0)
    x = qkv[:, at:]
    app = graft.graft_kv_append(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], cos_sin, mk["pos"], k, v, strides, table, dev([at]), dev([n]))
    queries.append(app["q"])
    tree = graft.graft_tree_attn(app["q"], k, v, strides, table, dev([at]), dev([n]), mk["mask"], Hkv, 1 / math.sqrt(D))
    outs.append(graft.graft_prompt_attn(app["q"], k, v, strides, table, dev([at]), dev([n]), Hkv, 1 / math.sqrt(D)))
    assert float((tree.float() - outs[-1].float()).abs().max()) <= 2e-2
    c = dict(dtype="bf16", B=1, T=T, Hq=Hq, Hkv=Hkv, D=D, P=np.zeros(1, np.int32), n=np.array([T]), layout="head", q=torch.cat(queries, 1).cpu(), k=k.cpu(),
             v=v.cpu(), table=table.cpu(), scale=1 / math.sqrt(D))
    check(c, torch.cat(outs, 1))
