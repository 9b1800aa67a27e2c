"""What a request needs before and behind its trees: attention of its prompt over the paged cache, and its rules on the
logits (penalties, biases, grammar masks), as cases whose time can be measured.

Three kinds of work, each through the package's public calls (`own`) or in plain torch operations:

  prompt   graft_prompt_attn: causal attention of a piece of a prompt, of one token or of thousands, over the paged cache that
           holds what came before it and the piece itself; optionally with capped scores and a window of the last positions.
  rules    graft_logits_adjust: penalties for tokens that the context or a node's path holds, biases and grammar masks on
           the logits of a tree's nodes, the greedy token of each, and where they are asked for the adjusted logits.
  counts   graft_token_counts: how often each token of the vocabulary occurs in the sequences' context buffers.

An entry of the counts has its top bit set where the token is in the prompt, and the number of its later occurrences below.
A mask of the grammar is a row of bits, bit v % 32 of word v / 32 for token v; a node names the row that holds for it.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
LATER = 0x7FFFFFFF


def listed():
    att = dict(kind="prompt", dtype="bf16", D=128, layout="head_major", ragged=False, cap=0.0, window=0)
    rule = dict(kind="rules", ragged=False, counts=True, bias=True, states=0, write=False)
    return [
        # One token of a toy model in float32: launches and latency.
        dict(att, name="prompt_token_f32", dtype="f32", B=1, T=1, Hq=8, Hkv=2, D=64, P=255),
        # Plain decoding of a serving batch, one token each over up to 16K: the cache is read once.
        dict(att, name="prompt_tokens", B=32, T=1, Hq=32, Hkv=8, P=16384, ragged=True),
        # A prompt of 4096 tokens of an 8B-class model, from an empty cache.
        dict(att, name="prompt_whole", B=1, T=4096, Hq=32, Hkv=8, P=0),
        # Four prompts behind a shared system prompt of odd length, head size 64 and the other cache layout.
        dict(att, name="prompt_ragged_64", B=4, T=2049, Hq=32, Hkv=8, D=64, P=301, layout="token_major", ragged=True),
        # A piece of 1024 tokens behind 32K that are in the cache already, 40 query and 8 KV heads: the largest.
        dict(att, name="prompt_piece_long", B=1, T=1024, Hq=40, Hkv=8, P=32768),
        # A layer of a model that caps its scores and looks back 4096 positions.
        dict(att, name="prompt_capped_window", B=2, T=2001, Hq=16, Hkv=8, P=6007, ragged=True, cap=50.0, window=4096),
        # float32 storage and arithmetic (validating a model against its float32 reference).
        dict(att, name="prompt_f32", dtype="f32", B=1, T=1000, Hq=32, Hkv=8, P=2001),
        # One token of a toy model with penalties: latency.
        dict(rule, name="rules_token", B=1, K=1, V=32000, L=301),
        # Ragged trees of three requests under a grammar, with penalties and a bias, a vocabulary of odd size; the greedy
        # tokens go to the acceptance.
        dict(rule, name="rules_tree", B=3, K=40, V=50257, L=1001, ragged=True, states=12),
        # The trees of a serving batch, everything on, the adjusted logits written.
        dict(rule, name="rules_batch", B=8, K=48, V=151936, L=8192, states=40, write=True),
        # The context of one request counted: latency.
        dict(name="counts_request", kind="counts", B=1, L=2048, V=32000, ragged=False),
        # The contexts of a serving batch counted, up to 16K tokens each.
        dict(name="counts_batch", kind="counts", B=16, L=16384, V=151936, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "rules", "rules", "counts"])
    c = dict(kind=kind, B=_log_int(rng, 1, 32), ragged=rng.random() < 0.5)
    if kind == "prompt":
        Hkv = rng.choice([1, 2, 3, 4, 8])
        c.update(dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), D=rng.choice([128, 128, 64]), Hkv=Hkv, Hq=Hkv * rng.randint(1, 16),
                 T=rng.choice([1, rng.randint(2, 128), _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)]),
                 P=rng.choice([0, _log_int(rng, 1, 65536), _log_int(rng, 1, 65536)]), layout=rng.choice(["head_major", "token_major"]),
                 cap=rng.choice([0.0, 0.0, 30.0]), window=rng.choice([0, 0, _log_int(rng, 1, 8192)]))
        most = 2.5e10 if c["dtype"] == "f32" else 3e11
        while (work(dict(c, window=0))["flops"] > most or c["B"] * Hkv * (c["P"] + c["T"]) * c["D"] > 3e8 or
               c["B"] * c["Hq"] * c["T"] * (c["P"] + c["T"]) > 1.2e9):
            c["B"], c["T"], c["P"] = max(1, c["B"] // 2), max(1, c["T"] * 2 // 3), c["P"] * 2 // 3
        return c
    c.update(V=rng.choice([_log_int(rng, 1000, 160000), 8 * _log_int(rng, 1000, 20000)]), L=_log_int(rng, 16, 32768))
    if kind == "rules":
        c.update(K=rng.choice([1, rng.randint(2, 128), rng.randint(2, 128)]), counts=rng.random() < 0.8, bias=rng.random() < 0.5,
                 states=rng.choice([0, 1, rng.randint(2, 60)]), write=rng.random() < 0.5)
        while c["B"] * c["K"] * c["V"] > 5.5e7:
            c["B"], c["K"] = max(1, c["B"] // 2), max(1, c["K"] * 2 // 3)
    return c


# ---------------------------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------------------------
def _lengths(c):
    """(tokens in front, new tokens or nodes) per sequence; a ragged batch has lengths down to about half."""
    P, new = c.get("P", 0), c["T"] if "T" in c else c.get("K", 1)
    out = []
    for b in range(c["B"]):
        if c["ragged"]:
            out.append((P - (b * 997) % (P // 2 + 1), new - (b * 7 + 3) % (new // 2 + 1)))
        else:
            out.append((P, new))
    return out


def _contexts(c):
    """(tokens in the context, those of them that are the prompt) per sequence."""
    out = []
    for b in range(c["B"]):
        n = c["L"] - (b * 131) % (c["L"] // 2 + 1) if c["ragged"] else c["L"]
        out.append((n, n * 3 // 4))
    return out


def work(c):
    if c["kind"] == "counts":
        return {"bytes": 4.0 * sum(n for n, _ in _contexts(c)) + 4.0 * c["B"] * c["V"], "flops": 0.0}
    if c["kind"] == "rules":
        V, rows = c["V"], sum(n for _, n in _lengths(c))
        shared = c["B"] * V * 4.0 * c["counts"] + V * 4.0 * c["bias"] + c["states"] * V / 8.0
        return {"bytes": rows * V * 4.0 * (2 if c["write"] else 1) + shared, "flops": 0.0}
    e = 2 if c["dtype"] == "bf16" else 4
    nbytes, pairs = 0.0, 0.0
    for P, n in _lengths(c):
        w = c["window"] if c["window"] else P + n
        first = max(0, P + 1 - w)                              # the first key that the first token sees
        nbytes += 2.0 * (P + n - first) * c["Hkv"] * c["D"] * e + (n + c["T"]) * c["Hq"] * c["D"] * e + 4 * ((P + n - first + PAGE - 1) // PAGE)
        grown = max(0, min(n, w - P))                          # tokens that see everything in front of them
        pairs += grown * P + grown * (grown + 1) / 2.0 + float(n - grown) * w
    return {"bytes": nbytes, "flops": 4.0 * c["D"] * c["Hq"] * pairs}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _normal(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _zipf(g, shape, V):
    """Token ids, the frequent ones spread over the vocabulary."""
    u = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)
    return ((torch.pow(float(V), u).long() - 1).clamp(0, V - 1) * 7919 % V).int()


def _trees(rng, c):
    """Parents of random trees, chains of about 8 below the first nodes: ancestor masks [B,K,2]."""
    B, K = c["B"], c["K"]
    mask, depth = np.zeros((B, K, 2), np.uint64), np.full((B, K), -1, np.int64)
    for b, (_, n) in enumerate(_lengths(c)):
        for i in range(n):
            up = -1 if i == 0 else i - 1 if rng.random() < 0.5 and depth[b, i - 1] < 12 else int(rng.integers(0, (i + 1) // 2))
            depth[b, i] = 0 if i == 0 else depth[b, up] + 1
            if i:
                mask[b, i] = mask[b, up]
            mask[b, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return mask


def _bits(allowed):
    """Truth values [S,V] as rows of 32-bit words."""
    S, V = allowed.shape
    full = torch.zeros((S, (V + 31) // 32 * 32), dtype=torch.int64, device="cuda")
    full[:, :V] = allowed
    words = (full.view(S, -1, 32) << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(words > LATER, words - (1 << 32), words).int()


def prepare(c, seed):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    B = c["B"]
    s = dict(c=c)
    if c["kind"] == "prompt":
        Hkv, D, lengths, total = c["Hkv"], c["D"], _lengths(c), c["P"] + c["T"]
        dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        pages = (total + PAGE - 1) // PAGE
        n_pages = B * pages + 3
        s.update(prefix_len=_up([P for P, _ in lengths]), n_nodes=_up([n for _, n in lengths]))
        s["block_table"] = _up(rng.permutation(n_pages)[:B * pages].reshape(B, pages))
        s["q"] = _normal(g, (B, c["T"], c["Hq"], D), dtype)
        shape = (n_pages, Hkv, PAGE, D) if c["layout"] == "head_major" else (n_pages, PAGE, Hkv, D)
        s["strides"] = ({"page": Hkv * PAGE * D, "token": D, "head": PAGE * D} if c["layout"] == "head_major"
                        else {"page": Hkv * PAGE * D, "token": Hkv * D, "head": D})
        s["k_cache"], s["v_cache"] = _normal(g, shape, dtype), _normal(g, shape, dtype)
        s["out"] = torch.zeros_like(s["q"])
        return s
    V, contexts = c["V"], _contexts(c)
    ctx, ctx_len, prompt_len = _zipf(g, (B, c["L"]), V), _up([n for n, _ in contexts]), _up([p for _, p in contexts])
    if c["kind"] == "counts":
        s.update(ctx=ctx, ctx_len=ctx_len, prompt_len=prompt_len, counts=torch.zeros((B, V), dtype=torch.int32, device="cuda"))
        return s
    K = c["K"]
    s["n_nodes"] = _up([n for _, n in _lengths(c)])
    s["logits"] = _normal(g, (B, K, V)).mul_(3.0)
    s["tokens"] = s["mask"] = None
    if K > 1:
        s["mask"] = torch.from_numpy(_trees(rng, c).view(np.int64)).cuda()
        # a draft's tokens are much like the context's
        s["tokens"] = torch.gather(ctx, 1, torch.randint(0, c["L"], (B, K), generator=g, device="cuda"))
    s["counts"] = s["repetition"] = s["frequency"] = s["presence"] = s["bias"] = s["allow"] = s["allow_index"] = None
    if c["counts"]:
        s["counts"] = _plain_counts(dict(c=c, ctx=ctx, ctx_len=ctx_len, prompt_len=prompt_len, counts=torch.zeros((B, V), dtype=torch.int32, device="cuda")))
        s["repetition"] = 1.0 + 0.3 * torch.rand((B,), generator=g, device="cuda")
        s["frequency"] = 0.7 * torch.rand((B,), generator=g, device="cuda")
        s["presence"] = 0.5 * torch.rand((B,), generator=g, device="cuda")
    if c["bias"]:
        # a few tokens pushed, a few nearly forbidden
        s["bias"] = torch.zeros((V,), device="cuda")
        s["bias"][torch.randint(0, V, (50,), generator=g, device="cuda")] = _normal(g, (50,)).mul_(4.0)
        s["bias"][torch.randint(0, V, (50,), generator=g, device="cuda")] = -100.0
    if c["states"]:
        # states of a grammar: free text, a few tokens, about half; one that ends here and allows nothing
        kind = torch.arange(c["states"], device="cuda") % 4
        p = torch.tensor([0.97, 0.0005, 0.5, 0.0], device="cuda")[kind]
        s["allow"] = _bits(torch.rand((c["states"], V), generator=g, device="cuda") < p[:, None])
        s["allow_index"] = torch.randint(-1, c["states"], (B, K), generator=g, device="cuda").int()
    s["result"] = torch.zeros_like(s["logits"]) if c["write"] else None
    s["out"] = {x: torch.zeros(shape, dtype=torch.int32, device="cuda") for x, shape in (("target_ids", (B, K)), ("status", (B,)))}
    return s


# ---------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------
def _plain_prompt(s):
    c = s["c"]
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    table = s["block_table"].long()
    pages = [s[x][table] if c["layout"] == "head_major" else s[x][table].transpose(2, 3) for x in ("k_cache", "v_cache")]      # [B,pages,Hkv,16,D]
    k, v = (x.transpose(1, 2).flatten(2, 3).float() for x in pages)                                                          # [B,Hkv,tokens,D]
    t, i = torch.arange(k.shape[2], device="cuda")[None, None], torch.arange(T, device="cuda")[None, :, None]
    P, n = s["prefix_len"].long()[:, None, None], s["n_nodes"].long()[:, None, None]
    seen = (i < n) & (t <= P + i)
    if c["window"]:
        seen &= t > P + i - c["window"]
    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).flatten(2, 3)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(1 / math.sqrt(D))
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    x = x.view(B, Hkv, T, Hq // Hkv, -1).masked_fill_(~seen[:, None, :, None], -math.inf).flatten(2, 3)
    x = x.sub_(x.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, v) / torch.where(total > 0, total, 1.0)
    return out.view(B, Hkv, T, Hq // Hkv, D).permute(0, 2, 1, 3, 4).flatten(2, 3).to(s["q"].dtype)


def _plain_counts(s):
    B, V = s["counts"].shape
    at = torch.arange(s["ctx"].shape[1], device="cuda")[None]
    place = s["ctx"].long() + V * torch.arange(B, device="cuda")[:, None]
    prompt, later = at < s["prompt_len"][:, None], (at >= s["prompt_len"][:, None]) & (at < s["ctx_len"][:, None])
    flat = torch.zeros((B * V,), dtype=torch.int32, device="cuda")
    flat.index_add_(0, place[later], torch.ones((), dtype=torch.int32, device="cuda").expand(int(later.sum())))
    flat[place[prompt]] |= -LATER - 1
    return s["counts"].copy_(flat.view(B, V))


def _live(s):
    return torch.arange(s["c"]["K"], device="cuda")[None] < s["n_nodes"][:, None]


def _plain_rules(s):
    c = s["c"]
    B, K, V = c["B"], c["K"], c["V"]
    x = s["logits"]
    later = torch.zeros((B, K, V), dtype=torch.int32, device="cuda") if s["counts"] is None else (s["counts"] & LATER)[:, None].repeat(1, K, 1)
    if K > 1:
        # nodes below the root on the path of node i, itself among them
        j = torch.arange(K, device="cuda")
        on = ((s["mask"][:, :, j // 64] >> (j % 64)) & 1).bool() & (j > 0) & _live(s)[:, :, None]
        b, i, j = torch.nonzero(on, as_tuple=True)
        later.view(-1).index_add_(0, (b * K + i) * V + s["tokens"].long()[b, j], torch.ones((), dtype=torch.int32, device="cuda").expand(len(b)))
    row = lambda name: s[name][:, None, None]                                                                                # noqa: E731
    if s["repetition"] is not None:
        r = row("repetition")
        x = torch.where((later > 0) | (s["counts"] < 0)[:, None], torch.where(x > 0, x / r, x * r), x)
        x = torch.where(later > 0, (x - later.float() * row("frequency")) - row("presence"), x)
    if s["bias"] is not None:
        x = x + s["bias"]
    if s["allow"] is not None:
        v = torch.arange(V, device="cuda")
        allowed = ((s["allow"][:, v // 32] >> (v % 32)) & 1).bool()
        index = s["allow_index"].long()
        x = torch.where((index < 0)[..., None] | allowed[index.clamp(min=0)], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    ids = torch.where(x == top, torch.arange(V, device="cuda", dtype=torch.int32), V).amin(-1)
    ids = torch.where(_live(s) & (top[..., 0] > -math.inf), ids, -1).int()
    out = {"target_ids": s["out"]["target_ids"].copy_(ids)}
    if s["result"] is not None:
        out["logits"] = s["result"].copy_(torch.where(_live(s)[..., None], x, s["result"]))
    return out


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(s):
    c = s["c"]
    if not own:
        return {"prompt": _plain_prompt, "rules": _plain_rules, "counts": _plain_counts}[c["kind"]](s)
    import paper_2605_20104_amd as graft
    if c["kind"] == "prompt":
        return graft.graft_prompt_attn(s["q"], s["k_cache"], s["v_cache"], s["strides"], s["block_table"], s["prefix_len"], s["n_nodes"], c["Hkv"],
                                       1 / math.sqrt(c["D"]), softcap=c["cap"], window=c["window"], out=s["out"])
    if c["kind"] == "counts":
        graft.graft_token_counts(s["ctx"], s["ctx_len"], s["prompt_len"], s["counts"])
        return s["counts"]
    out = graft.graft_logits_adjust(s["logits"], s["n_nodes"], tokens=s["tokens"], mask=s["mask"], counts=s["counts"], repetition=s["repetition"],
                                    frequency=s["frequency"], presence=s["presence"], bias=s["bias"], allow=s["allow"],
                                    allow_index=s["allow_index"], result=s["result"], out=s["out"])
    return {"target_ids": out["target_ids"]} if s["result"] is None else {"target_ids": out["target_ids"], "logits": s["result"]}


# ---------------------------------------------------------------------------------------------
# from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_prompt(s, c):
    G = c["Hq"] // c["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (P, n) in enumerate(_lengths(c)):
        t = torch.arange(P + n, device="cuda")
        page, at = s["block_table"][b].long()[t // PAGE], t % PAGE
        for g in range(c["Hkv"]):
            k, v = (s[x][page, g, at].double() if c["layout"] == "head_major" else s[x][page, at, g].double() for x in ("k_cache", "v_cache"))
            step = max(1, int(2e8) // ((P + n) * G))
            for i0 in range(0, n, step):
                i1 = min(n, i0 + step)
                far = (torch.arange(P + i0, P + i1, device="cuda")[:, None] - t[None])
                hide = (far < 0) | (far >= c["window"]) if c["window"] else far < 0
                x = torch.einsum("ihd,td->iht", s["q"][b, i0:i1, g * G:(g + 1) * G].double(), k) / math.sqrt(c["D"])
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                out[b, i0:i1, g * G:(g + 1) * G] = torch.einsum("iht,td->ihd", torch.softmax(x.masked_fill(hide[:, None], -math.inf), -1), v)
    return out


def _exact_rules(s, c):
    out = s["result"].double()
    bits = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint64)
    tokens = None if s["mask"] is None else s["tokens"].cpu().numpy()
    index = None if s["allow"] is None else s["allow_index"].cpu().numpy()
    for b, (_, n) in enumerate(_lengths(c)):
        for i in range(n):
            x = s["logits"][b, i].double()
            if c["counts"]:
                packed = s["counts"][b].long() & 0xFFFFFFFF
                times = (packed % (1 << 31)).double()
                if bits is not None:
                    for j in range(1, n):
                        if int(bits[b, i, j // 64]) >> (j % 64) & 1:
                            times[int(tokens[b, j])] += 1
                r = s["repetition"][b].double()
                seen = (times > 0) | (packed >= 1 << 31)
                x = torch.where(seen, x * torch.where(x > 0, 1 / r, r), x)
                x = x - times * s["frequency"][b].double() - (times > 0) * s["presence"][b].double()
            if c["bias"]:
                x = x + s["bias"].double()
            if index is not None and index[b, i] >= 0:
                words = s["allow"][int(index[b, i])].long() & 0xFFFFFFFF
                flags = torch.stack([(words >> k) & 1 for k in range(32)], 1).flatten()[:c["V"]]
                x = x.masked_fill(flags == 0, -math.inf)
            out[b, i] = x
    return {"target_ids": None, "logits": out}


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "prompt":
        return _exact_prompt(s, c)
    if c["kind"] == "rules" and c["write"]:
        return _exact_rules(s, c)
    return None
