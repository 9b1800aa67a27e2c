"""Keys and values on their way into a paged cache, and attention over a cache held in 4 bits, as cases
whose time can be measured.

Four kinds of work, each through the package's public calls (`own`) or in plain torch operations:

  append      graft_kv_append: queries and keys of new tokens are rotated by their positions, keys and
              values written to their slots of the paged cache (float32 or bfloat16).
  append_mx   graft_kv_append_mx: the same into a cache of 4-bit elements, and graft_kv_gather_mx, which
              reads the rows back as numbers.
  attn_mx     graft_tree_attn_mx: tree-masked attention over such a cache, optionally with capped
              scores and a window of the last positions.
  compact_mx  graft_kv_compact_mx: after acceptance the accepted path's rows move behind the prefix, in
              all layers, and graft_kv_gather_mx, which reads them back.

The 4-bit cache holds e2m1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) in blocks of 32 along the head
dimension with one power of two each, 2^(byte - 127).  The 16 tokens that a page holds of one KV head are
one run of 17 D / 2 bytes.  Keys: 16 D / 2 bytes of elements, token after token, two to a byte, the even one
in the low half; then D / 32 rows of 16 scale bytes, one per token.  Values: the same, with the elements in
the order [token / 4][part 0..15][token % 4][D / 16 elements of the part].
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    app = dict(interleaved=False, ragged=False, layout="head_major")
    att = dict(kind="attn_mx", D=128, ragged=False, cap=0.0, window=0)
    return [
        # One token of a toy model in float32, with the even and odd elements as pairs: launches and latency.
        dict(app, name="append_token_f32", kind="append", dtype="f32", B=1, T=1, Hq=8, Hkv=2, D=64, R=64, P=257, interleaved=True),
        # A ragged batch of two prompts of an 8B-class model into the bfloat16 cache.
        dict(app, name="append_prompt_bf16", kind="append", dtype="bf16", B=2, T=8191, Hq=32, Hkv=8, D=128, R=128, P=0, ragged=True),
        # The trees of a serving batch on one GPU's share of a large model's heads.
        dict(app, name="append_mx_tree", kind="append_mx", dtype="bf16", B=8, T=48, Hq=64, Hkv=4, D=128, R=128, P=4096),
        # Four prompts behind a shared system prompt of odd length.
        dict(app, name="append_mx_prompt", kind="append_mx", dtype="bf16", B=4, T=4097, Hq=32, Hkv=8, D=128, R=128, P=301, ragged=True),
        # One token of a toy model: latency.
        dict(att, name="attn_mx_token_small", B=1, K=1, Hq=8, Hkv=2, D=64, P=255),
        # Plain decoding of a serving batch, one token each over up to 16K: the cache is read once.
        dict(att, name="attn_mx_tokens", B=32, K=1, Hq=32, Hkv=8, P=16384, ragged=True),
        # One chat request on an 8B-class model: a 2K prefix, 40 tree nodes.
        dict(att, name="attn_mx_tree_short", B=1, K=40, Hq=32, Hkv=8, P=2048),
        # One request with a 32K prefix (meeting transcripts, repositories), 40 query and 8 KV heads.
        dict(att, name="attn_mx_tree_long", B=1, K=64, Hq=40, Hkv=8, P=32768),
        # Four requests with 64K prefixes and a 96-node tree: the largest.
        dict(att, name="attn_mx_tree_batch", B=4, K=96, Hq=32, Hkv=8, P=65536),
        # A layer of a model that caps its scores and looks back 4096 positions, ragged batch.
        dict(att, name="attn_mx_capped_window", B=6, K=33, Hq=16, Hkv=8, P=20011, ragged=True, cap=50.0, window=4096),
        # After one request's verification: 32 layers, 4 accepted nodes.
        dict(name="compact_mx_request", kind="compact_mx", B=1, K=40, layers=32, Hkv=8, D=128, P=2048, accept=4, ragged=False),
        # A serving batch of 16, all 94 layers of a large model, up to 9 accepted nodes.
        dict(name="compact_mx_batch", kind="compact_mx", B=16, K=48, layers=94, Hkv=4, D=128, P=4095, accept=9, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append_mx", "attn_mx", "attn_mx", "attn_mx", "compact_mx"])
    D = rng.choice([128, 128, 128, 64])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    Hq = Hkv * rng.randint(1, 16)
    c = dict(kind=kind, B=_log_int(rng, 1, 32), D=D, Hkv=Hkv, ragged=rng.random() < 0.5)
    if kind == "compact_mx":
        accept = rng.randint(0, 16)
        c.update(K=rng.randint(2 * accept + 2, 128), layers=_log_int(rng, 1, 94), P=_log_int(rng, 16, 4096), accept=accept)
        while c["B"] * c["layers"] * Hkv * (c["P"] + c["K"]) * D > 16 * 94 * 4 * 4096 * 128:
            c["B"], c["P"] = max(1, c["B"] // 2), max(16, c["P"] // 2)
        return c
    if kind == "attn_mx":
        c.update(K=rng.choice([1, 1, rng.randint(2, 16), rng.randint(8, 128), rng.randint(8, 128)]), Hq=Hq, P=_log_int(rng, 32, 65536),
                 cap=rng.choice([0.0, 0.0, 30.0]), window=rng.choice([0, 0, _log_int(rng, 16, 8192)]))
        while work(dict(c, window=0))["flops"] > 4.0e11 or c["B"] * Hkv * (c["P"] + c["K"]) * D > 5e8:
            c["B"], c["P"] = max(1, c["B"] // 2), max(32, c["P"] * 2 // 3)
        return c
    c.update(dtype=rng.choice(["bf16", "bf16", "f32"]), T=rng.choice([1, rng.randint(2, 128), _log_int(rng, 64, 8192)]), Hq=Hq,
             R=rng.choice([D, D, D // 2, D // 4]), P=_log_int(rng, 1, 16384), interleaved=rng.random() < 0.4,
             layout=rng.choice(["head_major", "token_major"]))
    while work(c)["bytes"] > 2.8e8:
        c["B"], c["T"] = max(1, c["B"] // 2), max(1, c["T"] * 2 // 3)
    return c


# ---------------------------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------------------------
def _lengths(c):
    """(tokens in front, new tokens or nodes) per sequence; a ragged batch has lengths down to about half."""
    new = c["T"] if "T" in c else c["K"]
    out = []
    for b in range(c["B"]):
        if c["ragged"]:
            out.append((c["P"] - (b * 997) % (c["P"] // 2 + 1), new - (b * 7 + 3) % (new // 2 + 1)))
        else:
            out.append((c["P"], new))
    return out


def _accepted(c):
    return [c["accept"] - (b * 5) % (c["accept"] // 2 + 1) if c["ragged"] else c["accept"] for b in range(c["B"])]


def work(c):
    Hkv, D = c["Hkv"], c["D"]
    row = Hkv * D * 17 / 32                                    # bytes of one token's keys or values in 4 bits
    if c["kind"] == "compact_mx":
        moved = sum(_accepted(c))
        read = moved + c["B"]
        return {"bytes": c["layers"] * (4 * moved * row + 2 * read * row + 4.0 * c["B"] * (c["accept"] + 1) * Hkv * D) + 8.0 * c["B"], "flops": 0.0}
    if c["kind"] == "attn_mx":
        nbytes, flops = 0.0, 0.0
        for P, n in _lengths(c):
            seen = min(P, c["window"]) if c["window"] else P
            nbytes += 2 * (seen + n) * row + (n + c["K"]) * c["Hq"] * D * 2 + 24 * n + 4 * ((seen + n + PAGE - 1) // PAGE)
            flops += 4.0 * n * c["Hq"] * D * (seen + min(n, 8))        # the prefix and about 8 nodes of the own path
        return {"bytes": nbytes, "flops": flops}
    e = 2 if c["dtype"] == "bf16" else 4
    N = sum(n for _, n in _lengths(c))
    nbytes = N * (2 * c["Hq"] * D * e + 2 * Hkv * D * e + 4.0 * c["R"] + 8)
    if c["kind"] == "append":
        return {"bytes": nbytes + N * 2 * Hkv * D * e, "flops": 3.0 * N * c["R"] * (c["Hq"] + Hkv)}
    return {"bytes": nbytes + N * 4 * row + 4.0 * c["B"] * c["T"] * Hkv * D, "flops": 3.0 * N * c["R"] * (c["Hq"] + Hkv)}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _normal(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _trees(rng, c):
    """Parents of random trees, chains of about 8 below the first nodes: ancestor masks [B,K,2] and depths [B,K]."""
    B, K = c["B"], c["T"] if "T" in c else c["K"]
    mask, depth = np.zeros((B, K, 2), np.uint64), np.full((B, K), -1, np.int64)
    for b, (_, n) in enumerate(_lengths(c)):
        for i in range(n):
            up = -1 if i == 0 else i - 1 if rng.random() < 0.5 and depth[b, i - 1] < 12 else int(rng.integers(0, (i + 1) // 2))
            depth[b, i] = 0 if i == 0 else depth[b, up] + 1
            if i:
                mask[b, i] = mask[b, up]
            mask[b, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return mask, depth


def _table(rng, c, tokens):
    """A page table of random pages for `tokens` tokens a sequence, and the number of pages of the cache."""
    pages = (tokens + PAGE - 1) // PAGE
    total = c["B"] * pages + 3
    return _up(rng.permutation(total)[:c["B"] * pages].reshape(c["B"], pages)), total


def _cos_sin(n_pos, R):
    """Cosines, then sines of position * 10000^(-2j/R), [n_pos, R], the angles in 64 bits."""
    if R == 0:
        return torch.zeros((n_pos, 0), device="cuda")
    angle = torch.arange(n_pos, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(c, seed):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    B, Hkv, D, lengths = c["B"], c["Hkv"], c["D"], _lengths(c)
    new = c["T"] if "T" in c else c["K"]
    s = dict(c=c, prefix_len=_up([P for P, _ in lengths]), n_nodes=_up([n for _, n in lengths]))
    s["block_table"], total = _table(rng, c, c["P"] + new)
    block = 17 * D // 2
    s["mx_strides"] = {"page": Hkv * block, "head": block}
    if c["kind"] == "compact_mx":
        # what matters is that the bytes arrive: elements and scales are drawn as such
        L, a = c["layers"], _accepted(c)
        s["layer_stride"] = total * Hkv * block
        for x in ("k_cache", "v_cache"):
            s[x] = torch.randint(0, 256, (L, total, Hkv, block), generator=g, device="cuda", dtype=torch.uint8)
            s[x][..., 8 * D:].bitwise_and_(7).add_(120)
        path = np.full((B, c["accept"] + 1), -1)
        for b in range(B):
            path[b, 0] = 0
            path[b, 1:a[b] + 1] = np.sort(rng.choice(np.arange(a[b] + 1, lengths[b][1] if lengths[b][1] > 2 * a[b] else c["K"]), a[b], replace=False))
        s.update(path=_up(path), accept_len=_up(a), count=_up([x + 1 for x in a]))
        return s
    if c["kind"] == "attn_mx":
        mask, depth = _trees(rng, c)
        s["mask"] = torch.from_numpy(mask.view(np.int64)).cuda()
        s["pos"] = _up(np.where(depth < 0, -1, depth + np.array([P for P, _ in lengths])[:, None]))
        s["q"] = _normal(g, (B, c["K"], c["Hq"], D), torch.bfloat16)
        s["k_cache"] = _pack(_normal(g, (total, Hkv, PAGE, D)), False)
        s["v_cache"] = _pack(_normal(g, (total, Hkv, PAGE, D)), True)
        return s
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    # queries, keys and values as one projection leaves them
    qkv = _normal(g, (B, new, c["Hq"] + 2 * Hkv, D), dtype)
    s["q"], s["k"], s["v"] = qkv[:, :, :c["Hq"]], qkv[:, :, c["Hq"]:c["Hq"] + Hkv], qkv[:, :, c["Hq"] + Hkv:]
    P = np.array([P for P, _ in lengths])[:, None]
    if new <= 128:
        _, depth = _trees(rng, c)
        s["pos"] = _up(np.where(depth < 0, -1, depth + P))
    else:
        s["pos"] = _up(P + np.arange(new)[None])
    s["cos_sin"] = _cos_sin(c["P"] + new, c["R"])
    s["out"] = {"q": torch.zeros((B, new, c["Hq"], D), dtype=dtype, device="cuda"), "status": torch.zeros(B, dtype=torch.int32, device="cuda")}
    if c["kind"] == "append":
        shape = (total, Hkv, PAGE, D) if c["layout"] == "head_major" else (total, PAGE, Hkv, D)
        s["strides"] = ({"page": Hkv * PAGE * D, "token": D, "head": PAGE * D} if c["layout"] == "head_major"
                        else {"page": Hkv * PAGE * D, "token": Hkv * D, "head": D})
        s["k_cache"], s["v_cache"] = torch.zeros(shape, dtype=dtype, device="cuda"), torch.zeros(shape, dtype=dtype, device="cuda")
    else:
        s["k_cache"], s["v_cache"] = (torch.zeros((total, Hkv, block), dtype=torch.uint8, device="cuda") for _ in range(2))
    return s


# ---------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------
def _rotate(x, s):
    """Rows [B,T,H,D] turned by their positions: float32, rounded once."""
    R, c = s["c"]["R"], s["c"]
    if R == 0:
        return x
    row = s["cos_sin"][s["pos"].clamp(min=0).long()]
    cos, sin = row[:, :, None, :R // 2], row[:, :, None, R // 2:]
    f = x.float()
    if c["interleaved"]:
        a, b = f[..., 0:R:2], f[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = f[..., :R // 2], f[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, f[..., R:]], -1)


def _quantise(x):
    """Elements (0..15) and scale bytes of float32 rows [..., D]: blocks of 32, the largest magnitude within (3.5, 7] scales."""
    y = x.unflatten(-1, (-1, 32))
    top = (y.view(torch.int32) & 0x7FFFFFFF).amax(-1)
    byte = (((top + 0x1FFFFF) >> 23) - 2).clamp(2, 252)
    m = y.abs() * ((254 - byte) << 23).view(torch.float32)[..., None]
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)) | (torch.signbit(y).to(torch.uint8) << 3)
    return code.flatten(-2), byte.to(torch.uint8)


def _dequantise(code, byte):
    value = torch.tensor(GRID + tuple(-x for x in GRID), device=code.device)[code.int()]
    return (value.unflatten(-1, (-1, 32)) * (byte.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _pack(x, values):
    """Pages [..., 16, D] of float32 -> their runs of bytes [..., 17 D / 2]."""
    code, byte = _quantise(x)
    if values:
        D = x.shape[-1]
        code = code.unflatten(-1, (16, D // 16)).unflatten(-3, (4, 4)).transpose(-3, -2)
    code = code.flatten(x.dim() - 2)
    return torch.cat([code[..., 0::2] | (code[..., 1::2] << 4), byte.transpose(-1, -2).flatten(-2)], -1)


def _unpack(run, values):
    """Runs of bytes [..., 17 D / 2] -> elements [..., 16, D] and scale bytes [..., 16, D / 32]."""
    D = run.shape[-1] * 2 // 17
    code = torch.stack([run[..., :8 * D] & 15, run[..., :8 * D] >> 4], -1).flatten(-2)
    if values:
        code = code.unflatten(-1, (4, 16, 4, D // 16)).transpose(-3, -2).flatten(-4)
    return code.unflatten(-1, (16, D)), run[..., 8 * D:].unflatten(-1, (-1, 16)).transpose(-1, -2)


def _bytes_of(D, values):
    """Where a token's bytes are in a run: [16, 17 D / 32]."""
    t, i = torch.arange(16, device="cuda")[:, None], torch.arange(D // 2, device="cuda")[None]
    part = D // 32                                             # bytes of one token in one part
    at = ((t // 4 * 16 + i // part) * 4 + t % 4) * part + i % part if values else t * (D // 2) + i
    return torch.cat([at, 8 * D + torch.arange(D // 32, device="cuda")[None] * 16 + t], 1)


def _slots(s, first, count):
    """Page, place in the page, sequence and row of rows first[b] .. first[b] + count[b]."""
    b, i = torch.nonzero(torch.arange(int(count.max()), device="cuda")[None] < count[:, None], as_tuple=True)
    t = first.long()[b] + i
    return s["block_table"].long()[b, t // PAGE], t % PAGE, b, i


def _read(cache, s, first, count, T, values):
    """Rows as numbers, [L,B,T,Hkv,D] in bfloat16; zeros behind a sequence's last."""
    page, at, b, i = _slots(s, first, count)
    c = s["c"]
    where = _bytes_of(c["D"], values)[at]                      # [N, bytes of a row]
    runs = cache if cache.dim() == 4 else cache[None]          # [L, page, head, bytes]
    rows = torch.gather(runs[:, page], -1, where[None, :, None].expand(runs.shape[0], -1, c["Hkv"], -1))
    n = c["D"] // 2
    code = torch.stack([rows[..., :n] & 15, rows[..., :n] >> 4], -1).flatten(-2)
    out = torch.zeros((runs.shape[0], c["B"], T, c["Hkv"], c["D"]), dtype=torch.bfloat16, device="cuda")
    out[:, b, i] = _dequantise(code, rows[..., n:]).bfloat16()
    return out


def _write_mx(cache, s, rows, values):
    """float32 rows [B,T,Hkv,D] to their slots."""
    page, at, b, i = _slots(s, s["prefix_len"], s["n_nodes"])
    code, byte = _quantise(rows[b, i])
    new = torch.cat([code[..., 0::2] | (code[..., 1::2] << 4), byte], -1)
    head = torch.arange(s["c"]["Hkv"], device="cuda")[None, :, None]
    cache[page[:, None, None], head, _bytes_of(s["c"]["D"], values)[at][:, None]] = new


def _plain_append(s):
    c = s["c"]
    q, k = _rotate(s["q"], s), _rotate(s["k"], s)
    page, at, b, i = _slots(s, s["prefix_len"], s["n_nodes"])
    dtype = s["q"].dtype
    rows = torch.zeros_like(s["out"]["q"])
    rows[b, i] = q[b, i].to(dtype)
    if c["kind"] == "append_mx":
        _write_mx(s["k_cache"], s, k.float(), False)
        _write_mx(s["v_cache"], s, s["v"].float(), True)
        return {"q": rows, "k": _read(s["k_cache"], s, s["prefix_len"], s["n_nodes"], c["T"], False),
                "v": _read(s["v_cache"], s, s["prefix_len"], s["n_nodes"], c["T"], True)}
    head = torch.arange(c["Hkv"], device="cuda")[None]
    place = (page[:, None], head, at[:, None]) if c["layout"] == "head_major" else (page[:, None], at[:, None], head)
    s["k_cache"][place] = k[b, i].to(dtype)
    s["v_cache"][place] = s["v"][b, i]
    return {"q": rows, "k": s["k_cache"], "v": s["v_cache"]}


def _seen(s, T):
    """Which tokens 0..T a node sees, [B,K,T]: the prefix, its ancestors and itself, the last `window` positions of them."""
    c = s["c"]
    t, P = torch.arange(T, device="cuda")[None, None], s["prefix_len"].long()[:, None, None]
    j = (t - P).clamp(0, 127)
    word = torch.gather(s["mask"], 2, (j // 64).expand(c["B"], c["K"], -1))
    live = torch.arange(c["K"], device="cuda")[None, :, None] < s["n_nodes"][:, None, None]
    seen = live & ((t < P) | ((t < P + s["n_nodes"][:, None, None]) & ((word >> (j % 64)) & 1).bool()))
    if c["window"]:
        pos = s["pos"].long()
        place = torch.where(t < P, t, torch.gather(pos, 1, j[:, 0].clamp(max=c["K"] - 1))[:, None])
        seen &= pos[:, :, None] - place < c["window"]
    return seen


def _plain_attn(s):
    c = s["c"]
    B, K, Hq, Hkv, D = c["B"], c["K"], c["Hq"], c["Hkv"], c["D"]
    table = s["block_table"].long()
    k, v = (_dequantise(*_unpack(s[x][table], x == "v_cache")).transpose(1, 2).flatten(2, 3) for x in ("k_cache", "v_cache"))   # [B,Hkv,T,D]
    q = s["q"].float().view(B, K, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).flatten(2, 3)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(1 / math.sqrt(D))
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    x = x.view(B, Hkv, K, Hq // Hkv, -1).masked_fill_(~_seen(s, x.shape[-1])[:, None, :, None], -math.inf).flatten(2, 3)
    x = x.sub_(x.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, v) / torch.where(total > 0, total, 1.0)
    return out.view(B, Hkv, K, Hq // Hkv, D).permute(0, 2, 1, 3, 4).flatten(2, 3).bfloat16()


def _plain_compact(s):
    c = s["c"]
    page_to, at_to, b, i = _slots(s, s["prefix_len"] + 1, s["accept_len"])
    t = s["prefix_len"].long()[b] + s["path"].long()[b, i + 1]
    page, at = s["block_table"].long()[b, t // PAGE], t % PAGE
    layer, head = torch.arange(c["layers"], device="cuda")[:, None, None, None], torch.arange(c["Hkv"], device="cuda")[None, None, :, None]
    for x in ("k_cache", "v_cache"):
        where = _bytes_of(c["D"], x == "v_cache")
        at4 = lambda p, a: (layer, p[None, :, None, None], head, where[a][None, :, None])       # noqa: E731
        s[x][at4(page_to, at_to)] = s[x][at4(page, at)]
    T = c["accept"] + 1
    return {"new_prefix_len": s["prefix_len"] + s["accept_len"] + 1, "k": _read(s["k_cache"], s, s["prefix_len"], s["count"], T, False),
            "v": _read(s["v_cache"], s, s["prefix_len"], s["count"], T, True)}


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(s):
    c = s["c"]
    if not own:
        return {"append": _plain_append, "append_mx": _plain_append, "attn_mx": _plain_attn, "compact_mx": _plain_compact}[c["kind"]](s)
    import paper_2605_20104_amd as graft
    place = (s["block_table"], s["prefix_len"])
    if c["kind"] == "append":
        out = graft.graft_kv_append(s["q"], s["k"], s["v"], s["cos_sin"], s["pos"], s["k_cache"], s["v_cache"], s["strides"], *place,
                                    s["n_nodes"], interleaved=c["interleaved"], out=s["out"])
        return {"q": out["q"], "k": s["k_cache"], "v": s["v_cache"]}
    caches = (s["k_cache"], s["v_cache"])
    if c["kind"] == "append_mx":
        out = graft.graft_kv_append_mx(s["q"], s["k"], s["v"], s["cos_sin"], s["pos"], *caches, s["mx_strides"], *place, s["n_nodes"],
                                       interleaved=c["interleaved"], out=s["out"])
        back = graft.graft_kv_gather_mx(*caches, 0, 1, s["mx_strides"], *place, s["n_nodes"], c["T"], c["Hkv"], c["D"])
        return {"q": out["q"], "k": back["k"], "v": back["v"]}
    if c["kind"] == "attn_mx":
        return graft.graft_tree_attn_mx(s["q"], *caches, s["mx_strides"], *place, s["n_nodes"], s["mask"], c["Hkv"], 1 / math.sqrt(c["D"]),
                                        softcap=c["cap"], window=c["window"], pos=s["pos"])
    out = graft.graft_kv_compact_mx(*caches, s["layer_stride"], c["layers"], s["mx_strides"], *place, s["path"], s["accept_len"], c["K"],
                                    c["Hkv"], c["D"])
    back = graft.graft_kv_gather_mx(*caches, s["layer_stride"], c["layers"], s["mx_strides"], *place, s["count"], c["accept"] + 1, c["Hkv"],
                                    c["D"])
    return {"new_prefix_len": out["new_prefix_len"], "k": back["k"], "v": back["v"]}


# ---------------------------------------------------------------------------------------------
# from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_turn(x, table, pos, R, interleaved):
    """One row's elements as complex numbers times e^(i angle)."""
    x = x.double()
    out = x.clone()
    if R:
        turn = torch.complex(table[pos, :R // 2].double(), table[pos, R // 2:].double())[:, None]
        lo, hi = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
        z = torch.complex(x[..., lo].contiguous(), x[..., hi].contiguous()) * turn
        out[..., lo], out[..., hi] = z.real, z.imag
    return out


def _exact_mx(x):
    """The numbers that the 4-bit elements of double rows stand for."""
    y = x.unflatten(-1, (-1, 32))
    mant, exp = torch.frexp(y.abs().amax(-1, keepdim=True))    # the largest is mant 2^exp, mant within [0.5, 1)
    exp = torch.where(mant * 8 > 7, exp - 2, exp - 3).clamp(-125, 125)
    exp = torch.where(mant == 0, torch.full_like(exp, -125), exp)
    m = torch.ldexp(y.abs(), -exp).clamp(max=6.0)
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    near = torch.round(m / step) * step                        # ties to even, as the elements' last bits are
    return (torch.ldexp(near, exp) * torch.sign(y)).flatten(-2)


def _exact_numbers(run, values):
    """Runs [N, 17 D / 2] of bytes -> [N, 16, D] in double, element by element of the format."""
    D = run.shape[-1] * 2 // 17
    t, d = torch.arange(16, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    part = D // 16
    number = ((t // 4 * 16 + d // part) * 4 + t % 4) * part + d % part if values else t * D + d
    four = (run[:, number // 2].int() >> (number % 2 * 4)) & 15
    e, m = (four >> 1) & 3, four & 1
    size = torch.where(e == 0, m * 0.5, (1 + m * 0.5) * torch.exp2(e.double() - 1))
    return torch.where(four >= 8, -size, size).double() * torch.exp2(run[:, 8 * D + d // 32 * 16 + t].double() - 127)


def exact(c, seed):
    s = prepare(c, seed)
    lengths, B, Hkv, D = _lengths(c), c["B"], c["Hkv"], c["D"]
    table = s["block_table"].cpu().numpy()
    if c["kind"] == "attn_mx":
        K, G = c["K"], c["Hq"] // Hkv
        out = torch.zeros((B, K, c["Hq"], D), dtype=torch.float64, device="cuda")
        bits = s["mask"].cpu().numpy().view(np.uint64)
        for b, (P, n) in enumerate(lengths):
            used = torch.from_numpy(table[b, :(P + n + 15) // 16].astype(np.int64)).cuda()
            pos = s["pos"][b].long()
            see = np.array([[bool(int(bits[b, i, j // 64]) >> (j % 64) & 1) for j in range(n)] for i in range(n)])
            see = torch.cat([torch.ones((n, P), dtype=torch.bool, device="cuda"), torch.from_numpy(see).cuda()], 1)
            if c["window"]:
                place = torch.cat([torch.arange(P, device="cuda"), pos[:n]])
                see &= pos[:n, None] - place[None] < c["window"]
            for g in range(Hkv):
                k, v = (_exact_numbers(s[x][used, g], x == "v_cache").flatten(0, 1)[:P + n] for x in ("k_cache", "v_cache"))
                x = s["q"][b, :n, g * G:(g + 1) * G].double().flatten(0, 1) @ k.T / math.sqrt(D)
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                x = x.view(n, G, -1).masked_fill(~see[:, None], -math.inf)
                out[b, :n, g * G:(g + 1) * G] = (torch.softmax(x, -1).flatten(0, 1) @ v).view(n, G, D)
        return out
    if c["kind"] == "compact_mx":
        T, a = c["accept"] + 1, _accepted(c)
        out = {x: torch.zeros((c["layers"], B, T, Hkv, D), dtype=torch.float64, device="cuda") for x in "kv"}
        path = s["path"].cpu().numpy()
        for b, (P, _) in enumerate(lengths):
            for i in range(a[b] + 1):
                t = P + int(path[b, i])
                for x in "kv":
                    out[x][:, b, i] = _exact_numbers(s[x + "_cache"][:, table[b, t // 16]].flatten(0, 1), x == "v")[:, t % 16].reshape(-1, Hkv, D)
        return {"new_prefix_len": None, "k": out["k"], "v": out["v"]}
    pos = s["pos"].long().clamp(min=0)
    q = torch.zeros((B, c["T"], c["Hq"], D), dtype=torch.float64, device="cuda")
    mx = c["kind"] == "append_mx"
    k, v = (torch.zeros((B, c["T"], Hkv, D), dtype=torch.float64, device="cuda") if mx else s[x].double() for x in ("k_cache", "v_cache"))
    for b, (P, n) in enumerate(lengths):
        q[b, :n] = _exact_turn(s["q"][b, :n], s["cos_sin"], pos[b, :n], c["R"], c["interleaved"])
        new_k, new_v = _exact_turn(s["k"][b, :n], s["cos_sin"], pos[b, :n], c["R"], c["interleaved"]), s["v"][b, :n].double()
        if mx:
            k[b, :n], v[b, :n] = _exact_mx(new_k), _exact_mx(new_v)
            continue
        t = torch.arange(P, P + n, device="cuda")
        page, at = s["block_table"][b].long()[t // 16], t % 16
        for cache, new in ((k, new_k), (v, new_v)):
            pages = cache if c["layout"] == "head_major" else cache.transpose(1, 2)            # [page, head, place, D]
            pages[page, :, at] = new
    return {"q": q, "k": k, "v": v}
