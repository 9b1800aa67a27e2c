"""Cases of graft_prompt_attn and the same attention in 64 bits, with the bound that its arithmetic gives each element."""
import math

import numpy as np
import torch

import paper_2605_20104_amd as graft


def make(seed, dtype="bf16", B=1, T=1, Hq=4, Hkv=2, D=64, P=0, n=None, layout="head", size=1.0, extra_pages=0):
    """Queries, caches and tables; prefix lengths `P` and lengths `n` per sequence, or one for all."""
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    tt = torch.float32 if dtype == "f32" else torch.bfloat16
    P = np.broadcast_to(np.asarray(P, np.int32), (B,)).copy()
    n = np.broadcast_to(np.asarray(T if n is None else n, np.int32), (B,)).copy()
    pages = max(1, -(-int((P.astype(np.int64) + n).max()) // 16)) + extra_pages
    total = B * pages + 3
    shape, strides = {
        "head": ((total, Hkv, 16, D), {"page": Hkv * 16 * D, "token": D, "head": 16 * D}),
        "token": ((total, 16, Hkv, D), {"page": Hkv * 16 * D, "token": Hkv * D, "head": D}),
        "gap": ((total, Hkv, 16, D + 24), {"page": Hkv * 16 * (D + 24), "token": D + 24, "head": 16 * (D + 24)}),
    }[layout]
    table = rng.permutation(total)[:B * pages].reshape(B, pages).astype(np.int32)
    k, v = (torch.randn(shape, generator=g).to(tt) for _ in range(2))
    return dict(dtype=dtype, B=B, T=T, Hq=Hq, Hkv=Hkv, D=D, P=P, n=n, layout=layout, strides=strides, pages=pages,
                q=(torch.randn((B, T, Hq, D), generator=g) * size).to(tt), k=k, v=v, table=torch.from_numpy(table), scale=1 / math.sqrt(D))


def rows(c, which, b):
    """Keys or values of sequence b's logical tokens, [tokens, Hkv, D]."""
    x = c[which][c["table"][b].long()]
    x = x if c["layout"] == "token" else x.transpose(1, 2)
    return x.flatten(0, 1)[..., :c["D"]]


def call(c, window=0, softcap=0.0, stream=None, **kw):
    up = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()                                            # noqa: E731
    return graft.graft_prompt_attn(c["q"].cuda(), c["k"].cuda(), c["v"].cuda(), c["strides"], c["table"].cuda(), up(c["P"]), up(c["n"]), c["Hkv"],
                                   c["scale"], softcap=softcap, window=window, stream=stream, **kw)


def exact(c, window=0, softcap=0.0):
    """The result in 64 bits, and what it may be off by (elementwise)."""
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64)
    size = torch.zeros_like(out)                               # sum of p |v|
    worst = torch.zeros((B, T, Hq, 1), dtype=torch.float64)    # relative error of a probability
    half = 2.0 ** -24 if c["dtype"] == "f32" else 2.0 ** -8
    for b in range(B):
        P, n = int(c["P"][b]), int(c["n"][b])
        if n == 0:
            continue
        k, v = rows(c, "k", b)[:P + n].double(), rows(c, "v", b)[:P + n].double()
        far = P + torch.arange(n)[:, None] - torch.arange(P + n)[None]
        seen = (far >= 0) & ((far < window) if window else True)
        for h in range(Hq):
            g = h // (Hq // Hkv)
            q = c["q"][b, :n, h].double()
            x = q @ k[:, g].T * c["scale"]
            x_abs = q.abs() @ k[:, g].abs().T * abs(c["scale"])
            y = softcap * torch.tanh(x / softcap) if softcap else x
            p = torch.softmax(y.masked_fill(~seen, -math.inf), -1)
            out[b, :n, h], size[b, :n, h] = p @ v[:, g], p @ v[:, g].abs()
            # a score: D products summed in fp32, scaled (3 roundings more); its exponential and the two sums; a cap by its own bound
            score = (x_abs * (D + 8) * 2.0 ** -24).masked_fill(~seen, 0).amax(-1, keepdim=True) + (2.0 ** -20 * softcap)
            worst[b, :n, h] = 2 * score + (P + n + 16) * 2.0 ** -23
    probability = 0.0 if c["dtype"] == "f32" else half
    return out, (probability + worst) * size + half * out.abs() + 1e-30


def check(c, got, window=0, softcap=0.0):
    want, bound = exact(c, window, softcap)
    got = got.double().cpu()
    for b in range(c["B"]):
        assert bool((got[b, int(c["n"][b]):] == 0).all()), "rows of padding tokens are zeros"
    off = (got - want).abs()
    assert bool((off <= bound).all()), "off by %.3g where %.3g is allowed" % (float((off - bound).max() + 0), float(bound.flatten()[int((off - bound).argmax())]))
