"""graft_prompt_attn over sequences long enough that the kernels read page numbers again and again inside one split (64 stages of 64 tokens in
the tiles of 256 rows, 32 steps of 128 in those of 32 and 64): every row looks for a page of its own, so a wrong page is a wrong result.
Queries carry a page's code, which all of its keys have: the page's 16 tokens have nearly all of the row's weight."""
import math

import pytest
import torch

import paper_2605_20104_amd as graft

pytestmark = pytest.mark.gpu


# (B, T, Hq, Hkv, P): rows of a KV head T Hq / Hkv = 16, 48, 900 and 1024; heads enough that the keys are not split
@pytest.mark.parametrize("B,T,Hq,Hkv,P", [(1, 1, 4096, 256, 17001), (1, 12, 1024, 256, 17001), (1, 300, 384, 128, 9001), (1, 256, 512, 128, 13333)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 60.0])
def test_every_page_of_long_sequences(B, T, Hq, Hkv, P, D, cap):
    G, n_tok, scale = Hq // Hkv, P + T, 1 / math.sqrt(D)
    pages = -(-n_tok // 16)
    assert graft.graft_prompt_attn_workspace_bytes(B, T, Hq, Hkv, D, pages, 0, graft.GRAFT_BF16) == 0
    g = torch.Generator(device="cuda").manual_seed(D + T)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")                                  # noqa: E731
    total = B * pages + 3
    table = torch.randperm(total, generator=g, device="cuda")[:B * pages].view(B, pages)
    code = randn(pages, D).sign()
    k, v = torch.empty((total, Hkv, 16, D), dtype=torch.bfloat16, device="cuda"), torch.empty((total, Hkv, 16, D), dtype=torch.bfloat16, device="cuda")
    for b in range(B):
        k[table[b]] = (code[:, None, None] + 0.1 * randn(pages, Hkv, 16, D)).to(torch.bfloat16)
        v[table[b]] = (randn(pages, Hkv, 1, D) + 0.1 * randn(pages, Hkv, 16, D)).to(torch.bfloat16)
    whole = P // 16                                            # pages that every row sees whole: all of them are looked for
    target = ((torch.arange(B * Hkv, device="cuda")[:, None] * 16 + torch.arange(T * G, device="cuda")[None]) * (1 if T == 1 else 11) % whole).view(B, Hkv, T, G)
    assert len(target.unique()) == whole
    q = (30 / math.sqrt(D) * code[target].permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)).to(torch.bfloat16)       # its scores: about 30, the others' about 4 by 0
    i32 = lambda x: torch.full((B,), x, dtype=torch.int32, device="cuda")                                   # noqa: E731
    got = graft.graft_prompt_attn(q, k, v, {"page": Hkv * 16 * D, "token": D, "head": 16 * D}, table.int().contiguous(), i32(P), i32(T), Hkv, scale, softcap=cap)
    far = P + torch.arange(T, device="cuda")[:, None] - torch.arange(n_tok, device="cuda")[None]
    for b in range(B):
        for h in range(Hkv):
            kk, vv = (x[table[b], h].reshape(-1, D)[:n_tok].double() for x in (k, v))
            qq = q[b, :, h * G:(h + 1) * G].double().reshape(T * G, D)
            x = torch.mm(qq, kk.t().contiguous()) * scale
            products = torch.mm(qq.abs(), kk.abs().t().contiguous()).amax(-1, keepdim=True) * scale
            y = cap * torch.tanh(x / cap) if cap else x
            p = torch.softmax(y.masked_fill((far < 0).repeat_interleave(G, 0), -math.inf), -1)
            want, size = torch.mm(p, vv), torch.mm(p, vv.abs())
            # (as for shorter ones: a score's D products and 3 roundings more, its exponential, two sums, probabilities and result in bf16)
            bound = (2.0 ** -8 + 2 * (products * (D + 8) * 2.0 ** -24 + 2.0 ** -20 * cap) + (n_tok + 16) * 2.0 ** -23) * size + 2.0 ** -8 * want.abs()
            off = (got[b, :, h * G:(h + 1) * G].double().reshape(T * G, D) - want).abs()
            assert bool((off <= bound).all()), (b, h, float((off - bound).max()))
            # a row that found another page would be off by far more than the bound
            page = target[b, h].reshape(-1)
            other = (page + 1) % whole
            mean = vv[:whole * 16].view(whole, 16, D).mean(1)
            assert bool(((mean[page] - mean[other]).abs().amax(-1) > 10 * bound.amax(-1)).all())
