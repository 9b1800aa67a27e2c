"""graft_prompt_attn and keys that are no numbers where a row sees them, and workspaces given and not."""
import math

import pytest
import torch

import paper_2605_20104_amd as graft
from prompt_util import call, make, rows
from test_gpu_prompt_ways import SHAPES, _args

pytestmark = pytest.mark.gpu


def by_definition(c, window, cap):
    """The rows in 64 bits, NaN where a seen score is NaN or the largest is infinite, zeros where all of them are -infinity; what they may be
    off by; how many rows there are of each kind (some weight, no number, none)."""
    T, Hq, Hkv, D, P = c["T"], c["Hq"], c["Hkv"], c["D"], int(c["P"][0])
    out, bound, kinds = torch.zeros((T, Hq, D), dtype=torch.float64), torch.zeros((T, Hq, D), dtype=torch.float64), [0, 0, 0]
    k, v = rows(c, "k", 0)[:P + T].double(), rows(c, "v", 0)[:P + T].double()
    far = P + torch.arange(T)[:, None] - torch.arange(P + T)[None]
    seen = (far >= 0) & ((far < window) if window else True)
    half = 0.0 if c["dtype"] == "f32" else 2.0 ** -8       # of a probability
    for h in range(Hq):
        g = h // (Hq // Hkv)
        q = c["q"][0, :, h].double()
        x = q @ k[:, g].T * c["scale"]
        y = cap * torch.tanh(x / cap) if cap else x
        y = y.masked_fill(~seen, -math.inf)
        bad, none = (torch.isnan(y) | (y == math.inf)).any(-1), (y == -math.inf).all(-1)
        p = torch.softmax(torch.where((bad | none)[:, None], 0.0, y), -1)
        size = p @ v[:, g].abs()
        products = (q.abs() @ k[:, g].abs().T * abs(c["scale"])).masked_fill(~seen | ~torch.isfinite(x), 0).amax(-1, keepdim=True)
        score = products * (D + 8) * 2.0 ** -24 + 2.0 ** -20 * cap
        o = p @ v[:, g]
        bound[:, h] = (half + 2 * score + (P + T + 16) * 2.0 ** -23) * size + (2.0 ** -24 if c["dtype"] == "f32" else 2.0 ** -8) * o.abs() + 1e-30
        o[none] = 0.0
        o[bad] = math.nan
        out[:, h] = o
        for i, rows_of in enumerate((~bad & ~none, bad, none & ~bad)):
            kinds[i] += int(rows_of.sum())
    return out, bound, kinds


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P,T,window,cap", [(0, 1, 0, 0.0), (0, 3, 0, 0.0), (150, 3, 40, 0.0), (150, 9, 0, 0.0), (3000, 1, 0, 0.0), (3000, 12, 0, 0.0), (0, 300, 0, 0.0),
                                            (700, 300, 0, 0.0), (700, 300, 120, 0.0), (700, 40, 0, 20.0), (700, 300, 0, 20.0), (2000, 1, 64, 20.0)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_seen_keys(dtype, D, P, T, window, cap, bad):
    """Some keys of one element that is no number: by the query's sign their scores are infinite or -infinite."""
    c = make(21, dtype, 1, T, 6, 2, D, P)
    n = P + T
    for t in sorted({0, P // 2, n // 2, max(0, n - 30), n - 1}):
        c["k"][c["table"][0, t // 16], 1, t % 16, 5] = bad
    got = call(c, window, cap)[0].double().cpu()
    want, bound, kinds = by_definition(c, window, cap)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    off = (got - want).abs()
    assert bool((torch.isnan(want) | (off <= bound)).all()), float((off - bound)[~torch.isnan(want)].max())
    assert kinds[0] > 0 and (bad != bad or cap or n == 1 or kinds[1] > 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,T", [(0, 1), (100, 1), (3000, 2), (100, 20), (100, 300)])
def test_nothing_but_keys_without_weight(dtype, P, T):
    """Every score of KV head 1 is -infinity: zeros, and its values do not matter."""
    c = make(22, dtype, 1, T, 6, 2, 128, P)
    clean = call(c).cpu()
    c["q"][:, :, 3:, 5] = c["q"][:, :, 3:, 5].abs() + 0.1
    c["k"][:, 1, :, 5] = float("-inf")
    got = call(c).cpu()
    assert bool((got[:, :, 3:] == 0).all()) and torch.equal(got[:, :, :3], clean[:, :, :3])


@pytest.mark.parametrize("shape", SHAPES + [("bf16", 1, 1, 8, 2, 64, 3), ("f32", 1, 1, 8, 2, 64, 3), ("bf16", 1, 300, 8, 2, 128, 0)])
def test_workspaces(shape):
    """Too small a workspace is refused where there is one, and nobody asks for one where there is none."""
    a = _args(make(9, *shape))
    dtype = graft.GRAFT_F32 if shape[0] == "f32" else graft.GRAFT_BF16
    B, T, Hq, D = a["q"].shape
    n = graft.graft_prompt_attn_workspace_bytes(B, T, Hq, a["Hkv"], D, a["block_table"].shape[1], 0, dtype)
    want = graft.graft_prompt_attn(**a)
    ws = torch.full((max(n, 64),), 255, dtype=torch.uint8, device="cuda")         # (what is in it does not matter)
    assert torch.equal(graft.graft_prompt_attn(**a, workspace=ws[:n]), want)
    if n > 0:
        with pytest.raises(graft.GraftError) as e:
            graft.graft_prompt_attn(**a, workspace=ws[:n - 16])
        assert e.value.code == graft.GRAFT_ERR_WORKSPACE
    else:
        assert torch.equal(graft.graft_prompt_attn(**a, workspace=ws[:0]), want)
