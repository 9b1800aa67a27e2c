"""graft_prompt_attn with values next to the largest that its contract allows, 2^96, all of one sign, and scores that rise by less than what
makes a tile be done again: sums hold probabilities of up to 2^22 (in bf16, of the tokens between two looks at a row's reference)."""
import math

import pytest
import torch

from prompt_util import call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,P", [(1, 900), (20, 900), (300, 700), (300, 3000)])
@pytest.mark.parametrize("rise", [6, 12, 20, 22])
@pytest.mark.parametrize("window,cap", [(0, 0.0), (400, 0.0), (0, 900.0)])
def test_values_next_to_the_limit(dtype, D, T, P, rise, window, cap):
    c = make(rise, dtype, 1, T, 4, 2, D, P)
    n = P + T
    # in log2 units: `rise` more in the second 32 tokens of every 64 than in front, two more from one 64 to the next, up to 600 and down again
    t = torch.arange(n, dtype=torch.float64)
    height = ((t // 64) * (rise + 2) % 600 + (t // 32) % 2 * rise) * math.log(2.0)
    c["q"][..., 0] = 1.0
    keys = c["k"].float() * 0.1
    for s in range(c["pages"]):
        for o in range(16):
            if 16 * s + o < n:
                keys[c["table"][0, s], :, o, 0] = float(height[16 * s + o]) / c["scale"]
    c["k"] = keys.to(c["k"].dtype)
    c["v"] = ((0.5 + torch.rand(c["v"].shape, generator=torch.Generator().manual_seed(rise)) / 2) * 2.0 ** 96).to(c["v"].dtype)
    got = call(c, window, cap)
    assert bool(torch.isfinite(got[:, :T]).all())
    check(c, got, window, cap)
