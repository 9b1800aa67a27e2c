"""The workspace of graft_prompt_attn stays within 256 MiB (no GPU), whatever the sizes and however wide the table."""
import itertools

import pytest

import paper_2605_20104_amd as graft

MOST = 256 << 20


@pytest.mark.parametrize("dtype", [graft.GRAFT_BF16, graft.GRAFT_F32])
@pytest.mark.parametrize("D", [64, 128])
def test_workspace_is_bounded(dtype, D):
    split = 0
    for B, T, (Hq, Hkv), pages in itertools.product((1, 2, 4, 33), (1, 5, 40, 300, 1100, 2200, 4500, 9000, 100000, 1 << 20, 1 << 22), ((1, 1), (16, 1), (32, 8), (64, 8), (128, 8)),
                                                    (1, 300, 2311, 8192, 65536, 262144)):
        n = graft.graft_prompt_attn_workspace_bytes(B, T, Hq, Hkv, D, pages, 0, dtype)
        assert n <= MOST, (B, T, Hq, Hkv, pages, n)
        assert n == 0 or n >= 2 * B * T * Hq * (D + 2) * 4
        split += n > 0
    assert split > 300                                     # (splits there are)


# What was split before within the bound still is: single tokens, short pieces, pieces behind long prefixes.
@pytest.mark.parametrize("B,T,Hq,Hkv,pages,splits", [(1, 1024, 40, 8, 2112, 3), (1, 1100, 32, 8, 8192, 7), (1, 512, 32, 8, 8192, 4)])
def test_splits_within_the_bound(B, T, Hq, Hkv, pages, splits):
    assert graft.graft_prompt_attn_workspace_bytes(B, T, Hq, Hkv, 128, pages, 0, graft.GRAFT_BF16) == splits * B * T * Hq * 130 * 4
