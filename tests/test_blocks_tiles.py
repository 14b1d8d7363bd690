"""Which calls of attention over chosen blocks join the lists of several tokens, by the workspace that they ask for: nothing is launched here."""
import pytest

from test_pages_refusals import _pages


# 32 tokens of groups of 4 heads fill a tile (16 of fp32 rows of 128), 9 KV heads make more units than every token on its own is for
@pytest.mark.parametrize("dtype,d,tokens", [("bf16", 128, 32), ("bf16", 64, 32), ("fp32", 64, 32), ("fp32", 128, 16)])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_joined_lists_stay_in_the_range_of_32_bits(lazyev_lib, dtype, d, tokens, block):
    b = lazyev_lib
    p = _pages(b, dtype=b.DTYPE_FP32 if dtype == "fp32" else b.DTYPE_BF16, head_dim=d, n_kv_heads=9)
    heads, n = 9, 32

    def size(chosen):
        return b.lib.lazyev_blocks_attend_workspace(p, 128, block, chosen, n, 4 * heads)
    # of all numbers that a tile's tokens may list, each a pair of 8 bytes, 2^30 entries at most
    most = (1 << 30) // block // tokens
    assert size(most) >= heads * n * most * 8
    # beyond, every token is on its own: no pairs (parts of fewer bytes than there would be of them)
    for chosen in (most + 1, 2 * most, 4 * most + 1, (1 << 30) // block):
        assert size(chosen) < 1 << 30 and size(chosen) < heads * n * chosen * 8, chosen
