"""How the library cuts the tokens of a norm, rotation or append into launches and blocks, as it works it out on the host."""
import ctypes as C

import pytest

WAVES, BLOCK = 4, 256


class Cut(C.Structure):                            # lazyev::RopeCut (kernels.h)
    _fields_ = [("tokens", C.c_int32), ("shares", C.c_int32), ("past", C.c_int32), ("launch", C.c_int64)]


def _cut(b, tokens, heads, elem, d):
    fn = getattr(b.lib, "_ZN6lazyev8rope_cutExiii")   # lazyev::rope_cut (kernels.h)
    fn.restype, fn.argtypes = Cut, [C.c_longlong, C.c_int, C.c_int, C.c_int]
    return fn(tokens, heads, elem, d)


TYPES = [(2, 128), (2, 64), (4, 128), (4, 64)]
TOKENS = sorted({max(1, (1 << n) + o) for n in range(31) for o in (-1, 0, 1) if (1 << n) + o <= 1 << 30} | {1535, 1536, 2250})
HEADS = [1, 2, 3, 4, 7, 8, 15, 16, 17, 31, 32, 48, 96, 97, 384, 4000, 65535]


@pytest.mark.parametrize("elem,d", TYPES)
def test_launches_within_the_grid(lazyev_lib, elem, d):
    """No launch has 2^32 threads or more in a row of blocks, or more than 65535 shares, up to 2^30 tokens; the launches begin at whole blocks and every
    head of a token has a lane's turn."""
    rows = 64 // (d * elem // 16)
    for heads in HEADS:
        for tokens in TOKENS:
            c = _cut(lazyev_lib, tokens, heads, elem, d)
            assert c.tokens in (1, 4, WAVES * rows) and 1 <= c.shares <= 65535
            assert c.shares == 1 or (c.tokens == 1 and (c.shares - 1) * rows * WAVES < heads)
            assert c.launch > 0 and c.launch % c.tokens == 0
            blocks = -(-min(tokens, c.launch) // c.tokens)
            assert blocks * BLOCK < 1 << 32, (heads, tokens)
            assert -(-tokens // c.launch) * c.launch <= (1 << 30) + c.launch     # (token numbers stay in 32 bits)


@pytest.mark.parametrize("elem,d", TYPES)
def test_results_past_the_caches(lazyev_lib, elem, d):
    """All but those of one token a block that an XCD's L2 (4 MB) holds."""
    for heads in HEADS:
        for tokens in TOKENS:
            c = _cut(lazyev_lib, tokens, heads, elem, d)
            assert c.past == (c.tokens > 1 or tokens * heads * d * elem >= 4 << 20), (heads, tokens)
