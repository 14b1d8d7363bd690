"""The division of an entry's number by the page size as the kernels do it, through the code that they share with the host."""
import ctypes as C
import random

import pytest

LAST = (1 << 31) - 1


@pytest.mark.parametrize("seed", range(4))
def test_every_size_next_to_multiples(lazyev_lib, seed):
    fn = getattr(lazyev_lib.lib, "_ZN6lazyev13page_of_entryEii")   # lazyev::page_of_entry (kernels.h)
    fn.restype, fn.argtypes = C.c_int, [C.c_int, C.c_int]
    rng = random.Random(seed)
    sizes = [1, 2, 3, 5, 7, 16, 17, 24, 100, 127, 128, 129, 1000, 4097, (1 << 20) - 1, 1 << 20, 699051]
    sizes += [max(1, min(1 << 20, int(2 ** rng.uniform(0, 20)))) for _ in range(300)]
    for size in sizes:
        multiples = {0, 1, 2, LAST // size, (1 << 30) // size} | {rng.randrange(LAST // size + 1) for _ in range(20)}
        for m in multiples:
            for entry in (m * size - 1, m * size, m * size + 1, m * size + size - 1):
                if 0 <= entry <= LAST:
                    assert fn(size, entry) == entry // size, (size, entry)
