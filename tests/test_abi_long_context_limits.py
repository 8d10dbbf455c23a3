"""What the attention over a cache in 4 bits accepts: what the window call accepts, whatever
bound of the lengths is given (CPU only; host-side checks)."""
import random

import pytest

from tests.test_abi_cache import lib  # noqa: F401  (lib is a fixture)
from tests.test_abi_long_context import kv4, window


@pytest.mark.parametrize("hint", [0, 1000, 20000, 0x7FFFFFFF])
@pytest.mark.parametrize("window_,sinks", [(0, 0), (100, 4)])
def test_the_bound_of_the_lengths_decides_no_refusal(lib, hint, window_, sinks):  # noqa: F811
    shape = dict(B=64, N=40, Hq=32, Hkv=8, P=256, max_pages=200000, window=window_, sinks=sinks, max_kv_len=hint)
    assert window(lib, **shape) == -6 and kv4(lib, **shape) == -6


def test_the_limits_are_the_window_calls(lib):  # noqa: F811
    rng = random.Random(3)
    seen = {-2: 0, -6: 0}
    for _ in range(4000):
        G = rng.choice([1, 1, 2, 4, 7, 8, 16, 64])
        Hkv = rng.choice([1, 2, 8, 24, 32, 64])
        N = min(rng.choice([1, 3, 12, 16, 17, 32, 33, 40, 64, 100, 160, 256]), 2048 // G)
        P = 1 << rng.randrange(9)
        shape = dict(B=rng.choice([1, 7, 64, 256, 1024]), N=N, Hq=G * Hkv, Hkv=Hkv, D=rng.choice([64, 128]), P=P,
                     max_pages=int(2 ** rng.uniform(20, 31)) // P, window=rng.choice([0, 0, 100, 9000]),
                     max_kv_len=rng.choice([0, 700, 3000, 60000, 0x7FFFFFFF]))
        code = window(lib, **shape)
        assert kv4(lib, **shape) == code, shape
        seen[code] += 1
    assert min(seen.values()) > 500, seen
    # where the tiles of one row block just fit
    for N, G in ((4, 4), (8, 4), (16, 4), (24, 4), (40, 4), (64, 4)):
        for more in range(-12, 13):
            shape = dict(B=512, N=N, Hq=G, Hkv=1, P=64, max_pages=(1 << 21) + more)
            assert kv4(lib, **shape) == window(lib, **shape), shape
