"""CPU: new tables and lengths of a fork that lie in anything that the fork reads, or in each other, are refused."""
import ctypes
import itertools

import pytest

from test_pages_host import G  # noqa: F401  (a fixture)

N, S, M, NB = 2, 3, 4, 10
SIZES = {"out": N * M, "lens_out": N, "tables": S * M, "lens": S, "refs": NB, "parents": N}


@pytest.mark.parametrize("a,b", [p for p in itertools.permutations(SIZES, 2) if p[0] in ("out", "lens_out")])
def test_overlaps(G, a, b):  # noqa: F811
    """`a` ends with, or begins in, `b`'s last or first number; all others far apart.  (Never dereferenced: each call is refused.)"""
    f = G.load_library().optgqa_fork_sequences
    for at in ((1 << 40) + 4 * (SIZES[b] - 1), (1 << 40) - 4 * (SIZES[a] - 1)):
        places = {name: (1 << 20) * (i + 1) for i, name in enumerate(SIZES)}
        places.update({a: at, b: 1 << 40})
        assert f(*(ctypes.c_void_p(places[name]) for name in SIZES), N, S, M, NB, 16, None) == -2
