"""The set of caches that the page calls work on: what is in it stays what it was made of."""
import numpy as np
import pytest

from test_gpu_pages import G, bits_of, caches, dev  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_a_set_does_not_grow_behind_its_addresses(G, monkeypatch):  # noqa: F811
    """Tensors that come to the list it was made of, or to its own, are not counted: their addresses are not on the GPU."""
    import torch
    given = [torch.zeros(6, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
    s = G.CacheSet(given)
    given.append(given[0])
    try:
        s.caches.append(given[0])
    except AttributeError:
        pass
    counts = []

    class Recorder:
        def __getattr__(self, name):
            return lambda *args: counts.append((name, args[1])) or 0

    pair, one = dev([[0, 1]]), dev([1])
    with monkeypatch.context() as m:
        m.setattr(G, "load_library", Recorder)
        G.copy_blocks(s, pair, one)
        G.keep_tokens(s, pair, one, pair, one)
    assert counts == [("optgqa_copy_blocks", 2), ("optgqa_keep_tokens", 2)] and len(s.pointers) == 2
