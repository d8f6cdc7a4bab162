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


@pytest.mark.parametrize("dtype", ["float16", "uint8"])
def test_a_cache_that_layers_share_is_worked_on_once(G, dtype):  # noqa: F811
    """A cache given three times: kept rows move one place each, not on from where another's threads have put them."""
    import torch
    one, bits = caches(G, 2, (9, 2, 16, 64), getattr(torch, dtype), 4)
    k, v = one.caches
    s = G.CacheSet([k, v, k, k[:], v])
    assert len(s.caches) == 5 and s.count == 2 and s.pointers.tolist() == [k.data_ptr(), v.data_ptr()]
    # every row behind the first goes one place to the front: moved twice, it would go two
    table, n = np.array([[3, 1, 8, 0]]), 60
    G.keep_tokens(s, dev(table), dev([2]), dev(np.arange(1, n + 1)[None]), dev([n]))
    G.copy_blocks(s, dev([[3, 5]]), dev([1]))
    for w, t in zip(bits, (k, v)):
        src, dst = 2 + np.arange(1, n + 1), 2 + np.arange(n)
        w[table[0, dst // 16], :, dst % 16] = w[table[0, src // 16], :, src % 16]
        w[5] = w[3]
        assert (bits_of(t) == w).all()


def test_caches_that_overlap_are_refused(G):  # noqa: F811
    import torch
    flat = torch.zeros(7, 2, 16, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        G.CacheSet([flat[:4], flat[3:]])
    assert G.CacheSet([flat[:3], flat[3:6]]).count == 2
