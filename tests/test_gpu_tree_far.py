"""Trees whose tokens are said to have positions far from each other and from the keys in front of them: slopes go by distances of up to
2^32, of either sign."""
import numpy as np
import pytest

from test_gpu_tree import G, Trees  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

FAR = [-2 ** 31, -2 ** 31 + 77, -2 ** 30, -5, 40, 2 ** 30 + 3, 2 ** 31 - 90, 2 ** 31 - 1]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("dtype,shape", [("f16", (8, 2, 64, 16, 0, [100, 40], [30, 40])), ("bf16", (16, 2, 128, 16, 0, [300, 17, 700], [24, 16, 64])),
                                         ("f16", (8, 1, 128, 16, 3, [60, 48 + 5, 200], [12, 5, 31])), ("bf16", (32, 8, 64, 32, 8, [256 + 7, 400], [7, 60]))])
def test_any_positions(G, dtype, shape, kv8):  # noqa: F811
    """Slopes of 2^-30 to 2^-29: a distance's share of a score is up to 8, and off by less than 2^-20 where it is rounded to 24 bits; one whose
    sign has turned changes the weights by a factor of e^4 and more."""
    t = Trees(len(shape[5]), dtype, *shape, kind="any", slopes=True, kv8=kv8)
    rng = np.random.RandomState(3)
    t.positions = (rng.choice(FAR, t.T) + 0).astype(np.int32)
    t.slopes = (2.0 ** -30 * (1 + t.slopes)).float()
    t.upload()
    t.check(t.run(G))
