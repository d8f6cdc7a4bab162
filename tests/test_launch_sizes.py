"""CPU: calls whose launches would have 2^32 threads and more in a dimension, which the runtime cuts off without an error."""
from test_operators_host import G, ONE  # noqa: F401  (G: a fixture)


def test_verification(G):
    def v(B):
        return G.load_library().optgqa_verify_drafts(ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, B, 1, 1, 1, 1, None, 0, 2, None)
    assert v((1 << 22) - 1) == -4 and v(1 << 22) == -2           # (no workspace: the next thing that is looked at)


def test_common_prefix(G):
    def c(T, B, Hq, Hkv, Lmax):
        return G.load_library().optgqa_paged_attention_common(ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, None, 0.1, T, B, Hq, Hkv, 64, 16, 4, 1000, Lmax, 1, None, 0, 0, None)
    # the join has a workgroup for 32 rows of a KV head: 2^24 - 1 of them
    T = 32 * ((1 << 24) - 1) // 32
    assert c(T, 1, 32, 1, 64) == -4 and G.common_prefix_workspace_bytes(T, 1, 32, 1, 64, 16, 4, 64, 1) > 0
    assert c(T + 1, 1, 32, 1, 64) == -2 and G.common_prefix_workspace_bytes(T + 1, 1, 32, 1, 64, 16, 4, 64, 1) == 0
    # own parts: one for each sequence and KV head, and the shares
    assert c(1 << 20, 1 << 20, 8, 8, 1000) == -4
    assert c(1 << 21, 1 << 21, 8, 8, 1000) == -2 and G.common_prefix_workspace_bytes(1 << 21, 1 << 21, 8, 8, 64, 16, 4, 1000, 1) == 0
