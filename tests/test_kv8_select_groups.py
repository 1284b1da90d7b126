"""Selection's scores are whole numbers of 32 bits: groups whose scores may pass them are refused."""
import pytest

from test_kv8_abi import FAKE, L, attn, cache, seqs


@pytest.mark.parametrize("D", [64, 128, 256])
def test_groups_whose_scores_overflow(D):
    most = (2 ** 31 - 1) // (127 * 127 * D)
    c = cache(head_dim=D)
    for group, ok in ((most, True), (most + 1, False), (4 * most, False)):
        a = attn(n_q_heads=2 * group, n_picks=2)
        need = L().cg_kv8_select_workspace_bytes(c, seqs(), a)
        assert (need > 0) == ok
        # (with too little scratch a shape that is taken is refused for that)
        code = L().cg_kv8_select(c, seqs(), a, 1, FAKE, FAKE, max(0, need - 1), None)
        assert code == (-3 if ok else -2)
