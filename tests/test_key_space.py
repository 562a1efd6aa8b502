"""Output keys whose number passes 64 bits: the bound on a call's keys is its pairs, on the CPU."""
import pytest


@pytest.mark.parametrize("bits", [(18, 19, 27), (20, 20, 24), (21, 21, 21), (30, 30, 4), (19, 19, 26), (12, 25, 27), (16, 16, 5), (1, 1, 1)])
def test_key_bound(bits):
    """a, b from U and c from V: every pair may have a key of its own, 2^64 of them and more too."""
    import paper_2603_08957_amd as tre

    plan = tre.Plan("ab,c->abc", "abc", {l: 1 << b for l, b in zip("abc", bits)}, {l: 1 for l in "abc"})
    for n_u, n_v in ((5, 7), (1000, 3), (1 << 16, 1 << 10)):
        ws = plan.workspace_bytes(n_u, n_v, n_u * n_v)
        pairs, keys, _ = tre.output_bounds(plan, n_u, n_v, ws)
        assert pairs == n_u * n_v and keys == min(pairs, 1 << sum(bits))


def test_workspace_grows_with_pairs():
    """The partial tiles of a contraction that is split over U do not vanish where the key space passes 64 bits."""
    import paper_2603_08957_amd as tre

    def need(bits):
        ext = {l: 128 << b for l, b in zip("ik", bits)}
        ext.update(j=128, a=1 << bits[2])
        plan = tre.Plan("aij,jk->ika", "aik", ext, {"a": 1, "i": 128, "k": 128}, "bf16", u_ranges=2)
        return plan.workspace_bytes(300, 300, 90000)

    assert need((18, 18, 28)) == need((17, 17, 27)) == need((20, 20, 20))
