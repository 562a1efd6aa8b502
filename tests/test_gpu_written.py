"""What a call writes in place torch knows of: a tensor saved for a backward pass and then written is an error there, not another
gradient."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_stepped_weight():
    import torch

    import paper_2603_08957_amd as tre

    w = torch.randn(64, device="cuda", requires_grad=True)
    p, state = torch.ones(5, device="cuda"), tre.adamw_state([w, torch.ones(5, device="cuda")])
    g = [torch.ones(64, device="cuda"), torch.ones(5, device="cuda")]
    out = (w * w).sum()
    was = [t._version for t in (w, p, state, g[0])]
    tre.adamw([w, p], g, state, 1, 1e-3)
    assert [t._version for t in (w, p, state, g[0])] == [was[0] + 1, was[1] + 1, was[2] + 1, was[3]]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()
    with pytest.raises(tre.TreError):  # (nothing is written)
        tre.adamw([w, p], g, state, 0, 1e-3)
    assert w._version == was[0] + 1
    (w * w).sum().backward()
    assert torch.equal(w.grad, 2 * w.detach())


def test_scores_in_place():
    import torch

    import paper_2603_08957_amd as tre

    x = torch.randn(4, 50, device="cuda")
    a = torch.ones((), device="cuda", requires_grad=True)
    loss = (a * x).sum()
    ids, g = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.ones(4, device="cuda")
    r = tre.log_probs(x, ids)
    was = x._version
    tre.log_probs_grad(x, r.stats, ids, g)
    assert x._version == was
    tre.log_probs_grad(x, r.stats, ids, g, out=x)
    assert x._version == was + 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    out = torch.zeros(2, device="cuda")
    tre.grad_norm([x], out=out)
    assert out._version == 1


def test_inference_mode():
    import torch

    import paper_2603_08957_amd as tre

    with torch.inference_mode():
        p, g = [torch.ones(5, device="cuda")], [torch.ones(5, device="cuda")]
        state = tre.adamw_state(p)
        tre.adamw(p, g, state, 1, 1e-3)
    tre.adamw(p, g, state, 2, 1e-3)
    assert (p[0] != 1).all()
