"""AdamW steps whose second moments' roots are as small as eps, or whose eps is: against numpy in 64 bits.

With u = 2^-24 the part that is taken off a weight is off by c1, c2 / 2, lr and eps rounded (3.5 u), a root and a reciprocal
good to one unit (2 u each), five products and a sum (6 u), and a root below 2^-63 beside an eps of 2^-39 or more (u): under 16 u
of it.  The weight's own factor and product take 2 u, the last sum one more u of the result.
"""
import numpy as np
import pytest

from oracle import moments

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-8, 2.0 ** -39, 1.5e-12, 1e-15, 1e-20, 1e-22, 2.0 ** -100, 2.0 ** -126])
def test_small_second_moments(eps, bits):
    """Gradients from 1e-23, whose squares hardly are numbers, up to 1e-10, and none: a weight without moments stays."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(11)
    n = 32 * 200
    size = 10.0 ** rng.uniform(-23, -10, n // 32).repeat(32)
    size[:64] = 0
    g = (rng.standard_normal(n) * size).astype(np.float32)
    for t, beta1, beta2 in ((1, 0.0, 0.5), (2, 0.9, 0.999)):
        p = torch.zeros(n, device="cuda")
        state = tre.adamw_state([p], bits)
        tre.adamw([p], [torch.from_numpy(g).cuda()], state, t, 2.0 ** -7, beta1=beta1, beta2=beta2, eps=eps)
        m, v = moments.step32(np.zeros(n, np.float32), np.zeros(n, np.float32), g, beta1, beta2, 1.0)
        want, off = moments.weights64(np.zeros(n), m, v, t, 2.0 ** -7, beta1, beta2, float(np.float32(eps)), 0.0)
        # (no product lies below 2^-126: lr m c1 is 2^-110 and more where a gradient is not zero)
        tol = 16 * U * off + U * np.abs(want)
        got = p.double().cpu().numpy()
        ok = np.abs(want) < 1e38
        assert ok.any() and (got[:64] == 0).all()
        assert np.all(np.abs(got - want)[ok] <= tol[ok]), (np.abs(got - want)[ok] / np.maximum(np.abs(want)[ok], 1e-300)).max() / U
