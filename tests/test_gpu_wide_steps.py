"""Scores, gradients and weights of more than 2^32 elements, and launches of more than 2^32 threads: past those points the same
as in a small call."""
import math

import numpy as np
import pytest

from oracle import moments

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _memory():
    import torch

    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 200 << 30:
        pytest.skip("200 GiB of GPU memory wanted")
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,vocab,tile", [((1 << 26) + 5, 75, 0), (70001, 65536, 0), (70001, 65536, 128), (3, 1 << 30, 0), (2, 1 << 30, 1 << 21)])
def test_log_probs(n, vocab, tile):
    """A wavefront to a row, four, and rows cut into parts; rows and tiles."""
    import torch

    import paper_2603_08957_amd as tre

    shape = (vocab // tile, n, tile) if tile else (n, vocab)
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_()
    ids = torch.randint(0, vocab, (n,), device="cuda")
    r = tre.log_probs(x, ids, top=3, entropy=True)
    g = torch.full((n,), 0.5, device="cuda")
    few = 1000 if n > 1000 else n - 1  # the last rows
    at = n - few
    part = (x[:, at:] if tile else x[at:]).contiguous()
    small = tre.log_probs(part, ids[at:].contiguous(), top=3, entropy=True)
    for a, b in zip(vars(r).values(), vars(small).values()):
        if a.dtype == torch.int32:
            assert torch.equal(a[at:], b)
        else:  # (few rows are cut otherwise: sums in another order)
            assert ((a[at:] - b).abs() <= (vocab + 40) * 2.0 ** -24 * (2 + b.abs()) * 20).all()
    want = tre.log_probs_grad(part, small.stats, ids[at:].contiguous(), g[at:])
    tre.log_probs_grad(x, torch.cat([r.stats[:at], small.stats]), ids, g, out=x)
    assert torch.equal(x[:, at:] if tile else x[at:], want)
    # every row's gradient adds to zero, but for the rounding of each value (its half, 2^-8 of it: of 1 in all)
    rows = (x[:, ::max(1, n // 50)] if tile else x[::max(1, n // 50)]).float()
    total = rows.sum((0, 2) if tile else 1)
    assert (total.abs() <= 2.0 ** -7).all()


def test_norm_and_step_in_32_bits():
    import torch

    import paper_2603_08957_amd as tre

    n = (1 << 33) + 37
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    g[-1] = 64.0
    norm = tre.grad_norm([g], max_norm=1.0)
    want = math.sqrt((n - 1) * 2.0 ** -20 + 4096)
    assert abs(norm[0].item() - want) <= 2.0 ** -23 * want
    state = tre.adamw_state([p], 32)
    tre.adamw([p], [g], state, 1, 1e-2, grad_scale=norm[1:])
    tail = 4096 + 5
    at = n - tail - (n - tail) % 32
    q, h = torch.zeros(n - at, dtype=torch.bfloat16, device="cuda"), g[at:].clone()
    small = tre.adamw_state([q], 32)
    tre.adamw([q], [h], small, 1, 1e-2, grad_scale=norm[1:])
    assert torch.equal(p[at:], q)
    for a, b in zip(tre.adamw_moments(state), tre.adamw_moments(small)):
        assert torch.equal(a[at:], b)
    assert (p[:1 << 20] == p[0]).all() and p[0] != 0 and (p[1 << 32:(1 << 32) + (1 << 20)] == p[0]).all()


def test_step_in_8_bits_by_chance():
    """Elements past 2^32 draw by their whole number; the tensor that crosses it lies behind another."""
    import torch

    import paper_2603_08957_amd as tre

    sizes = [1000, (1 << 32) + 4000, 77]
    params = [torch.ones(s, dtype=torch.bfloat16, device="cuda") for s in sizes]
    grads = [torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_() for s in sizes]
    state = tre.adamw_state(params, 8)
    tre.adamw(params, grads, state, 3, 1e-2, beta1=0.5, beta2=0.75, seed=99)
    total = state.numel() * 16 // 33
    codes_m, codes_v, bytes_m, bytes_v = state.split([total, total, total // 32, total // 32])
    for start in (1024, 1 << 32, (1 << 32) - 2048, (1 << 32) + 1024):
        lo = start - 1024  # (the second tensor begins at element 1024)
        g = grads[1][lo:lo + 2048].float().cpu().numpy()
        m, v = moments.step32(np.zeros(2048, np.float32), np.zeros(2048, np.float32), g, 0.5, 0.75, 1.0)
        r = moments.chance(2048, 99, 3, start)
        want = moments.pack(m, v, r[:2])
        at = slice(start, start + 2048)
        got = torch.cat([codes_m[at], codes_v[at], bytes_m[start // 32:start // 32 + 64], bytes_v[start // 32:start // 32 + 64]])
        assert np.array_equal(got.cpu().numpy(), want), start
    m, v = tre.adamw_moments(state, dtype=torch.bfloat16)
    gm = grads[1][-4000:].float() * 0.5
    assert ((m[1024 + sizes[1] - 4000:1024 + sizes[1]].float() - gm).abs() <= gm.abs() / 8 + 2.0 ** -9).all()
