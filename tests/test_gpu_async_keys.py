"""Asynchronous calls over keys that are not in order, whose pairs are not
grouped by output key: segments that end before they begin, and ones that reach
over nearly all pairs.  The call says so in its counts and contracts nothing; it
writes nothing behind its workspace or its outputs, and the same buffers then
serve a call whose keys are in order."""
import pytest

pytestmark = pytest.mark.gpu

KINDS = [  # dtype, tile of i and k, tile of j, options
    ("f32", 4, 4, {"max_pairs_per_unit": 4}), ("f32", 16, 16, {"max_pairs_per_unit": 4}), ("f32", 16, 16, {}),
    ("bf16", 128, 64, {"max_pairs_per_unit": 4}), ("bf16", 128, 64, {}), ("bf16", 128, 64, {"pace_windows": 2}),
    ("mxfp4", 64, 128, {"max_pairs_per_unit": 4}), ("mxfp4", 64, 128, {}), ("mxfp4", 16, 32, {"max_pairs_per_unit": 4}),
    ("mxfp4", 16, 32, {}),
]


@pytest.mark.parametrize("dtype,t,tj,opt", KINDS)
def test_keys_out_of_order(dtype, t, tj, opt):
    import torch

    import paper_2603_08957_amd as tre

    ni, nj = 100, 1500
    ext, til = {"i": ni * t, "j": nj * tj, "k": t}, {"i": t, "j": tj}
    plan = tre.Plan("ij,jk->ik", "ij", ext, til, dtype, small_join=-1, **opt)
    rows = list(range(0, ni - 2, 2)) + [ni - 2] * nj + list(range(1, ni, 2))
    cols = [0] * (ni // 2 - 1) + list(range(nj)) + [1] * (ni // 2)
    bad = torch.tensor([rows, cols], dtype=torch.int32).T.contiguous()
    good = bad[torch.argsort(bad[:, 0].long() * nj + bad[:, 1].long())].contiguous().cuda()
    bad = bad.cuda()
    n = len(rows)
    g = torch.Generator(device="cuda").manual_seed(t)
    # whole numbers: every sum is exact, in 4 bits too
    u = torch.randint(-2, 3, (n, t * tj), generator=g, device="cuda").float()
    v = torch.randint(-2, 3, (nj, tj * t), generator=g, device="cuda").float()
    vk = torch.arange(nj, dtype=torch.int32, device="cuda").reshape(nj, 1)
    right = v.view(nj, tj, t)[good[:, 1].long()].contiguous()
    want = torch.zeros((ni, t, t), device="cuda").index_add_(0, good[:, 0].long(), torch.bmm(u.view(n, t, tj), right))
    if dtype == "mxfp4":
        u, v = tre.mx_quantize(plan, "u", u), tre.mx_quantize(plan, "v", v)
    elif dtype == "bf16":
        u, v = u.to(torch.bfloat16), v.to(torch.bfloat16)
    need = plan.workspace_bytes(n, nj, n)
    buf = torch.full((need + (16 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    ws = buf[:need]
    _, bound, ok = tre.output_bounds(plan, n, nj, need)
    assert ok and bound == ni
    wk = torch.full((ni + 50, 1), -9, dtype=torch.int32, device="cuda")
    wt = torch.full((ni + 50, t * t), -3.0, device="cuda")
    counts = torch.zeros(4, dtype=torch.int64, device="cuda")
    for keys, status in ((bad, "TRE_E_UNSORTED"), (good, "TRE_OK"), (bad, "TRE_E_UNSORTED"), (good, "TRE_OK")):
        wt[:ni] = -3.0
        tre.execute_async(plan, keys, u, vk, v, wk[:ni], wt[:ni], ws, counts)
        torch.cuda.synchronize()
        assert counts[2].item() == tre.tre.STATUS_CODE[status]
        assert bool((buf[need:] == 0x5A).all()) and bool((wt[ni:] == -3.0).all()) and bool((wk[ni:] == -9).all())
        if status == "TRE_OK":
            assert counts[:2].tolist() == [n, ni]
            assert torch.equal(wt[:ni].view(ni, t, t), want)
        else:
            assert bool((wt == -3.0).all())
