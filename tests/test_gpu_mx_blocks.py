"""EinSums over 4-bit tiles that fill the chip, each size one whose workgroups
take a certain block of outputs (64 x 64 to 128 x 256, as the call's timing
reports it): ragged edges, one stage of copies and many, several pairs to a
key, cut keys, batches, outputs of every order and type, against float64 on the
values that the tiles stand for (read back, which other tests hold to the
oracle).

A product of two 4-bit values under their powers of two is exact in fp32; n
additions are off by at most n 2^-24 of the sum of magnitudes, n the contracted
extent of a key's pairs padded to blocks and the partial sums.  A bf16 result is
rounded once more, by at most 2^-8 of its value.
"""
import pytest

from oracle import microscaled as mx

pytestmark = pytest.mark.gpu

U32, UB16 = 2.0 ** -24, 2.0 ** -8


def block(tm):
    return tm.contract_block >> 16, tm.contract_block & 0xffff


def near(got, ref, mag, terms, w_bf16):
    """terms: a number, or one for each tile of the first dimension."""
    err = (got.double() - ref).abs()
    tol = terms * U32 * mag
    if w_bf16:
        tol = tol * (1 + UB16) + UB16 * ref.abs()
    assert bool((err <= tol).all())
    assert float((got.double() - ref).norm() / ref.norm()) <= (UB16 if w_bf16 else 1e-6)


def values(plan, n, shape, operand, g):
    """Quantised tiles and what they stand for."""
    import torch

    import paper_2603_08957_amd as tre

    x = torch.randn((n, *shape), generator=g, device="cuda") * torch.exp2(torch.randint(-3, 4, (n, *[1] * len(shape)), generator=g,
                                                                                      device="cuda").float())
    q = tre.mx_quantize(plan, operand, x.view(n, -1))
    return q, tre.mx_dequantize(plan, operand, q).double().view(n, *shape)


def outputs(plan, n_w):
    """Buffers for n_w tiles, and one behind them that has to stay."""
    import torch

    wk = torch.full((n_w + 1, plan.key_arity[2]), -9, dtype=torch.int32, device="cuda")
    wt = torch.full((n_w + 1, plan.tile_elems[2]), -3.0, dtype=torch.bfloat16 if plan.w_bf16 else torch.float32, device="cuda")
    return wk, wt


def call(plan, uk, uq, vk, vq, n_w, n_pairs):
    import torch

    import paper_2603_08957_amd as tre

    ws = tre.alloc_workspace(plan.workspace_bytes(uq.shape[0], vq.shape[0], n_pairs))
    wk, wt = outputs(plan, n_w)
    tm = tre.Timing()
    assert tre.execute(plan, uk, uq, vk, vq, wk[:n_w], wt[:n_w], ws, timing=tm) == (n_w, n_pairs)
    # rows behind the last stay as they were
    assert torch.all(wt[n_w] == -3.0) and torch.all(wk[n_w] == -9)
    return wk[:n_w], wt[:n_w], tm


def range_keys(n):
    import torch

    return torch.arange(n, dtype=torch.int32, device="cuda").reshape(n, 1)


GRIDS = [  # rows and columns of a tile, tiles, groups of 128 of a row, block
    (67, 195, 23, 17, 7, (128, 256)), (257, 452, 26, 3, 5, (128, 256)),
    (130, 70, 10, 26, 9, (128, 128)), (129, 352, 18, 5, 5, (128, 128)),
    (66, 66, 16, 25, 9, (128, 64)), (203, 260, 11, 7, 3, (128, 64)), (69, 66, 23, 17, 2, (128, 64)),
    (34, 207, 35, 11, 2, (64, 256)), (129, 390, 16, 5, 3, (64, 256)),
    (50, 60, 33, 31, 5, (64, 64)), (144, 276, 2, 2, 3, (64, 64)), (130, 70, 5, 6, 1, (64, 64)),
]


@pytest.mark.parametrize("form", ["f32", "bf16", "across", "odd"])
@pytest.mark.parametrize("m,n,a,b,groups,want", GRIDS)
def test_grids(m, n, a, b, groups, want, form):
    """Two grids of tiles, one pair to a key.  across: W's tiles hold the other
    operand's label first; odd: bf16 outputs whose places come out of tables."""
    import torch

    k = 128 * groups - 37
    g = torch.Generator(device="cuda").manual_seed(m * n)
    import paper_2603_08957_amd as tre

    ext = {"n": m * a, "v": n * b, "d": k, "c": 1}
    if form == "odd":  # columns of two labels, the second beside the rows in memory
        n = n // 2 * 2
        ext = {"n": m * a, "v": n // 2 * b, "d": k, "c": 2}
        plan = tre.Plan("nd,vcd->vnc", "nv", ext, {"n": m, "v": n // 2}, "mxfp4", w_bf16=True)
    else:
        e = {"across": "vd,nd->nv"}.get(form, "nd,vd->nv")
        plan = tre.Plan(e, "nv", ext, {"n": m, "v": n}, "mxfp4", w_bf16=form == "bf16")
    if form == "across":
        uq, ud = values(plan, b, (n, k), "u", g)
        vq, vd = values(plan, a, (m, k), "v", g)
        rows, cols = vd, ud
    else:
        uq, ud = values(plan, a, (m, k), "u", g)
        vq, vd = values(plan, b, (n, k), "v", g)
        rows, cols = ud, vd
    wk, wt, tm = call(plan, range_keys(uq.shape[0]), uq, range_keys(vq.shape[0]), vq, a * b, a * b)
    assert block(tm) == want
    dense, scale = rows.reshape(a * m, k), cols.reshape(b * n, k)
    ref = (dense @ scale.T).view(a, m, b, n)
    mag = (dense.abs() @ scale.abs().T).view(a, m, b, n)
    if form == "odd":
        assert torch.equal(wk, torch.cartesian_prod(torch.arange(b), torch.arange(a)).to(torch.int32).cuda())
        order = lambda x: x.view(a, m, b, n // 2, 2).permute(2, 0, 3, 1, 4).reshape(a * b, -1)  # noqa: E731
    else:
        assert torch.equal(wk, torch.cartesian_prod(torch.arange(a), torch.arange(b)).to(torch.int32).cuda())
        order = lambda x: x.permute(0, 2, 1, 3).reshape(a * b, -1)  # noqa: E731
    near(wt, order(ref), order(mag), 32 * mx.row_blocks(k) + 2, plan.w_bf16)


BATCHES = [(65, 195, 38, 4, 5, (128, 256)), (67, 65, 18, 10, 5, (128, 128)), (66, 69, 15, 9, 7, (128, 64)),
           (35, 199, 11, 12, 9, (64, 256)), (40, 50, 5, 7, 2, (64, 64))]


@pytest.mark.parametrize("w_bf16", [False, True])
@pytest.mark.parametrize("m,n,a,b,groups,want", BATCHES)
def test_batches(m, n, a, b, groups, want, w_bf16):
    import torch

    import paper_2603_08957_amd as tre

    k = 128 * groups - 5
    g = torch.Generator(device="cuda").manual_seed(m + n)
    plan = tre.Plan("hnd,hvd->hnv", "nv", {"h": 3, "n": m * a, "v": n * b, "d": k}, {"n": m, "v": n}, "mxfp4", w_bf16=w_bf16)
    uq, ud = values(plan, a, (3, m, k), "u", g)
    vq, vd = values(plan, b, (3, n, k), "v", g)
    _, wt, tm = call(plan, range_keys(a), uq, range_keys(b), vq, a * b, a * b)
    assert block(tm) == want
    x, y = ud.transpose(0, 1).reshape(3, a * m, k).contiguous(), vd.transpose(0, 1).reshape(3, b * n, k).contiguous()
    yt = y.transpose(1, 2).contiguous()
    order = lambda z: z.view(3, a, m, b, n).permute(1, 3, 0, 2, 4).reshape(a * b, -1)  # noqa: E731
    near(wt, order(torch.bmm(x, yt)), order(torch.bmm(x.abs(), yt.abs())), 32 * mx.row_blocks(k) + 2, w_bf16)


SPARSE = [  # rows and columns of a tile (columns and rows in `across`), keys, pairs of a key on average, longest unit (0: whole keys), block
    (66, 193, 395, 9, 0, (128, 256)), (66, 193, 2560, 12, 0, (128, 256)), (131, 65, 259, 7, 0, (128, 128)), (65, 65, 388, 12, 0, (128, 64)),
    (33, 200, 386, 7, 0, (64, 256)), (40, 40, 30, 3, 0, (64, 64)),
    (65, 194, 161, 12, 7, (128, 256)), (66, 68, 192, 12, 7, (128, 128)), (66, 65, 124, 12, 5, (128, 64)),
    (33, 198, 120, 12, 5, (64, 256)), (40, 40, 30, 12, 2, (64, 64)),
]


@pytest.mark.parametrize("form", ["f32", "bf16", "across"])
@pytest.mark.parametrize("m,n,keys,avg,unit,want", SPARSE)
def test_sparse_rows(m, n, keys, avg, unit, want, form):
    """Keys of 1 to 2 avg - 1 pairs, each one stage of copies: whole (as the join
    left them, or longest first), or cut into units whose partial tiles are
    summed after."""
    import torch

    import paper_2603_08957_amd as tre

    k, nj = 100, 24
    w_bf16 = form == "bf16"
    if form == "across":
        m, n = n, m
    g = torch.Generator(device="cuda").manual_seed(keys + avg)
    plan = tre.Plan("ij,jk->ki" if form == "across" else "ij,jk->ik", "ij", {"i": m * keys, "j": k * nj, "k": n},
                    {"i": m, "j": k}, "mxfp4", w_bf16=w_bf16, max_pairs_per_unit=unit)
    counts = [1 + i % (2 * avg - 1) for i in range(keys)]
    pick = torch.Generator().manual_seed(keys)
    ij = [(i, j) for i, c in enumerate(counts) for j in sorted(torch.randperm(nj, generator=pick)[:c].tolist())]
    uk = torch.tensor(ij, dtype=torch.int32, device="cuda")
    uq, ud = values(plan, len(ij), (m, k), "u", g)
    vq, vd = values(plan, nj, (k, n), "v", g)
    wk, wt, tm = call(plan, uk, uq, range_keys(nj), vq, keys, len(ij))
    assert block(tm) == want
    assert unit or tm.n_units == keys
    assert tm.n_split_segments == (sum(c > unit for c in counts) if unit else 0)
    assert torch.equal(wk, range_keys(keys))
    at = uk[:, 0].long()
    right = vd[uk[:, 1].long()].contiguous()
    ref = torch.zeros((keys, m, n), dtype=torch.float64, device="cuda").index_add_(0, at, torch.bmm(ud, right))
    mag = torch.zeros_like(ref).index_add_(0, at, torch.bmm(ud.abs(), right.abs()))
    terms = torch.tensor(counts, device="cuda").double().mul_(32 * mx.row_blocks(k) + 2).view(keys, 1)
    order = lambda z: (z.transpose(1, 2) if form == "across" else z).reshape(keys, -1)  # noqa: E731
    near(wt, order(ref), order(mag), terms, w_bf16)


@pytest.mark.parametrize("upper", ["", "n"])
@pytest.mark.parametrize("m,n,k,want", [(2048, 2048, 8192, (128, 64)), (1500, 1700, 900, (64, 64)), (4000, 3900, 260, (128, 64)),
                                        (2900, 3000, 700, (128, 128)), (3000, 5000, 1000, (128, 256))])
def test_one_product(m, n, k, want, upper):
    """A product of two whole matrices is one unit, and of two tiles against one
    two: the block follows that count."""
    import torch

    import paper_2603_08957_amd as tre

    g = torch.Generator(device="cuda").manual_seed(m + n)
    parts = 2 if upper else 1
    plan = tre.Plan("nd,vd->nv", upper, {"n": m, "v": n, "d": k}, {"n": m // parts}, "mxfp4")
    uq, ud = values(plan, parts, (m // parts, k), "u", g)
    vq, vd = values(plan, 1, (n, k), "v", g)
    _, wt, tm = call(plan, range_keys(2) if upper else None, uq, None, vq, parts, parts)
    assert tm.n_units == parts and block(tm) == want
    x, y = ud.view(m, k), vd.view(n, k)
    near(wt.view(m, n), x @ y.T, x.abs() @ y.abs().T, 32 * mx.row_blocks(k) + 2, False)
