"""4-bit tiles on the GPU: quantising and reading back bit for bit against the
oracle, and EinSums over them against float64.

Sums: a product of two E2M1 values under their powers of two is exact in fp32,
so only the additions round.  n additions in fp32 in any order are off by at
most n 2^-24 of the sum of magnitudes (to first order); n is the contracted
extent of all pairs of a key, padded to blocks, plus the partial sums.  A bf16
result is rounded once more, by at most 2^-8 of its value.
"""
import itertools

import numpy as np
import pytest

from oracle import microscaled as mx

pytestmark = pytest.mark.gpu

U32, UB16 = 2.0 ** -24, 2.0 ** -8


def bf16(x):
    import torch

    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def special(rng, n, rows, k):
    """Values over many powers of two, with every kind of block among them."""
    x = rng.standard_normal((n, rows, k)) * np.exp2(rng.integers(-20, 20, (n, rows, 1)).astype(float))
    x = x.astype(np.float32)
    flat = x.reshape(-1, k)
    grid = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.75, -0.25, -0.75, -5, -0.0], np.float32)
    for i in range(0, flat.shape[0], 3):  # values on and beside the borders
        flat[i] = rng.choice(grid, k) * np.float32(2.0 ** rng.integers(-30, 30))
        flat[i] = np.nextafter(flat[i], rng.choice(np.array([-np.inf, np.inf], np.float32), k)) if i % 2 else flat[i]
    picks = [0.0, 1e-45, 2.0 ** -130, 2.0 ** -126, 2.0 ** -124, 3.4e38, np.inf, -np.inf, np.nan]
    for j, v in enumerate(picks):
        if flat.shape[0] > j + 1:
            if v == 0 or abs(v) < 1e-30:
                flat[j + 1] = 0
            flat[j + 1, k // 2] = v
    return x


FORMS = [  # (einsum, operand, the operand's labels in rows and contracted order are not its own order everywhere)
    ("ik,jk->ij", 0), ("ik,jk->ij", 1), ("ki,jk->ij", 0), ("ik,kj->ij", 1), ("ik,kj->ji", 0),
    ("bik,bjk->bij", 0), ("kib,bkj->ijb", 1), ("ikl,jlk->ij", 1), ("kil,jlk->ij", 0), ("aikc,ckj->jai", 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("einsum,op", FORMS)
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 5), (16, 31), (17, 32), (5, 33), (64, 64), (7, 65), (33, 96), (128, 128),
                                    (9, 130), (65, 257), (130, 100), (8, 1000)])
def test_quantize_and_back(einsum, op, rows, k, dtype):
    import torch

    import paper_2603_08957_amd as tre

    own, rl, kl = mx.roles(einsum, op)
    sizes = {c: 1 for c in "abcijkl"}
    # rows and k spread over the labels that stand for them
    for labels, total in ((rl, rows), (kl, k)):
        for c in labels[:-1]:
            sizes[c] = 2
        sizes[labels[-1]] = total
    other = {c: 3 for c in einsum if c.isalpha() and c not in own}
    plan = tre.Plan(einsum, "", {**{c: sizes[c] for c in own}, **other}, {}, "mxfp4")
    rng = np.random.default_rng(rows * 1000 + k)
    R, K = int(np.prod([sizes[c] for c in rl])), int(np.prod([sizes[c] for c in kl]))
    n = 3
    m = special(rng, n, R, K)
    if dtype == "bf16":
        m = bf16(m).float().numpy()
    # into the operand's own order
    t = m.reshape([n] + [sizes[c] for c in rl + kl]).transpose([0] + [1 + (rl + kl).index(c) for c in own])
    t = np.ascontiguousarray(t).reshape(n, -1)
    dev = (bf16(t) if dtype == "bf16" else torch.from_numpy(t)).cuda()
    assert plan.tile_bytes[op] == mx.tile_bytes(R, K)
    # written whole, and nothing behind it
    buf = torch.full((n + 1, plan.tile_bytes[op]), 0xA5, dtype=torch.uint8, device="cuda")
    q = tre.mx_quantize(plan, "uv"[op], dev, out=buf[:n])
    codes, scales = mx.encode(mx.matrix(einsum, op, sizes, t.astype(np.float64)))
    want = mx.pack(codes, scales)
    used = 17 * R * mx.row_blocks(K)
    got = buf.cpu().numpy()
    # (codes of blocks that are not finite stand for nothing)
    bad = np.repeat(want[:, 16 * R * mx.row_blocks(K):used] == 255, 16, axis=1)
    assert np.array_equal(got[:n, 16 * R * mx.row_blocks(K):used], want[:, 16 * R * mx.row_blocks(K):used]), "scales"
    assert np.array_equal(np.where(bad, 0, got[:n, :bad.shape[1]]), np.where(bad, 0, want[:, :bad.shape[1]])), "codes"
    assert np.all(got[n] == 0xA5)
    ref = mx.values(einsum, op, sizes, t.astype(np.float64))
    for dt in (torch.float32, torch.bfloat16):
        out = torch.full((n + 1, plan.tile_elems[op]), -7.0, dtype=dt, device="cuda")
        tre.mx_dequantize(plan, "uv"[op], q, out=out[:n])
        v = out.double().cpu().numpy()
        assert np.array_equal(v[:n], ref, equal_nan=True), dt
        assert np.all(v[n] == -7.0)


def relation(rng, labels, upper, ext, til, keep, dtype):
    """(keys, tiles) of a random relation, float64 tiles already in the type."""
    up = [c for c in labels if c in upper]
    space = [range(ext[c] // til.get(c, 1)) for c in up]
    keys = np.zeros((1, 0), np.int32)
    if up:
        keys = np.array([k for k in itertools.product(*space) if rng.random() < keep], np.int32).reshape(-1, len(up))
    te = int(np.prod([til.get(c, 1) if c in upper else ext[c] for c in labels]))
    t = rng.standard_normal((len(keys), te)) * np.exp2(rng.integers(-3, 4, (len(keys), 1)).astype(float))
    t = t.astype(np.float32)
    return keys, (bf16(t).float().numpy() if dtype == "bf16" else t)


def run(orc, einsum, upper, ext, til, dtype="bf16", seed=0, keep=0.7, w_bf16=False, how="einsum", **opt):
    """Quantise, run, compare with the oracle on the quantised values."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(seed)
    la, lb = einsum.split("->")[0].split(",")
    plan = tre.Plan(einsum, upper, ext, til, "mxfp4", w_bf16=w_bf16, **opt)
    assert plan.kernel_class == "mx"
    sizes = {c: til.get(c, 1) if c in upper else ext[c] for c in ext}
    rel, dev = [], []
    for o, lab in enumerate((la, lb)):
        k, t = relation(rng, lab, upper, ext, til, keep, dtype)
        x = (bf16(t) if dtype == "bf16" else torch.from_numpy(t)).cuda()
        dev += [torch.from_numpy(k).cuda(), tre.mx_quantize(plan, "uv"[o], x)]
        rel.append({"keys": k, "tiles": mx.values(einsum, o, sizes, t.astype(np.float64)).astype(np.float32), "dtype": "f32"})
    ref = orc.run(orc.Plan(einsum, upper, ext, {c: til.get(c, 1) for c in ext}), *rel)
    n_w, n_p = len(ref.wkeys), len(ref.pairs)
    rw, dt = plan.key_arity[2], torch.bfloat16 if w_bf16 else torch.float32
    if how == "einsum":
        out = tre.einsum(plan, *dev, want_pairs=True, timing=True)
        assert out.n_w == n_w and out.n_pairs == n_p
        assert n_p == 0 or out.timing["contract_path"] == "mx"
        assert np.array_equal(out.pairs.cpu().numpy().reshape(n_p, 2), ref.pairs.reshape(n_p, 2))
        wk, wt = out.w_keys, out.w_tiles
    else:
        ws = tre.alloc_workspace(plan.workspace_bytes(dev[1].shape[0], dev[3].shape[0], max(n_p, 1) * 4))
        _, kb, _ = tre.output_bounds(plan, dev[1].shape[0], dev[3].shape[0], ws.numel())
        wk = torch.zeros((max(kb, 1), max(rw, 1)), dtype=torch.int32, device="cuda")
        wt = torch.full((max(kb, 1), plan.tile_elems[2]), -3.0, dtype=dt, device="cuda")
        if how == "async":
            counts = torch.zeros(4, dtype=torch.int64, device="cuda")
            tre.execute_async(plan, *dev, wk, wt, ws, counts)
            assert counts.tolist() == [n_p, n_w, 0, 0]
        elif how == "noalloc":
            assert tre.execute_noalloc(plan, *dev, wk, wt) == (n_w, n_p)
        else:
            assert tre.execute(plan, *dev, wk, wt, ws) == (n_w, n_p)
        # rows behind the last output tile stay as they were
        assert torch.all(wt[n_w:] == -3.0)
    if n_w == 0:
        return plan
    assert np.array_equal(wk[:n_w].cpu().numpy().reshape(n_w, -1)[:, :rw], ref.wkeys.reshape(n_w, -1))
    got = wt[:n_w].double().cpu().numpy().reshape(ref.acc.shape)
    most = max(n_p, 1)  # pairs of one key, at most
    n = most * (32 * mx.row_blocks(plan.bmnk[3]) + 2)
    tol = n * U32 * ref.mag
    if w_bf16:
        tol = tol * (1 + UB16) + UB16 * np.abs(ref.acc)
    err = np.abs(got - ref.acc)
    assert np.all(err <= tol), (err / np.maximum(ref.mag, 1e-300)).max()
    # and nowhere near that in the norm: an fp32 sum of exact products
    rel_norm = np.linalg.norm(got - ref.acc) / max(np.linalg.norm(ref.acc), 1e-300)
    assert rel_norm <= (UB16 if w_bf16 else 1e-6), rel_norm
    return plan


PLANS = [  # einsum, promoted, extents, tiles
    ("ik,jk->ij", "", {"i": 1, "j": 1, "k": 1}, {}),
    ("ik,jk->ij", "", {"i": 17, "j": 70, "k": 100}, {}),
    ("ik,jk->ji", "", {"i": 3, "j": 65, "k": 1000}, {}),                       # W's unit stride along U's rows
    ("vd,nd->nv", "v", {"v": 1280, "n": 1, "d": 96}, {"v": 128}),               # a token's scores
    ("vd,nd->nv", "v", {"v": 500, "n": 13, "d": 1000}, {"v": 50}),
    ("vd,nd->nv", "v", {"v": 600, "n": 40, "d": 520}, {"v": 300}),
    ("ij,jk->ik", "ij", {"i": 512, "j": 512, "k": 100}, {"i": 64, "j": 64}),
    ("ij,jk->ik", "ij", {"i": 128, "j": 320, "k": 33}, {"i": 32, "j": 32}),     # one block a row: pairs share an instruction
    ("ij,jk->ki", "jk", {"i": 40, "j": 200, "k": 200}, {"j": 20, "k": 20}),
    ("ij,jk->ik", "ijk", {"i": 384, "j": 384, "k": 384}, {"i": 96, "j": 96, "k": 96}),
    ("ij,jk->ik", "ijk", {"i": 512, "j": 512, "k": 512}, {"i": 128, "j": 128, "k": 128}),
    ("ij,jk->ik", "ijk", {"i": 520, "j": 520, "k": 520}, {"i": 260, "j": 130, "k": 260}),
    ("nv,nd->vd", "nv", {"n": 256, "v": 384, "d": 200}, {"n": 64, "v": 128}),   # a weight's gradient
    ("bik,bkj->bij", "i", {"b": 3, "i": 96, "j": 50, "k": 40}, {"i": 24}),
    ("bik,kjb->jbi", "k", {"b": 2, "i": 20, "j": 70, "k": 256}, {"k": 32}),
    ("aikc,ckj->jai", "k", {"a": 2, "i": 11, "j": 9, "k": 96, "c": 3}, {"k": 24}),
    ("ij,j->i", "ij", {"i": 60, "j": 80}, {"i": 20, "j": 16}),                  # a matrix and a vector
    ("ij,ij->", "i", {"i": 40, "j": 70}, {"i": 8}),                             # one number
    ("ix,jx->ijx", "", {"i": 5, "j": 6, "x": 7}, {}),                           # nothing contracted
]


@pytest.mark.parametrize("how", ["einsum", "async", "noalloc"])
@pytest.mark.parametrize("case", range(len(PLANS)))
def test_product(orc, case, how):
    e, up, ext, til = PLANS[case]
    run(orc, e, up, ext, til, "bf16", seed=case, how=how)


@pytest.mark.parametrize("case", range(len(PLANS)))
def test_product_bf16_out(orc, case):
    e, up, ext, til = PLANS[case]
    run(orc, e, up, ext, til, "f32", seed=100 + case, w_bf16=True, keep=1.0)


@pytest.mark.parametrize("unit", [1, 2, 3, 7])
def test_product_split_keys(orc, unit):
    """Keys cut into units: partial tiles summed after, in fp32 and bf16."""
    for i, (e, up, ext, til) in enumerate(PLANS):
        if "j" in up or "n" in up and "v" in up:
            run(orc, e, up, ext, til, "bf16", seed=200 + i, max_pairs_per_unit=unit)
            run(orc, e, up, ext, til, "bf16", seed=300 + i, max_pairs_per_unit=unit, w_bf16=True, how="execute")


def test_no_pairs(orc):
    e, up, ext, til = PLANS[6]
    for how in ("einsum", "async", "execute"):
        run(orc, e, up, ext, til, keep=0.0, how=how)


@pytest.mark.parametrize("m,n,k", [(256, 256, 128), (256, 256, 640), (300, 515, 384), (129, 255, 2048), (512, 384, 1024),
                                   (1, 1000, 4096), (16, 260, 1500), (33, 129, 256), (64, 512, 64), (200, 200, 32)])
def test_product_large_tiles(m, n, k):
    """Tiles of several blocks, against float64 on the quantised values (read
    back, which the tests above hold to the oracle)."""
    import torch

    import paper_2603_08957_amd as tre

    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    for e, w_bf16 in (("ik,jk->ij", False), ("ik,jk->ji", True), ("ik,kj->ij", True)):
        plan = tre.Plan(e, "i", {"i": 2 * m, "j": n, "k": k}, {"i": m}, "mxfp4", w_bf16=w_bf16)
        u = torch.randn((2, m * k), generator=g, device="cuda")
        v = torch.randn((1, n * k), generator=g, device="cuda")
        uq, vq = tre.mx_quantize(plan, "u", u), tre.mx_quantize(plan, "v", v)
        ud = tre.mx_dequantize(plan, "u", uq).double().view(2 * m, k)
        vd = tre.mx_dequantize(plan, "v", vq).double()
        vd = vd.view(k, n) if e.startswith("ik,kj") else vd.view(n, k).T
        ref, mag = ud @ vd, ud.abs() @ vd.abs()
        keys = torch.arange(2, dtype=torch.int32, device="cuda").reshape(2, 1)
        out = tre.einsum(plan, keys, uq, None, vq).w_tiles.double()
        out = out.view(2, n, m).transpose(1, 2).reshape(2 * m, n) if e.endswith("ji") else out.view(2 * m, n)
        tol = (k + 128) * U32 * mag + (UB16 * ref.abs() if w_bf16 else 0)
        assert bool(((out - ref).abs() <= tol).all())
        if not w_bf16:
            assert float((out - ref).norm() / ref.norm()) <= 1e-6


def test_not_finite():
    """A block that is not finite makes the sums that it enters NaN, and no others."""
    import torch

    import paper_2603_08957_amd as tre

    for k in (20, 60, 100, 400):
        plan = tre.Plan("ik,jk->ij", "", {"i": 40, "j": 50, "k": k}, {}, "mxfp4")
        u = torch.randn((40, k), device="cuda")
        v = torch.randn((50, k), device="cuda")
        u[3, k // 2], u[39, 0], v[7, k - 1] = float("nan"), float("inf"), -float("inf")
        w = tre.einsum(plan, None, tre.mx_quantize(plan, "u", u.view(1, -1)), None, tre.mx_quantize(plan, "v", v.view(1, -1)))
        bad = torch.zeros((40, 50), dtype=torch.bool, device="cuda")
        bad[3], bad[39], bad[:, 7] = True, True, True
        assert torch.equal(w.w_tiles.view(40, 50).isnan(), bad)


def test_same_bits_streams_and_graphs():
    """Two calls give the same bits; on another stream and replayed from a graph
    too, between eager calls that use the same workspace."""
    import torch

    import paper_2603_08957_amd as tre

    n, c, t = 1024, 200, 64
    plan = tre.Plan("ij,jk->ik", "ij", {"i": n, "j": n, "k": c}, {"i": t, "j": t}, "mxfp4", max_pairs_per_unit=3)
    nb = n // t
    keys = torch.cartesian_prod(torch.arange(nb), torch.arange(nb)).to(torch.int32).cuda()
    bk = torch.arange(nb, dtype=torch.int32, device="cuda").reshape(nb, 1)
    a = torch.randn((nb * nb, t * t), device="cuda").to(torch.bfloat16)
    b = torch.randn((nb, t * c), device="cuda").to(torch.bfloat16)
    ws = tre.alloc_workspace(plan.workspace_bytes(nb * nb, nb, nb * nb))
    wk, wt = torch.zeros((nb, 1), dtype=torch.int32, device="cuda"), torch.zeros((nb, t * c), device="cuda")
    counts = torch.zeros(4, dtype=torch.int64, device="cuda")
    aq, bq = tre.mx_quantize(plan, "u", a), torch.zeros((nb, plan.tile_bytes[1]), dtype=torch.uint8, device="cuda")

    def step():
        tre.mx_quantize(plan, "v", b, out=bq)
        tre.execute_async(plan, keys, aq, bk, bq, wk, wt, ws, counts)

    step()
    torch.cuda.synchronize()
    first = wt.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    wt.zero_()
    side.wait_stream(torch.cuda.current_stream())
    out = tre.mx_quantize(plan, "v", b, stream=side)
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(wt, first) and torch.equal(out, bq)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        b.copy_(torch.randn_like(b.float()))
        step()
        torch.cuda.synchronize()
        want = wt.clone()
        wt.zero_()
        bq.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(wt, want), i


@pytest.mark.parametrize("t,how", [(16, "execute"), (64, "async"), (96, "execute")])
def test_one_long_key(t, how):
    """One key with nearly all pairs, the others with one or none: it is cut and
    its partial tiles summed, with no unit far longer than the launch."""
    import torch

    import paper_2603_08957_amd as tre

    nb, long = 6000, 5000
    plan = tre.Plan("ij,jk->ik", "ij", {"i": nb * t, "j": nb * t, "k": t}, {"i": t, "j": t}, "mxfp4", w_bf16=t == 96)
    g = torch.Generator(device="cuda").manual_seed(t)
    keys = torch.cat([torch.stack([torch.full((long,), 7), torch.arange(long) + 500], 1),
                      torch.stack([torch.arange(8, 408), torch.arange(8, 408)], 1)]).to(torch.int32).cuda()
    a = torch.randn((keys.shape[0], t * t), generator=g, device="cuda")
    b = torch.randn((nb, t * t), generator=g, device="cuda")
    bk = torch.arange(nb, dtype=torch.int32, device="cuda").reshape(nb, 1)
    aq, bq = tre.mx_quantize(plan, "u", a), tre.mx_quantize(plan, "v", b)
    ws = tre.alloc_workspace(plan.workspace_bytes(keys.shape[0], nb, keys.shape[0]))
    n_w = 401
    wk = torch.zeros((keys.shape[0], 1), dtype=torch.int32, device="cuda")
    wt = torch.zeros((keys.shape[0], t * t), dtype=torch.bfloat16 if t == 96 else torch.float32, device="cuda")
    if how == "async":
        counts = torch.zeros(4, dtype=torch.int64, device="cuda")
        tre.execute_async(plan, keys, aq, bk, bq, wk, wt, ws, counts)
        assert counts.tolist() == [keys.shape[0], n_w, 0, 0]
    else:
        tm = tre.Timing()
        assert tre.execute(plan, keys, aq, bk, bq, wk, wt, ws, timing=tm) == (n_w, keys.shape[0])
        assert tm.n_split_segments == 1 and tm.n_partials > 4
    ad = tre.mx_dequantize(plan, "u", aq).double().view(-1, t, t)
    bd = tre.mx_dequantize(plan, "v", bq).double().view(-1, t, t)[keys[:, 1].long()].contiguous()
    ref, mag = torch.bmm(ad, bd), torch.bmm(ad.abs(), bd.abs())
    ref = torch.cat([ref[:long].sum(0, keepdim=True), ref[long:]])
    mag = torch.cat([mag[:long].sum(0, keepdim=True), mag[long:]])
    got = wt[:n_w].double().view(n_w, t, t)
    n = torch.ones((n_w, 1, 1), device="cuda", dtype=torch.float64)
    n[0] = long
    tol = (n * (32 * mx.row_blocks(t) + 2)) * U32 * mag + (UB16 * ref.abs() if t == 96 else 0)
    assert bool(((got - ref).abs() <= tol).all())
    assert float((got - ref).norm() / ref.norm()) <= (UB16 if t == 96 else 1e-6)


def test_far_offsets():
    """Tiles past 2^31 elements and 2^32 bytes, in and out."""
    import torch

    import paper_2603_08957_amd as tre

    n, r, k = 40000, 256, 1024
    plan = tre.Plan("ik,jk->ij", "i", {"i": n * r, "j": 16, "k": k}, {"i": r}, "mxfp4")
    far = [0, 12345, 30839, 30840, n - 1]
    q = torch.zeros((n, plan.tile_bytes[0]), dtype=torch.uint8, device="cuda")  # 5.6 GB; zero codes, scale 2^-127
    x = torch.randn((len(far), r * k), device="cuda")
    q[far] = tre.mx_quantize(plan, "u", x)
    v = tre.mx_quantize(plan, "v", torch.randn((1, 16 * k), device="cuda"))
    keys = torch.arange(n, dtype=torch.int32, device="cuda").reshape(n, 1)
    w = tre.einsum(plan, keys, q, None, v).w_tiles
    xd = tre.mx_dequantize(plan, "u", q[far].contiguous()).double().view(-1, k)
    vd = tre.mx_dequantize(plan, "v", v).double().view(16, k)
    ref, mag = xd @ vd.T, xd.abs() @ vd.abs().T
    assert bool(((w[far].double().view(-1, 16) - ref).abs() <= (k + 2) * U32 * mag).all())
    w[far] = 0
    assert not bool(w.any())
    del w, keys
    m = 20500  # 5.4 G values of bf16: 10.7 GB
    tiles = torch.zeros((m, r * k), dtype=torch.bfloat16, device="cuda")
    tiles[m - 1] = x[0].to(torch.bfloat16)
    tre.mx_quantize(plan, "u", tiles, out=q[:m])
    assert torch.equal(q[m - 1], tre.mx_quantize(plan, "u", tiles[m - 1:].contiguous())[0])
    back = tre.mx_dequantize(plan, "u", q[:m], out=tiles)
    assert torch.equal(back[m - 1], tre.mx_dequantize(plan, "u", q[m - 1:m].contiguous(), dtype=torch.bfloat16)[0])
    assert not bool(back[:m - 1].any())


@pytest.mark.parametrize("t", [64, 24])  # fragments from LDS, and straight from memory
def test_keys_out_of_order_async(t):
    """Keys that are not sorted leave output keys whose pairs end before they
    begin: the call says so in its counts, and reads and writes nothing of
    theirs.  Keys in order then give their sums in the same buffers."""
    import torch

    import paper_2603_08957_amd as tre

    nb, k = 8, 128
    # (the join in several launches: the one-workgroup one leaves no such segments)
    plan = tre.Plan("ij,jk->ik", "ij", {"i": nb * t, "j": nb * k, "k": t}, {"i": t, "j": k}, "mxfp4", small_join=-1)
    g = torch.Generator(device="cuda").manual_seed(t)
    keys = torch.cartesian_prod(torch.arange(nb), torch.arange(nb)).to(torch.int32).cuda()
    bk = torch.arange(nb, dtype=torch.int32, device="cuda").reshape(nb, 1)
    u = tre.mx_quantize(plan, "u", torch.randn((nb * nb, t * k), generator=g, device="cuda"))
    v = tre.mx_quantize(plan, "v", torch.randn((nb, k * t), generator=g, device="cuda"))
    ws = tre.alloc_workspace(plan.workspace_bytes(nb * nb, nb, nb * nb))
    wk = torch.zeros((nb + 1, 1), dtype=torch.int32, device="cuda")
    wt = torch.full((nb + 1, t * t), -3.0, device="cuda")
    counts = torch.zeros(4, dtype=torch.int64, device="cuda")
    tre.execute_async(plan, keys.flip(0).contiguous(), u, bk, v, wk[:nb], wt[:nb], ws, counts)
    assert counts[2].item() == tre.tre.STATUS_CODE["TRE_E_UNSORTED"]
    assert torch.all(wt[nb] == -3.0) and wk[nb].item() == 0
    tre.execute_async(plan, keys, u, bk, v, wk[:nb], wt[:nb], ws, counts)
    assert counts.tolist() == [nb * nb, nb, 0, 0]
    ud = tre.mx_dequantize(plan, "u", u).double().view(nb, nb, t, k).transpose(1, 2).reshape(nb * t, nb * k)
    vd = tre.mx_dequantize(plan, "v", v).double().view(nb * k, t)
    ref, mag = ud @ vd, ud.abs() @ vd.abs()
    assert bool(((wt[:nb].double().view(nb * t, t) - ref).abs() <= (nb * k + 2) * U32 * mag).all())
    assert torch.all(wt[nb] == -3.0)


def test_einsum_refuses_tiles_off_the_current_gpu(monkeypatch):
    import torch

    import paper_2603_08957_amd as tre

    plan = tre.Plan("ik,jk->ij", "", {"i": 4, "j": 5, "k": 40}, {}, "mxfp4")
    u, v = tre.mx_quantize(plan, "u", torch.ones((1, 160), device="cuda")), tre.mx_quantize(plan, "v", torch.ones((1, 200), device="cuda"))
    assert torch.all(tre.einsum(plan, None, u, None, v).w_tiles == 40)
    for a, b in ((u.cpu(), v), (u, v.cpu())):
        with pytest.raises(tre.TreError) as e:
            tre.einsum(plan, None, a, None, b)
        assert e.value.status == "TRE_E_ARG"
    monkeypatch.setattr(torch.cuda, "current_device", lambda: u.device.index + 1)
    with pytest.raises(tre.TreError) as e:
        tre.einsum(plan, None, u, None, v)
    assert e.value.status == "TRE_E_ARG"


@pytest.mark.parametrize("small_join", [0, -1])
def test_timing_of_whole_keys(small_join):
    """A call that cuts no key counts none as cut, whatever its workspace held."""
    import torch

    import paper_2603_08957_amd as tre

    nb, t = 12, 64
    plan = tre.Plan("ij,jk->ik", "ij", {"i": nb * t, "j": nb * t, "k": t}, {"i": t, "j": t}, "mxfp4", small_join=small_join)
    keys = torch.cartesian_prod(torch.arange(nb), torch.arange(nb)).to(torch.int32).cuda()
    bk = torch.arange(nb, dtype=torch.int32, device="cuda").reshape(nb, 1)
    u = tre.mx_quantize(plan, "u", torch.randn((nb * nb, t * t), device="cuda"))
    v = tre.mx_quantize(plan, "v", torch.randn((nb, t * t), device="cuda"))
    ws = tre.alloc_workspace(plan.workspace_bytes(nb * nb, nb, nb * nb))
    wk, wt = torch.zeros((nb, 1), dtype=torch.int32, device="cuda"), torch.zeros((nb, t * t), device="cuda")
    for fill in (0, 0x33):
        ws.fill_(fill)
        tm = tre.Timing()
        assert tre.execute(plan, keys, u, bk, v, wk, wt, ws, timing=tm) == (nb, nb * nb)
        assert (tm.n_units, tm.n_split_segments, tm.n_partials) == (nb, 0, 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("einsum,op", FORMS)
@pytest.mark.parametrize("rows,k", [(16, 1), (33, 1), (1, 40), (2, 3), (3, 2), (2, 64), (300, 4)])
def test_quantize_thin_tiles(einsum, op, rows, k, dtype):
    """One value to a row, one or two rows, rows longer than their contracted index."""
    test_quantize_and_back(einsum, op, rows, k, dtype)


def test_count_of_tiles_on_the_device():
    """U's tuple count known on the device alone: tiles past it are neither read
    as operands nor written."""
    import torch

    import paper_2603_08957_amd as tre

    most, t, k, n = 40, 70, 200, 90
    plan = tre.Plan("vd,nd->nv", "v", {"v": most * t, "n": n, "d": k}, {"v": t}, "mxfp4")
    g = torch.Generator(device="cuda").manual_seed(2)
    u = tre.mx_quantize(plan, "u", torch.randn((most, t * k), generator=g, device="cuda"))
    v = tre.mx_quantize(plan, "v", torch.randn((1, n * k), generator=g, device="cuda"))
    uk = torch.arange(most, dtype=torch.int32, device="cuda").reshape(most, 1)
    want = tre.einsum(plan, uk, u, None, v).w_tiles
    ws = tre.alloc_workspace(plan.workspace_bytes(most, 1, most))
    counts = torch.zeros(4, dtype=torch.int64, device="cuda")
    for here in (0, 1, 17, most):
        wk = torch.full((most, 1), -9, dtype=torch.int32, device="cuda")
        wt = torch.full((most, n * t), -3.0, device="cuda")
        tre.execute_async(plan, uk, u, None, v, wk, wt, ws, counts, n_u=most,
                          n_u_dev=torch.tensor([here], dtype=torch.int64, device="cuda"))
        assert counts.tolist() == [here, here, 0, 0]
        assert torch.equal(wt[:here], want[:here]) and torch.equal(wk[:here], uk[:here])
        assert torch.all(wt[here:] == -3.0) and torch.all(wk[here:] == -9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("einsum", ["ik,jk->ij", "ki,jk->ij", "kil,jlk->ij"])
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 32), (5, 20), (7, 64), (3, 70), (9, 300), (16, 32)])
def test_padding_of_tiles_is_written(einsum, dtype, rows, k):
    """Every byte of a 4-bit tile follows from its values, the ones behind its last
    scale too (zero)."""
    import torch

    import paper_2603_08957_amd as tre

    sizes = {"i": rows, "k": k, "l": 2, "j": 3}
    plan = tre.Plan(einsum, "", {c: sizes[c] for c in einsum if c.isalpha()}, {}, "mxfp4")
    n, kk = 3, k * (2 if "l" in einsum else 1)
    x = torch.randn((n, plan.tile_elems[0]), device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    a, b = (torch.full((n, plan.tile_bytes[0]), fill, dtype=torch.uint8, device="cuda") for fill in (0xA5, 0x3C))
    tre.mx_quantize(plan, "u", x, out=a)
    tre.mx_quantize(plan, "u", x, out=b)
    assert torch.equal(a, b)
    assert not bool(a[:, 17 * rows * mx.row_blocks(kk):].any())
