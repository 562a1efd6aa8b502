"""Rows of a table by token and the table's gradient on the GPU, against float64.

A looked-up value is one fp32 product (2^-24 of it) rounded once more to the
output's type (half a step: 2^-8 for bf16).  A gradient is a sum of c rows (c
additions: c 2^-24 of the sum of magnitudes), times the scale, rounded once.
"""
import numpy as np
import pytest

from oracle import microscaled as mx

pytestmark = pytest.mark.gpu

U32, UB16 = 2.0 ** -24, 2.0 ** -8
HALF = {"f32": U32, "bf16": UB16}


def types():
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16}


def tokens(rng, n, vocab, kind):
    if kind == "one":
        return np.full(n, vocab // 2, np.int64)
    if kind == "each":
        return rng.permutation(max(n, vocab))[:n] % vocab
    if kind == "none":
        return np.full(n, -1, np.int64)
    ids = np.floor(np.exp(rng.random(n) * np.log(vocab))).astype(np.int64) - 1
    if kind == "padded":
        ids[rng.random(n) < 0.3] = -5
    return np.clip(ids, -5, vocab - 1)


@pytest.mark.parametrize("tdt", ["f32", "bf16"])
@pytest.mark.parametrize("odt", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (3, 7, 5), (8, 100, 767), (33, 50, 64), (1000, 333, 129), (5, 9, 512),
                                       (64, 64, 520), (7, 40, 4097), (257, 31, 8)])
def test_lookup(n, vocab, d, tdt, odt):
    import torch

    import paper_2603_08957_amd as tre

    T = types()
    rng = np.random.default_rng(n + d)
    table = torch.from_numpy(rng.standard_normal((vocab, d)).astype(np.float32)).to(T[tdt]).cuda()
    ids = tokens(rng, n, vocab, "padded")
    ref = np.where(ids[:, None] >= 0, table.double().cpu().numpy()[np.maximum(ids, 0)] * np.float64(np.float32(1.7)), 0)
    for it in (torch.int32, torch.int64):
        dev = torch.from_numpy(ids).to(it).cuda()
        buf = torch.full((n + 1, d), -7.0, dtype=T[odt], device="cuda")
        status = torch.zeros(1, dtype=torch.int64, device="cuda")
        got = tre.lookup(table, dev, scale=1.7, out=buf[:n], status=status)
        assert got.data_ptr() == buf.data_ptr() and status.item() == 0
        v = buf.double().cpu().numpy()
        assert np.all(np.abs(v[:n] - ref) <= (U32 + HALF[odt] * (1 + U32)) * np.abs(ref))
        assert np.all(v[n] == -7.0)
    # scale one keeps bits
    if tdt == odt:
        got = tre.lookup(table, dev).cpu()
        want = torch.where(dev.cpu()[:, None] >= 0, table.cpu()[dev.cpu().clamp_min(0).long()], torch.zeros((), dtype=T[odt]))
        assert torch.equal(got, want)


@pytest.mark.parametrize("k", [1, 30, 33, 64, 100, 767, 1024])
@pytest.mark.parametrize("tile", [1, 5, 128])
def test_lookup_mx(k, tile):
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(k)
    n_tiles = 4
    vocab = n_tiles * tile
    table = rng.standard_normal((n_tiles, tile * k)) * np.exp2(rng.integers(-9, 9, (n_tiles, 1)).astype(float))
    table[0, 0] = np.nan
    table = table.astype(np.float32)
    ids = tokens(rng, 50, vocab, "padded").reshape(5, 10)
    ids[0, 0] = 0
    for e, op, lab in (("vd,nd->nv", "u", "vd"), ("nd,dv->nv", "v", "dv")):
        plan = tre.Plan(e, "v", {"v": vocab, "n": 3, "d": k}, {"v": tile}, "mxfp4")
        sizes = {"v": tile, "n": 3, "d": k}
        src = table.reshape(n_tiles, tile, k)
        t = src if lab == "vd" else src.transpose(0, 2, 1)
        t = np.ascontiguousarray(t).reshape(n_tiles, -1)
        q = tre.mx_quantize(plan, op, torch.from_numpy(t).cuda())
        vals = mx.decode(*mx.encode(src.astype(np.float64)), k).reshape(vocab, k)
        ref = np.where(ids[..., None] >= 0, vals[np.maximum(ids, 0)] * 2.0, 0)
        for odt in (torch.float32, torch.bfloat16):
            got = tre.lookup(q, torch.from_numpy(ids).cuda(), scale=2.0, dtype=odt, plan=plan, operand=op)
            assert got.shape == (5, 10, k)
            assert np.array_equal(got.double().cpu().numpy(), ref, equal_nan=True)


def test_ids_out_of_range():
    """Tokens past the table read and write nothing but a zero row and the status."""
    import torch

    import paper_2603_08957_amd as tre

    ids = torch.tensor([0, 5, 4, 2 ** 31 - 1, -2 ** 31, 3, 2 ** 40, -1], device="cuda")
    table = torch.randn((5, 70), device="cuda")
    ok = [0, None, 4, None, None, 3, None, None]
    for it in (torch.int64, torch.int32):
        x = ids.to(it) if it == torch.int64 else ids.clamp(-2 ** 31, 2 ** 31 - 1).to(it)
        status = torch.zeros(1, dtype=torch.int64, device="cuda")
        got = tre.lookup(table, x, status=status)
        assert status.item() == tre.tre.STATUS_CODE["TRE_E_KEYRANGE"]
        for i, j in enumerate(ok):
            assert torch.equal(got[i], table[j] if j is not None else torch.zeros_like(got[i]))
        status.zero_()
        g = torch.randn((8, 70), device="cuda")
        dt = tre.lookup_grad(g, x, 5, status=status)
        assert status.item() == tre.tre.STATUS_CODE["TRE_E_KEYRANGE"]
        want = torch.zeros_like(table)
        want[0], want[4], want[3] = g[0], g[2], g[5]
        assert torch.equal(dt, want)
        # without a status the call is the same
        assert torch.equal(tre.lookup(table, x), got) and torch.equal(tre.lookup_grad(g, x, 5), want)


GRADS = [  # tokens, rows, row, kind: at and around the chunks of 8 and 32, their groups of 16, the sorts' tiles and limits
    (1, 1, 1, "one"), (1, 50, 9, "each"), (31, 5, 8, "zipf"), (32, 5, 33, "one"), (33, 40, 64, "one"), (64, 70, 7, "each"),
    (65, 3, 513, "padded"), (200, 10, 767, "none"), (500, 2000, 20, "zipf"), (1000, 100, 130, "padded"),
    (4096, 1000, 16, "zipf"), (4097, 300, 24, "one"), (9000, 70000, 8, "padded"), (20000, 50, 8, "zipf"),
    (8192, 300, 6, "padded"), (8193, 9000, 6, "each"), (16384, 40, 10, "zipf"), (16385, 40, 10, "one"),
    (300000, 9, 3, "zipf"), (140000, 3, 2, "one"),
]


@pytest.mark.parametrize("scale", [-2.0, float("inf"), float("nan")])
@pytest.mark.parametrize("d", [24, 1200])
def test_rows_of_no_token_under_any_scale(d, scale):
    """Such rows are +0, whatever the others become."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(d)
    table = torch.from_numpy(1 + rng.random((9, d)).astype(np.float32)).cuda()
    ids = torch.tensor([3, -1, 8, 0, -7, 2, -1], device="cuda")
    plan = tre.Plan("vd,td->vt", "v", {"v": 9, "d": d, "t": 16}, {"v": 3}, dtype="mxfp4")
    q = tre.mx_quantize(plan, "u", table.view(3, 3 * d))
    for got, rows in ((tre.lookup(table, ids, scale=scale), table),
                      (tre.lookup(table.bfloat16(), ids, scale=scale, dtype=torch.float32), table.bfloat16().float()),
                      (tre.lookup(q, ids, scale=scale, plan=plan), tre.mx_dequantize(plan, "u", q).view(9, d))):
        v, none = got.cpu().numpy(), (ids < 0).cpu().numpy()
        assert np.all(v[none].view(np.uint32) == 0)
        np.testing.assert_array_equal(v[~none], (rows[ids[~torch.from_numpy(none).cuda()]] * scale).cpu().numpy())
    grad = tre.lookup_grad(tre.lookup(table, ids), ids, 9, scale=scale).cpu().numpy()
    assert np.all(grad[[1, 4, 5, 6, 7]].view(np.uint32) == 0)


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
@pytest.mark.parametrize("odt", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,kind", GRADS)
def test_lookup_grad(n, vocab, d, kind, gdt, odt):
    import torch

    import paper_2603_08957_amd as tre

    T = types()
    rng = np.random.default_rng(n * 7 + d)
    ids = tokens(rng, n, vocab, kind)
    grad = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(T[gdt]).cuda()
    ref, mag = mx.lookup_grad(grad.double().cpu().numpy(), ids, vocab, float(np.float32(0.3)))
    c = np.bincount(ids[ids >= 0], minlength=vocab)[:, None]
    dev = torch.from_numpy(ids).cuda()
    buf = torch.full((vocab + 1, d), -7.0, dtype=T[odt], device="cuda")
    ws = tre.alloc_workspace(tre.lookup_grad_workspace_bytes(n, vocab, d))
    tre.lookup_grad(grad, dev, vocab, scale=0.3, out=buf[:vocab], ws=ws)
    v = buf.double().cpu().numpy()
    assert np.all(v[vocab] == -7.0)
    # (c additions, the product with the scale, the rounding)
    tol = ((c + 1) * U32 * mag) * (1 + HALF[odt]) + HALF[odt] * np.abs(ref)
    assert np.all(np.abs(v[:vocab] - ref) <= tol)
    assert np.all(v[:vocab][c[:, 0] == 0] == 0)
    # again, with a workspace that held other data and other ids' type: the same bits
    ws.fill_(0xC3)
    again = tre.lookup_grad(grad, dev.int(), vocab, scale=0.3, dtype=T[odt], ws=ws)
    assert torch.equal(again, buf[:vocab])
    # added to what is there; rows that no token has keep their bits
    base = torch.from_numpy(rng.standard_normal((vocab, d)).astype(np.float32)).to(T[odt]).cuda()
    out = base.clone()
    tre.lookup_grad(grad, dev, vocab, scale=0.3, out=out, accumulate=True)
    b = base.double().cpu().numpy()
    tol = ((c + 2) * U32 * (mag + np.abs(b))) * (1 + HALF[odt]) + HALF[odt] * np.abs(ref + b)
    assert np.all(np.abs(out.double().cpu().numpy() - (ref + b)) <= tol)
    assert torch.equal(out[torch.from_numpy(c[:, 0] == 0).cuda()], base[torch.from_numpy(c[:, 0] == 0).cuda()])


@pytest.mark.parametrize("odt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,d", [(1, 1), (300, 1), (130, 37), (1000, 64), (70, 8193), (9, 20000), (5000, 3), (200, 1001)])
def test_zero_rows(vocab, d, odt):
    """Every row without a token is zero, none behind the last is touched."""
    import torch

    import paper_2603_08957_amd as tre

    T = types()
    rng = np.random.default_rng(vocab + d)
    for n in (0, 1, vocab // 2, vocab):
        ids = torch.from_numpy(rng.integers(0, vocab, n)).cuda()
        grad = torch.ones((n, d), device="cuda")
        buf = torch.full((vocab + 1, d), float("nan"), dtype=T[odt], device="cuda")
        buf[vocab] = -7.0
        tre.lookup_grad(grad, ids, vocab, out=buf[:vocab])
        want = torch.bincount(ids.cpu(), minlength=vocab).float()[:, None].expand(vocab, d)
        assert torch.equal(buf[:vocab].float().cpu(), want)  # counts below 256: exact in bf16
        assert torch.all(buf[vocab] == -7.0)


def test_lookup_grad_by_differences():
    """The gradient of sum(g * lookup(E)) by differences: with small whole
    numbers and a scale of 2 every step is exact."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(5)
    ids = torch.from_numpy(tokens(rng, 40, 6, "padded")).cuda()
    e = torch.from_numpy(rng.integers(-4, 5, (6, 3)).astype(np.float32)).cuda()
    g = torch.from_numpy(rng.integers(-4, 5, (40, 3)).astype(np.float32)).cuda()
    loss = lambda t: float((tre.lookup(t, ids, scale=2.0) * g).sum())  # noqa: E731
    grad = tre.lookup_grad(g, ids, 6, scale=2.0)
    at = loss(e)
    for i in range(6):
        for j in range(3):
            e[i, j] += 1
            assert loss(e) - at == grad[i, j].item()
            e[i, j] -= 1


def test_empty():
    import torch

    import paper_2603_08957_amd as tre

    table = torch.randn((5, 12), device="cuda")
    none = torch.zeros((0,), dtype=torch.int64, device="cuda")
    assert tre.lookup(table, none).shape == (0, 12)
    assert tre.lookup(table, none.view(0, 3)).shape == (0, 3, 12)
    assert torch.equal(tre.lookup_grad(table[:0], none, 5), torch.zeros_like(table))
    assert torch.equal(tre.lookup_grad(table[:0], none, 5, out=table.clone(), accumulate=True), table)
    assert tre.lookup(table, torch.tensor(3, device="cuda")).equal(table[3])


def test_refused_on_the_gpu():
    import torch

    import paper_2603_08957_amd as tre

    table = torch.randn((6, 16), device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")

    def refused(status, f, *a, **kw):
        with pytest.raises(tre.TreError) as e:
            f(*a, **kw)
        assert e.value.status == status

    refused("TRE_E_SHAPE", tre.lookup, table.T, ids)
    refused("TRE_E_SHAPE", tre.lookup, table, ids[::2])
    refused("TRE_E_DTYPE", tre.lookup, table, ids.short())
    refused("TRE_E_ARG", tre.lookup, table, ids.cpu())
    refused("TRE_E_SHAPE", tre.lookup, table, ids, out=torch.empty((4, 15), device="cuda"))
    refused("TRE_E_DTYPE", tre.lookup, table, ids, dtype=torch.float16)
    refused("TRE_E_ARG", tre.lookup, table.view(-1)[1:81].view(5, 16), ids)  # begins off 16 bytes
    g = torch.randn((4, 16), device="cuda")
    refused("TRE_E_SHAPE", tre.lookup_grad, g, ids[:3], 6)
    refused("TRE_E_SHAPE", tre.lookup_grad, g, ids, 0)
    refused("TRE_E_ARG", tre.lookup_grad, g, ids, 6, accumulate=True)
    refused("TRE_E_WORKSPACE", tre.lookup_grad, g, ids, 6, ws=tre.alloc_workspace(256))
    plan = tre.Plan("vd,nd->nv", "v", {"v": 6, "n": 2, "d": 16}, {"v": 3}, "mxfp4")
    refused("TRE_E_DTYPE", tre.lookup, table.view(2, 48), ids, plan=plan)
    refused("TRE_E_SHAPE", tre.lookup, tre.mx_quantize(plan, "u", table.view(2, 48))[:, :-1], ids, plan=plan)
    refused("TRE_E_SHAPE", tre.mx_quantize, plan, "u", table)
    refused("TRE_E_SHAPE", tre.mx_quantize, plan, "v", g[:2].T.contiguous())


@pytest.mark.parametrize("n", [60, 5000, 20000])  # one chunk's groups, tokens ranked, tokens sorted by digits
def test_streams_and_graphs(n):
    """On another stream, and replayed from a graph between eager calls that
    share its workspace."""
    import torch

    import paper_2603_08957_amd as tre

    vocab, d = 700, 40
    ids = torch.randint(-1, vocab, (n,), device="cuda")
    g = torch.randn((n, d), device="cuda")
    table = torch.randn((vocab, d), device="cuda")
    ws = tre.alloc_workspace(tre.lookup_grad_workspace_bytes(n, vocab, d))
    want = tre.lookup_grad(g, ids, vocab, ws=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tre.lookup_grad(g, ids, vocab, stream=side)  # buffers made here, used there
    rows = tre.lookup(table, ids, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(rows, tre.lookup(table, ids))
    out, look = torch.zeros_like(table), torch.zeros_like(g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tre.lookup(table, ids, out=look)
        tre.lookup_grad(look, ids, vocab, out=out, ws=ws)
    for i in range(4):
        ids.copy_(torch.randint(-1, vocab, (n,), device="cuda"))
        table.normal_()
        eager = tre.lookup_grad(tre.lookup(table, ids), ids, vocab, ws=ws)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i


def test_far_offsets():
    """Rows past 2^31 elements and 2^32 bytes into table and output."""
    import torch

    import paper_2603_08957_amd as tre

    d, vocab = 1 << 16, 40000
    table = torch.zeros((vocab, d), dtype=torch.bfloat16, device="cuda")
    for r in (0, 32767, 32768, 39999):
        table[r] = r % 251 + 1
    ids = torch.tensor([39999, 0, 32768, 32767, 39999], device="cuda")
    got = tre.lookup(table, ids)
    assert [int(x) for x in got[:, -1].tolist()] == [i % 251 + 1 for i in ids.tolist()]
    grad = tre.lookup_grad(got, ids, vocab, out=table)
    sums = grad.float().sum(1) / d
    for r, c in ((0, 1), (32767, 1), (32768, 1), (39999, 2)):
        assert float(sums[r]) == c * (r % 251 + 1), r
    assert int((sums != 0).sum()) == 4


def test_training_step_of_a_tied_table():
    """Rows looked up in a 4-bit table, scores against the same tiles, and both
    gradients of the table: what a step calls, in one run, against float64 on
    the values that the quantised tiles stand for."""
    import torch

    import paper_2603_08957_amd as tre

    n, vocab, d, t = 96, 256, 80, 64
    ext, til = {"n": n, "v": vocab, "d": d}, {"v": t}
    nt = vocab // t
    scores = tre.Plan("vd,nd->nv", "v", ext, til, "mxfp4")       # W keyed by v: [n][t]
    back = tre.Plan("vn,vd->nd", "v", ext, til, "mxfp4")         # the rows' gradient, the table along v
    weight = tre.Plan("vn,nd->vd", "v", ext, til, "mxfp4")       # the table's, both along n
    g = torch.Generator(device="cuda").manual_seed(3)
    table = torch.randn((vocab, d), generator=g, device="cuda").to(torch.bfloat16)
    ids = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    ids[::7] = -1
    dy = torch.randn((n, vocab), generator=g, device="cuda")
    vk = torch.arange(nt, dtype=torch.int32, device="cuda").reshape(nt, 1)
    tiles = table.view(nt, -1)
    q = tre.mx_quantize(scores, "u", tiles)
    x = tre.lookup(q, ids, scale=3.0, plan=scores)
    y = tre.einsum(scores, vk, q, None, tre.mx_quantize(scores, "v", x.view(1, -1)))
    dyt = dy.T.contiguous().view(nt, -1)                          # keyed by v: [t][n]
    dx = tre.einsum(back, vk, tre.mx_quantize(back, "u", dyt), vk, tre.mx_quantize(back, "v", tiles))
    dw = tre.einsum(weight, vk, tre.mx_quantize(weight, "u", dyt), None, tre.mx_quantize(weight, "v", x.view(1, -1)))
    de = dw.w_tiles.view(vocab, d)
    tre.lookup_grad(dx.w_tiles.view(n, d), ids, vocab, scale=3.0, out=de, accumulate=True)

    tab, ids_h, dyh = table.double().cpu().numpy(), ids.cpu().numpy(), dy.double().cpu().numpy()
    along = lambda m: mx.decode(*mx.encode(m), m.shape[-1])  # noqa: E731
    tq = along(tab)
    xr = np.where(ids_h[:, None] >= 0, tq[np.maximum(ids_h, 0)] * 3.0, 0)
    xr = xr.astype(np.float32).astype(np.float64)
    assert np.array_equal(x.double().cpu().numpy(), xr)
    xq = along(xr)
    yr = xq @ tq.T

    def near(got, ref, mag, terms):
        assert np.all(np.abs(got - ref) <= terms * U32 * mag)

    near(y.w_tiles.view(nt, n, t).transpose(0, 1).reshape(n, vocab).double().cpu().numpy(), yr, np.abs(xq) @ np.abs(tq).T, 130)
    # contracted along v in tiles of 64: blocks of 32 begin anew in each
    gv = along(dyh.reshape(n, nt, t)).reshape(n, vocab)
    tv = along(tab.reshape(nt, t, d).transpose(0, 2, 1)).transpose(0, 2, 1).reshape(vocab, d)
    dxr, dxm = gv @ tv, np.abs(gv) @ np.abs(tv)
    near(dx.w_tiles.view(n, d).double().cpu().numpy(), dxr, dxm, vocab + 4)
    gn, xn = along(dyh.T), along(xr.T).T
    e1, m1 = mx.lookup_grad(dxr, ids_h, vocab, 3.0)
    _, m2 = mx.lookup_grad(dxm, ids_h, vocab, 3.0)
    dwr, dwm = gn @ xn, np.abs(gn) @ np.abs(xn)
    near(de.double().cpu().numpy(), dwr + e1, dwm + m1 + m2, vocab + 2 * n + 140)


@pytest.mark.parametrize("d", [1, 2, 3, 63, 127, 129, 250])
@pytest.mark.parametrize("n", [8 * 40, 8 * 64, 32 * 600])
def test_runs_that_end_in_every_chunk(n, d):
    """Each chunk of tokens ends one run and begins the next, so that every lane
    of the wavefront that joins partial sums holds the key of a row, those past
    the row's end too.  Whole numbers: every sum is exact."""
    import torch

    import paper_2603_08957_amd as tre

    chunk = 8 if n <= 16384 else 32
    ids = (torch.arange(n) + chunk // 2) // chunk  # runs of a chunk's length, half a chunk off
    vocab = int(ids[-1]) + 1
    g = torch.randint(-8, 9, (n, d), generator=torch.Generator().manual_seed(n + d)).float()
    want = torch.zeros((vocab, d)).index_add_(0, ids, g) * 2
    assert torch.equal(tre.lookup_grad(g.cuda(), ids.cuda(), vocab, scale=2.0).cpu(), want)
    out = torch.ones((vocab, d), device="cuda")
    tre.lookup_grad(g.cuda(), ids.cuda(), vocab, scale=2.0, out=out, accumulate=True)
    assert torch.equal(out.cpu(), want + 1)


def test_buffers_of_a_callers_stream():
    """What a call allocates for a caller's stream is not memory that the
    current stream still works on: blocks given back there, with work on them
    queued, that have just the sizes of the call's buffers."""
    import torch

    import paper_2603_08957_amd as tre

    n, vocab, d = 2048, 4096, 1024
    table = torch.randn((vocab, d), device="cuda")
    ids = torch.randint(0, vocab, (n,), device="cuda")
    g = torch.randn((n, d), device="cuda")
    plan = tre.Plan("vd,nd->nv", "v", {"v": vocab, "n": 4, "d": d}, {"v": 64}, "mxfp4")
    tiles = table.view(vocab // 64, -1)
    q = tre.mx_quantize(plan, "u", tiles)
    side = torch.cuda.Stream()
    calls = {
        "lookup": lambda **kw: tre.lookup(table, ids, scale=2.0, **kw),
        "lookup_grad": lambda **kw: tre.lookup_grad(g, ids, vocab, **kw),
        "mx_quantize": lambda **kw: tre.mx_quantize(plan, "u", tiles, **kw),
        "mx_dequantize": lambda **kw: tre.mx_dequantize(plan, "u", q, **kw),
    }
    busy = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for name, call in calls.items():
        want = call()
        ws_bytes = tre.lookup_grad_workspace_bytes(n, vocab, d)
        torch.cuda.synchronize()
        # the current stream's queue: long work, then writes to blocks that are given back at once
        blocks = [torch.empty_like(want), torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")]
        for _ in range(100):
            busy.fill_(1)
        for b in blocks:
            b.view(torch.uint8).fill_(0x55)
        del blocks, b
        got = call(stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want), name
        # and a result given back is not handed out while the current stream reads it
        for _ in range(100):
            busy.fill_(1)
        copy = got.clone()
        del got
        with torch.cuda.stream(side):
            torch.empty_like(want).view(torch.uint8).fill_(0x55)
        torch.cuda.synchronize()
        assert torch.equal(copy, want), name


@pytest.mark.parametrize("odt", ["f32", "bf16"])
@pytest.mark.parametrize("gdt", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,kind", [
    (16384, 40, 10, "one"), (16385, 40, 10, "one"), (16385, 40, 130, "zipf"), (33000, 5, 3, "zipf"), (140000, 3, 2, "one"),
    (140000, 3, 257, "zipf"), (300000, 9, 3, "zipf"), (300000, 9, 5, "padded"), (600000, 4, 1, "one"),
])
def test_long_runs_exactly(n, vocab, d, kind, gdt, odt):
    """Runs of one token over many chunks and their groups, of whole numbers whose
    sums fp32 holds exactly in any order (up to 4 n < 2^24): no row of a run may
    be missing or counted twice.  A bf16 result is the sum rounded once."""
    import torch

    import paper_2603_08957_amd as tre

    assert 4 * n < 1 << 24
    T = types()
    rng = np.random.default_rng(n + d)
    ids = tokens(rng, n, vocab, kind)
    whole = rng.integers(-2, 3, (n, d))
    total = np.zeros((vocab, d), np.int64)
    np.add.at(total, ids[ids >= 0], whole[ids >= 0])
    grad = torch.from_numpy(whole.astype(np.float32)).to(T[gdt]).cuda()
    want = torch.from_numpy(2.0 * total).float().to(T[odt])
    dev = torch.from_numpy(ids).cuda()
    got = tre.lookup_grad(grad, dev, vocab, scale=2.0, dtype=T[odt])
    assert torch.equal(got.cpu(), want)
    # added to whole numbers that are there
    base = torch.from_numpy(rng.integers(-2, 3, (vocab, d)).astype(np.float32)).to(T[odt])
    out = base.cuda()
    tre.lookup_grad(grad, dev, vocab, scale=2.0, out=out, accumulate=True)
    there = torch.from_numpy((ids[ids >= 0][None, :] == np.arange(vocab)[:, None]).any(1))[:, None]
    assert torch.equal(out.cpu(), torch.where(there, (base.double() + torch.from_numpy(2.0 * total)).float().to(T[odt]), base))
    # all ones: the number of a row's tokens
    ones = torch.ones((n, d), dtype=T[gdt], device="cuda")
    count = torch.bincount(torch.from_numpy(ids[ids >= 0]), minlength=vocab).float()[:, None].expand(vocab, d)
    assert torch.equal(tre.lookup_grad(ones, dev, vocab).cpu(), count)


@pytest.mark.parametrize("n", [8192, 9000, 140000])  # ranked; sorted in small tiles and in large ones
def test_many_ids_out_of_range(n):
    import torch

    import paper_2603_08957_amd as tre

    vocab, d = 300, 5
    g = torch.Generator().manual_seed(n)
    ids = torch.randint(-2, vocab, (n,), generator=g)
    ids[::97] = vocab
    ids[5::89] = 2 ** 40 + 3  # its low half is a row's number
    ids[7::83] = -2 ** 40 + 3
    grad = torch.randint(-2, 3, (n, d), generator=g).float()
    ok = (ids >= 0) & (ids < vocab)
    want = torch.zeros((vocab, d)).index_add_(0, ids[ok], grad[ok])
    status = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert torch.equal(tre.lookup_grad(grad.cuda(), ids.cuda(), vocab, status=status).cpu(), want)
    assert status.item() == tre.tre.STATUS_CODE["TRE_E_KEYRANGE"]
    table = torch.randn((vocab, d), generator=g)
    status.zero_()
    rows = tre.lookup(table.cuda(), ids.cuda(), status=status).cpu()
    assert status.item() == tre.tre.STATUS_CODE["TRE_E_KEYRANGE"]
    assert torch.equal(rows, torch.where(ok[:, None], table[ids.clamp(0, vocab - 1)], torch.zeros(())))


@pytest.mark.parametrize("n", [7, 60, 5000, 20000])
@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_values_of_no_token_do_not_count(n, gdt):
    """NaN and infinities in the gradient's rows of no token, and in table rows
    that no token names, reach nothing."""
    import torch

    import paper_2603_08957_amd as tre

    vocab, d = 50, 37
    g = torch.Generator().manual_seed(n)
    ids = torch.randint(0, vocab - 1, (n,), generator=g)
    ids[::3] = -1
    ids[1::7] = vocab + 4
    grad = torch.randint(-2, 3, (n, d), generator=g).float()
    ok = (ids >= 0) & (ids < vocab)
    want = torch.zeros((vocab, d)).index_add_(0, ids[ok], grad[ok])
    grad[~ok] = float("nan")
    grad[0] = float("inf")
    assert torch.equal(tre.lookup_grad(grad.to(types()[gdt]).cuda(), ids.cuda(), vocab).cpu(), want)
    table = torch.ones((vocab, d)) * 2
    table[vocab - 1] = float("nan")
    table = table.to(types()[gdt]).cuda()
    rows = tre.lookup(table, ids.cuda(), dtype=torch.float32).cpu()
    assert torch.equal(rows, torch.where(ok, 2.0, 0.0)[:, None].expand(n, d))


def test_inputs_given_back_before_a_callers_stream_is_done():
    """Inputs of a call queued on a busy stream, given back at once: their memory
    is not handed out before the call has read them."""
    import torch

    import paper_2603_08957_amd as tre

    n, vocab, d = 2048, 4096, 1024
    table = torch.randn((vocab, d), device="cuda")
    ids = torch.randint(0, vocab, (n,), device="cuda")
    g = torch.randn((n, d), device="cuda")
    plan = tre.Plan("vd,nd->nv", "v", {"v": vocab, "n": 4, "d": d}, {"v": 64}, "mxfp4")
    tiles = table.view(vocab // 64, -1)
    q = tre.mx_quantize(plan, "u", tiles)
    side = torch.cuda.Stream()
    busy = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for name, call, args in (("lookup", lambda t, i, **kw: tre.lookup(t, i, scale=2.0, **kw), (table, ids)),
                             ("lookup_grad", lambda t, i, **kw: tre.lookup_grad(t, i, vocab, **kw), (g, ids)),
                             ("mx_quantize", lambda t, **kw: tre.mx_quantize(plan, "u", t, **kw), (tiles,)),
                             ("mx_dequantize", lambda t, **kw: tre.mx_dequantize(plan, "u", t, **kw), (q,))):
        want = call(*args)
        copies = [a.clone() for a in args]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(100):
                busy.fill_(1)
        got = call(*copies, stream=side)
        del copies
        others = [torch.zeros_like(a) for a in args for _ in range(2)]
        torch.cuda.synchronize()
        assert torch.equal(got, want) and len(others) == 2 * len(args), name
