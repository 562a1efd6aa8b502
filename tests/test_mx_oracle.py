"""4-bit tiles and table rows without a GPU: the oracle's own pins, the sizes
that the library reports, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest

from oracle import microscaled as mx


@pytest.fixture(scope="module")
def tre():
    import paper_2603_08957_amd as t

    t.lib()
    return t


def test_encode_pins():
    x = np.zeros((1, 32))
    x[0, :12] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, -0.0, 0.2500001, 7.9]
    c, s = mx.encode(x)
    # largest 7.9: e = 2 - 2 = 0
    assert s[0, 0] == 127
    assert c[0, 0, :12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 14, 8, 1, 7]
    for m, byte in ((1.0, 125), (2.0 ** -125, 0), (2.0 ** -126, 0), (0.0, 0), (2.0 ** 127, 252), (np.inf, 255), (np.nan, 255)):
        x[:] = 0
        x[0, 3] = m
        assert mx.encode(x)[1][0, 0] == byte, m
    v = np.random.default_rng(0).standard_normal((3, 70))
    codes, scales = mx.encode(v)
    once = mx.decode(codes, scales, 70)
    # in units of 2^e: steps of 0.5 up to 2, of 1 up to 4, of 2 up to 6, and less than 8 cut to 6
    unit = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=-1)[..., :70]
    assert np.all(np.abs(once - v) <= np.maximum(np.abs(v) / 4, unit / 4))
    # a block's largest stays within its power of two: quantised values are kept
    assert np.array_equal(mx.decode(*mx.encode(once), 70), once)


def test_sizes_agree(tre):
    rng = np.random.default_rng(1)
    for _ in range(60):
        n, v, d = (int(x) for x in rng.integers(1, 300, 3))
        p = tre.Plan("nd,vd->nv", "", {"n": n, "v": v, "d": d}, {}, "mxfp4")
        assert p.kernel_class == "mx"
        assert p.tile_bytes == [mx.tile_bytes(n, d), mx.tile_bytes(v, d), 4 * n * v]
    assert tre.Plan("nd,vd->nv", "", {"n": 3, "v": 5, "d": 7}, {}, "f32").tile_bytes == [84, 140, 60]
    assert tre.Plan("nd,vd->nv", "", {"n": 3, "v": 5, "d": 7}, {}, "mxfp4", w_bf16=True).tile_bytes[2] == 30
    assert tre.lib().tre_tile_bytes(None, 0) == -1
    p = tre.Plan("nd,vd->nv", "", {"n": 3, "v": 5, "d": 7}, {}, "mxfp4")
    assert tre.lib().tre_tile_bytes(p.handle, 3) == -1


def refused(tre, status, f, *a, **kw):
    with pytest.raises(tre.TreError) as e:
        f(*a, **kw)
    assert e.value.status == status, e.value


def test_plans_refused(tre):
    # summed inside one operand's tile alone
    refused(tre, "TRE_E_SHAPE", tre.Plan, "ijp,jk->ik", "", {"i": 4, "j": 4, "k": 4, "p": 2}, {}, "mxfp4")
    tre.Plan("ijp,jk->ik", "p", {"i": 4, "j": 4, "k": 4, "p": 2}, {"p": 1}, "mxfp4")
    # a row of one value takes a block of 17 bytes: 2^30 rows pass 2^31 bytes
    refused(tre, "TRE_E_SHAPE", tre.Plan, "i,ik->ik", "k", {"i": 1 << 30, "k": 2}, {"k": 1}, "mxfp4")
    # more than eight labels in a tile's rows: five of both operands, four of U
    lab = {c: 2 for c in "abcdefghix"}
    refused(tre, "TRE_E_SHAPE", tre.Plan, "abcdefghix,abcdex->abcdefghi", "", lab, {}, "mxfp4")


def test_entry_points_refuse(tre):
    """Refusals that come before any device work."""
    L = tre.lib()
    S = tre.tre.STATUS
    p = tre.Plan("nd,vd->nv", "", {"n": 3, "v": 5, "d": 7}, {}, "mxfp4")
    f = tre.Plan("nd,vd->nv", "", {"n": 3, "v": 5, "d": 7}, {}, "f32")
    a, odd = ctypes.c_void_p(4096), ctypes.c_void_p(4100)

    def q(plan, op, src, dt, n, dst):
        return S[L.tre_mx_quantize(plan, op, src, dt, n, dst, None)], S[L.tre_mx_dequantize(plan, op, dst, n, src, dt, None)]

    assert q(None, 0, a, 0, 1, a) == ("TRE_E_ARG",) * 2
    assert q(p.handle, 2, a, 0, 1, a) == ("TRE_E_ARG",) * 2
    assert q(p.handle, 0, None, 0, 1, a) == ("TRE_E_ARG",) * 2
    assert q(p.handle, 0, a, 0, -1, a) == ("TRE_E_ARG",) * 2
    assert q(p.handle, 0, odd, 0, 1, a) == ("TRE_E_ARG",) * 2
    assert q(p.handle, 0, a, 0, 1, odd) == ("TRE_E_ARG",) * 2
    assert q(p.handle, 0, a, 2, 1, a) == ("TRE_E_DTYPE",) * 2
    assert q(f.handle, 0, a, 0, 1, a) == ("TRE_E_DTYPE",) * 2
    assert q(p.handle, 0, a, 0, 1 << 31, a) == ("TRE_E_SHAPE",) * 2
    assert q(p.handle, 1, None, 1, 0, None) == ("TRE_OK",) * 2

    def look(table=a, tdt=0, rows=10, elems=8, tile=1, ids=a, ib=8, n=4, out=a, odt=0, st=None):
        return S[L.tre_lookup(table, tdt, rows, elems, tile, ids, ib, n, 1.0, out, odt, st, None)]

    assert look(tdt=3) == look(odt=2) == look(odt=-1) == "TRE_E_DTYPE"
    assert look(rows=0) == look(elems=0) == look(n=-1) == look(rows=1 << 31) == look(elems=(1 << 30) + 1) == "TRE_E_SHAPE"
    assert look(tdt=2, tile=3) == look(tdt=2, tile=0) == look(tdt=2, tile=20) == "TRE_E_SHAPE"
    assert look(tdt=2, rows=1 << 22, tile=1 << 22, elems=1 << 12) == "TRE_E_SHAPE"
    assert look(ib=2) == look(table=None) == look(ids=None) == look(out=None) == "TRE_E_ARG"
    assert look(table=odd) == look(out=odd) == look(ids=odd) == look(st=odd) == "TRE_E_ARG"
    assert look(n=0, table=None, ids=None, out=None) == "TRE_OK"

    need = L.tre_lookup_grad_workspace_bytes(4, 10, 8)

    def grad(g=a, gdt=0, ids=a, ib=8, n=4, out=a, odt=0, rows=10, elems=8, acc=0, st=None, ws=a, wb=need):
        return S[L.tre_lookup_grad(g, gdt, ids, ib, n, 1.0, out, odt, rows, elems, acc, st, ws, wb, None)]

    assert grad(gdt=2) == grad(odt=2) == "TRE_E_DTYPE"
    assert grad(rows=0) == grad(elems=0) == grad(n=-1) == "TRE_E_SHAPE"
    assert grad(ib=1) == grad(g=None) == grad(ids=None) == grad(out=None) == grad(ws=None) == "TRE_E_ARG"
    assert grad(g=odd) == grad(out=odd) == grad(ids=odd) == grad(ws=odd) == grad(st=odd) == "TRE_E_ARG"
    assert grad(wb=need - 1) == "TRE_E_WORKSPACE"
    assert L.tre_lookup_grad_workspace_bytes(4, 0, 8) == L.tre_lookup_grad_workspace_bytes(-1, 1, 8) == 0
    assert L.tre_lookup_grad_workspace_bytes(5000, 10, 8) > L.tre_lookup_grad_workspace_bytes(1, 10, 8) > 0


def test_binding_refuses(tre):
    """CPU tensors, wrong types and operands never reach the library."""
    import torch

    p = tre.Plan("nd,vd->nv", "v", {"n": 3, "v": 8, "d": 7}, {"v": 4}, "mxfp4")
    f = tre.Plan("nd,vd->nv", "", {"n": 3, "v": 5, "d": 7}, {}, "f32")
    x = torch.zeros(2, 28)
    refused(tre, "TRE_E_ARG", tre.mx_quantize, p, "v", x)
    refused(tre, "TRE_E_ARG", tre.mx_quantize, p, "w", x)
    refused(tre, "TRE_E_DTYPE", tre.mx_quantize, f, "v", x)
    refused(tre, "TRE_E_DTYPE", tre.mx_quantize, p, "v", x.half())
    refused(tre, "TRE_E_ARG", tre.mx_dequantize, p, "v", torch.zeros(2, p.tile_bytes[1], dtype=torch.uint8))
    ids = torch.zeros(3, dtype=torch.int64)
    refused(tre, "TRE_E_ARG", tre.lookup, x, ids)
    refused(tre, "TRE_E_DTYPE", tre.lookup, x.double(), ids)
    refused(tre, "TRE_E_SHAPE", tre.lookup, x[0], ids)
    refused(tre, "TRE_E_ARG", tre.lookup_grad, x, ids, 4)
    refused(tre, "TRE_E_DTYPE", tre.lookup_grad, x.half(), ids, 4)
    u = torch.zeros(2, 28)
    refused(tre, "TRE_E_SHAPE", tre.contract, p, tre.JoinResult(), u, u, None, u)
    refused(tre, "TRE_E_SHAPE", tre.einsum, p, None, u, None, u)


@pytest.mark.parametrize("where", ["cpu", "meta"])
def test_einsum_refuses_tiles_that_are_not_on_the_gpu(tre, where):
    """Tiles of the right shape and type, but not on a GPU: no entry point that
    takes them hands their addresses on."""
    import torch

    p = tre.Plan("nd,vd->nv", "", {"n": 3, "v": 5, "d": 7}, {}, "mxfp4")
    u, v = (torch.zeros((1, b), dtype=torch.uint8, device=where) for b in p.tile_bytes[:2])
    w, counts = torch.zeros((1, 15)), torch.zeros(4, dtype=torch.int64)
    ws = torch.zeros(p.workspace_bytes(1, 1, 1), dtype=torch.uint8)
    refused(tre, "TRE_E_ARG", tre.einsum, p, None, u, None, v)
    refused(tre, "TRE_E_ARG", tre.execute, p, None, u, None, v, None, w, ws)
    refused(tre, "TRE_E_ARG", tre.execute_async, p, None, u, None, v, None, w, ws, counts)
    refused(tre, "TRE_E_ARG", tre.execute_noalloc, p, None, u, None, v, None, w)
    refused(tre, "TRE_E_ARG", tre.contract, p, tre.JoinResult(), u, v, None, w)


def test_streams_of_another_gpu_refused(tre):
    import torch

    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 0

    refused(tre, "TRE_E_ARG", tre.tre._Here, torch.device("cuda", 0), Stream(), "tre.lookup")


@pytest.mark.parametrize("einsum,upper,tiles,operand", [
    ("vd,nd->nv", "vd", {"v": 4, "d": 32}, "u"),      # rows in pieces, a tile of each
    ("vd,nd->nv", "d", {"d": 32}, "u"),
    ("nd,dv->nv", "dv", {"v": 4, "d": 32}, "v"),
    ("vpd,nd->nvp", "v", {"v": 4}, "u"),              # two labels for the token
    ("vpd,nd->nvp", "vp", {"v": 4, "p": 1}, "u"),
    ("vpd,nd->nv", "vp", {"v": 4, "p": 1}, "u"),      # a promoted label that neither side has
    ("d,nd->n", "", {}, "u"),                         # none
])
def test_lookup_refuses_plans_of_other_tables(tre, einsum, upper, tiles, operand):
    """A table's key is the token alone: what else a plan promotes, or keeps,
    would give pieces of rows, or rows in another order."""
    import torch

    p = tre.Plan(einsum, upper, {"v": 8, "d": 64, "n": 3, "p": 1 if "nvp" not in einsum else 2}, tiles, "mxfp4")
    o = "uv".index(operand)
    t = torch.zeros((2, p.tile_bytes[o]), dtype=torch.uint8)
    ids = torch.zeros(3, dtype=torch.int64)
    refused(tre, "TRE_E_SHAPE", tre.lookup, t, ids, plan=p, operand=operand)


@pytest.mark.parametrize("einsum,upper,tiles,operand", [
    ("vd,nd->nv", "v", {"v": 4}, "u"), ("vd,nd->nv", "", {}, "u"), ("nd,dv->nv", "v", {"v": 2}, "v"),
    ("vd,nd->nv", "vn", {"v": 4, "n": 1}, "u"), ("vdc,ncd->nv", "v", {"v": 4}, "u"),
])
def test_lookup_takes_plans_of_tables(tre, einsum, upper, tiles, operand):
    """Plans that a lookup takes get as far as the tensors' place."""
    import torch

    p = tre.Plan(einsum, upper, {"v": 8, "d": 64, "n": 3, "c": 2}, tiles, "mxfp4")
    t = torch.zeros((2, p.tile_bytes["uv".index(operand)]), dtype=torch.uint8)
    refused(tre, "TRE_E_ARG", tre.lookup, t, torch.zeros(3, dtype=torch.int64), plan=p, operand=operand)
