"""Calls that take more than 2^32 threads, which one dimension of a launch does
not hold.  Those of the 4-bit tile and row entry points give, past that point,
the results of the same rows in a small call; contractions of the other types,
which have one dimension, say that they cannot."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _memory():
    import torch

    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 200 << 30:
        pytest.skip("200 GiB of GPU memory wanted")
    yield
    torch.cuda.empty_cache()


def test_products_of_one_row_tiles():
    """A workgroup to a key."""
    import torch

    import paper_2603_08957_amd as tre

    keys, k = (1 << 24) + 1000, 32
    plan = tre.Plan("vd,nd->nv", "v", {"v": keys, "n": 1, "d": k}, {"v": 1}, "mxfp4")
    # whole numbers up to 6: quantised as they are, and every sum exact
    u = torch.randint(-4, 5, (keys, k), dtype=torch.int8, device="cuda").float()
    u[:, 0] = 4
    v = torch.randint(-4, 5, (1, k), device="cuda").float()
    v[0, 1] = 4
    uk = torch.arange(keys, dtype=torch.int32, device="cuda").reshape(keys, 1)
    out = tre.einsum(plan, uk, tre.mx_quantize(plan, "u", u), None, tre.mx_quantize(plan, "v", v))
    assert out.n_w == keys and torch.equal(out.w_keys, uk)
    assert torch.equal(out.w_tiles.view(-1), (u * v).sum(1))


@pytest.mark.parametrize("n,d", [((1 << 26) + 5, 513), ((1 << 28) + 9, 257)])  # a wavefront to a row, to four rows
def test_lookup(n, d):
    import torch

    import paper_2603_08957_amd as tre

    vocab = 1000
    table = torch.randn((vocab, d), device="cuda").to(torch.bfloat16)
    ids = torch.randint(-1, vocab, (n,), dtype=torch.int32, device="cuda")
    out = tre.lookup(table, ids)
    step = 1 << 22
    for at in range(0, n, step):
        assert torch.equal(out[at:at + step], tre.lookup(table, ids[at:at + step].contiguous())), at


@pytest.mark.parametrize("labels,k,dtype", [("ik", {"k": 1}, "bf16"), ("ki", {"k": 2}, "f32"), ("kil", {"k": 2, "l": 2}, "bf16")])
def test_quantize_and_back(labels, k, dtype):
    """Along rows, across them, and element by element."""
    import torch

    import paper_2603_08957_amd as tre

    n, rows, step = 4097, 1 << 20, 64
    plan = tre.Plan(f"{labels},{'jlk' if 'l' in labels else 'jk'}->ij", "i", {"i": rows, "j": 1, **k}, {"i": rows}, "mxfp4")
    x = torch.empty((n, plan.tile_elems[0]), dtype={"f32": torch.float32, "bf16": torch.bfloat16}[dtype], device="cuda").normal_()
    q = tre.mx_quantize(plan, "u", x)
    for at in range(0, n, step):
        assert torch.equal(q[at:at + step], tre.mx_quantize(plan, "u", x[at:at + step])), at
    tre.mx_dequantize(plan, "u", q, out=x)
    for at in range(0, n, step):
        assert torch.equal(x[at:at + step], tre.mx_dequantize(plan, "u", q[at:at + step], dtype=x.dtype)), at


def test_contractions_of_other_types_refuse():
    """Above 2^24 keys of a workgroup each."""
    import torch

    import paper_2603_08957_amd as tre

    d = 130
    v = torch.randn((1, d), device="cuda")
    for keys in ((1 << 24) - 10, 1 << 24):
        plan = tre.Plan("id,d->id", "i", {"i": keys, "d": d}, {"i": 1})
        uk = torch.arange(keys, dtype=torch.int32, device="cuda").reshape(keys, 1)
        u = torch.ones((keys, d), device="cuda")
        if keys < 1 << 24:
            assert torch.equal(tre.einsum(plan, uk, u, None, v).w_tiles, v.expand(keys, d))
            continue
        with pytest.raises(tre.TreError) as e:
            tre.einsum(plan, uk, u, None, v)
        assert e.value.status == "TRE_E_DEVICE"
