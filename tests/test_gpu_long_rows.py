"""Log probabilities of long rows on the GPU, against float64 with bounds by the longest chain of sums, and against counts that
fp32 holds exactly.

With u = 2^-24.  A lane takes 4 runs of 16 bytes a step: so many additions, and the product that brings its sum to the new
maximum, whose factor is good to 2 u (and to 4 u of the exponent, which with the score's own makes 4 u |d|).  A row of up to
3584 runs may be one wavefront's, others are taken by 256 lanes at least, by 1024 where they are cut into parts.  At most 16 joins follow (64 lanes 6, 16 wavefronts 4,
32 parts 5; 4 wavefronts 3), each a factor, a product and a sum: 4 u.  So a sum is off by (steps (4 E + 3) + 66 + 4 A) u, E the
scores of 16 bytes and A the mean of |d|, of itself: some hundred u, where the number of words alone would allow as many u as
there are words, and one lost run of them among 50,000 would pass.
"""
import math

import numpy as np
import pytest

from test_gpu_probs import SIZES, U, Reference, check_grad, place, rows_of, scores_of, types

pytestmark = pytest.mark.gpu


def runs_of(vocab, tile, dtype):
    e = 4 if dtype == "f32" else 8
    cols = tile or vocab
    return vocab // cols * -(-cols // e)


class Chain(Reference):
    def __init__(self, x, ids, scale, tile, dtype, parts=False):
        super().__init__(x, ids, scale)
        runs, e = runs_of(self.vocab, tile, dtype), 4 if dtype == "f32" else 8
        steps = -(-runs // (4096 if parts else 256 if runs <= 3584 else 1024))
        self.e_s = (steps * (4 * e + 3) + 66 + 4 * self.mean) * U


def in_parts(n, vocab, tile, dtype, top):
    """Asked of the library: rows that are cut into parts, which take a workspace."""
    import paper_2603_08957_amd as tre

    return tre.log_probs_workspace_bytes(n, vocab, tile or None, types()[dtype], top) > 0


def check_all(n, vocab, tile, dtype, parts, modes, rng):
    import torch

    import paper_2603_08957_amd as tre

    for k, (top, entropy, scale, strided) in enumerate(modes):
        assert not parts or in_parts(n, vocab, tile, dtype, top)
        x, rows = scores_of(rng, n, vocab, tile, dtype, strided=strided)
        ids = rng.integers(0, vocab, n)
        ids[rng.random(n) < 0.2] = -3
        dev = torch.from_numpy(ids).to(torch.int32 if k % 2 else torch.int64).cuda()
        ref = Chain(rows, ids, scale, tile, dtype, parts)
        r = tre.log_probs(x, dev, scale=scale, top=top, entropy=entropy)
        ref.check(r, ids, top, entropy)
        again = tre.log_probs(x, dev, scale=scale, top=top, entropy=entropy)
        for a, b in zip(vars(r).values(), vars(again).values()):
            assert a is None and b is None or torch.equal(a, b)
        if entropy:
            g = torch.from_numpy(rng.standard_normal((3, n)).astype(np.float32)).cuda()
            dx = tre.log_probs_grad(x, r.stats, dev, *g, entropy=r.entropy, scale=scale)
            check_grad(rows_of(dx), ref, ids, *g.double().cpu().numpy(), dtype)


MODES = [(0, False, 1.0, False), (5, True, 0.7, True), (64, False, 1.9, False), (1, True, 1.0, True), (0, True, 1.3, False)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,tile", [s for s in SIZES if s[1] >= 64])
def test_rows(n, vocab, tile, dtype):
    check_all(n, vocab, tile, dtype, False, MODES[:4], np.random.default_rng(n + vocab))


# rows of more than 16384 runs, few enough: whole runs, overlapping last ones, tiles shorter than a run, 2 to 17 parts
PARTS = [(2, 66000, 0, "f32"), (3, 140001, 0, "f32"), (5, 75000, 250, "f32"), (2, 196608, 128, "f32"), (2, 60000, 3, "f32"),
         (100, 66002, 0, "f32"), (1, 263000, 0, "f32"), (2, 135000, 0, "bf16"), (3, 262151, 0, "bf16"), (2, 300000, 250, "bf16"),
         (4, 140288, 128, "bf16"), (2, 100005, 5, "bf16"), (1, 500002, 250001, "bf16"), (128, 131200, 400, "bf16")]


@pytest.mark.parametrize("n,vocab,tile,dtype", PARTS)
def test_rows_in_parts(n, vocab, tile, dtype):
    check_all(n, vocab, tile, dtype, True, MODES if n < 50 else MODES[1:3], np.random.default_rng(n + vocab))


@pytest.mark.parametrize("n,vocab,tile,dtype", [(5, 70000, 250, "f32"), (5, 140001, 0, "f32"), (5, 270000, 0, "bf16"), (5, 100005, 5, "bf16")])
def test_rows_in_parts_of_few_words(n, vocab, tile, dtype):
    """-inf: parts and rows without a word that can come, fewer of them than top words; all alike; rising and falling."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(vocab)
    rows = torch.from_numpy((rng.standard_normal((n, vocab)) * 2).astype(np.float32)).to(types()[dtype])
    inf = math.inf

    def some(r, at, value=None):
        r.fill_(-inf)
        r[at] = torch.arange(len(at)).to(r.dtype) / 8 if value is None else value

    cases = [lambda r: r.fill_(-inf), lambda r: r.fill_(1.5), lambda r: some(r, [vocab - 1]), lambda r: some(r, [0]),
             lambda r: r.copy_(torch.arange(vocab).float() / 64), lambda r: r.copy_(-torch.arange(vocab).float() / 64),
             lambda r: r.copy_((torch.arange(vocab) % 2).float() * -0.0), lambda r: r.fill_(torch.finfo(r.dtype).min),
             lambda r: r.fill_(-inf)[vocab // 2:vocab // 2 + 70].fill_(3.0), lambda r: r.fill_(-0.0)[vocab // 2:].fill_(0.0),
             lambda r: some(r, list(range(7, vocab, vocab // 20))), lambda r: some(r, list(range(5, vocab, vocab // 63)), 2.0),
             lambda r: r[:vocab * 3 // 4].fill_(-inf), lambda r: r[vocab // 9:].fill_(-inf), lambda r: r[::3].fill_(-inf)]
    for at in range(0, len(cases), n):
        for i, f in enumerate(cases[at:at + n]):
            f(rows[i])
        ids = rng.integers(0, vocab, n)
        dev = torch.from_numpy(ids).cuda()
        x = place(rows, tile)
        ref = Chain(rows.double().numpy(), ids, 1.25, tile, dtype, True)
        for top in (0, 3, 64):
            assert in_parts(n, vocab, tile, dtype, top)
            r = tre.log_probs(x, dev, scale=1.25, top=top, entropy=True)
            ref.check(r, ids, top, True)
        g = torch.ones(n, device="cuda")
        dx = rows_of(tre.log_probs_grad(x, r.stats, dev, g, g, g, r.entropy, scale=1.25, dtype=torch.float32))
        check_grad(dx, ref, ids, np.ones(n), np.ones(n), np.ones(n), "f32")


@pytest.mark.parametrize("n,vocab,tile,dtype", [(3, 70000, 0, "f32"), (2, 140000, 250, "f32"), (3, 300000, 0, "bf16")])
def test_rows_in_parts_with_nan_and_inf(n, vocab, tile, dtype):
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(vocab)
    assert in_parts(n, vocab, tile, dtype, 2)
    for bad in (math.nan, math.inf):
        for at in (0, vocab // 3, vocab - 1):
            _, rows = scores_of(rng, n, vocab, 0, dtype)
            rows = torch.from_numpy(rows).to(types()[dtype])
            rows[1, at] = bad
            x = place(rows, tile)
            ids = torch.arange(n, device="cuda")
            r = tre.log_probs(x, ids, top=2, entropy=True)
            ok = torch.arange(n) != 1
            for t in (r.log_prob, r.lse, r.entropy, r.top_log_probs):
                assert t[1].isnan().all() and t[ok].isfinite().all()
            if bad == math.inf:
                assert r.top_ids[1, 0] == at
            else:
                best = torch.where(rows[1].isnan(), -math.inf, rows[1].float()).numpy()
                assert r.top_ids[1].tolist() == np.lexsort((np.arange(vocab), -best))[:2].tolist()
            dx = rows_of(tre.log_probs_grad(x, r.stats, ids, torch.ones(n, device="cuda")))
            assert dx[1].isnan().all() and dx[ok].isfinite().all()
    rows[1] = math.nan  # (ranks as -inf: words in their order)
    assert tre.log_probs(place(rows, tile), top=3).top_ids[1].tolist() == [0, 1, 2]


@pytest.mark.parametrize("n,vocab,tile,dtype", [(7, 40960, 128, "f32"), (2, 263000, 0, "f32"), (3, 300000, 250, "bf16"), (513, 20000, 0, "bf16"),
                                                (2050, 9000, 250, "f32"), (70001, 65536, 0, "bf16"), (70001, 65536, 128, "bf16"),
                                                (3, 1 << 30, 0, "bf16"), (2, 1 << 30, 1 << 21, "bf16")])
def test_words_are_counted(n, vocab, tile, dtype):
    """Scores of 0 and -inf: the sum is the number of words that can come, whole numbers that fp32 sums exactly up to 2^24 and
    whose joins are off by u each; then one logarithm.  One lost word in 100,000 is seen."""
    import torch

    import paper_2603_08957_amd as tre

    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GiB of GPU memory wanted")
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.empty((vocab // tile, n, tile) if tile else (n, vocab), dtype=types()[dtype], device="cuda")
    x.bernoulli_(0.5, generator=gen).log_()  # 0 or -inf
    ids = torch.randint(0, vocab, (n,), device="cuda", generator=gen)
    words = torch.arange(n, device="cuda")
    given = x[ids // tile, words, ids % tile] if tile else x[words, ids]
    count = torch.zeros(n, dtype=torch.float64, device="cuda")
    for part in (x.split(1) if tile else x.T.split(1 << 20)):  # (no second copy of it all)
        count += (part[0] == 0).sum(1) if tile else (part == 0).sum(0)
    r = tre.log_probs(x, ids, top=3, entropy=True)
    logs = count.log()
    tol = (16 + 4) * U + 4 * U * logs
    assert (r.stats[:, 0] == 0).all()
    for got in (r.stats[:, 1], r.lse, r.entropy, -r.top_log_probs[:, 0], -r.top_log_probs[:, 2]):
        assert ((got.double() - logs).abs() <= tol).all(), ((got.double() - logs).abs() / tol).max()
    assert torch.equal(r.log_prob.isneginf(), given.isneginf())
    assert ((r.log_prob.double() + logs).abs() <= tol)[given == 0].all()
    # the first three words that can come, within 64 words but once in 2^53 rows
    head = rows_of(x[:max(1, 64 // tile) + 1] if tile else x[:, :64])[:, :64] == 0
    order = torch.where(head, torch.arange(head.shape[1], device="cuda"), 64).sort(1)[0][:, :3]
    assert torch.equal(r.top_ids.long(), order)
    # g [given] - g p, p = 0 for words that cannot come; p off by tol, log s rounded in units of log 2, the exponential and rounding
    g = torch.full((n,), 0.5, device="cuda")
    mask = x == 0
    tre.log_probs_grad(x, r.stats, ids, g, out=x)
    p = 1 / count
    half = 2.0 ** -8 if dtype == "bf16" else U
    here = x[ids // tile, words, ids % tile] if tile else x[words, ids]
    want = 0.5 - 0.5 * torch.where(given == 0, p, 0.0)
    assert ((here.double() - want).abs() <= half * want + 8 * U).all()
    if tile:
        x[ids // tile, words, ids % tile] = 0
        mask[ids // tile, words, ids % tile] = False
    else:
        x[words, ids] = 0
        mask[words, ids] = False
    low, high = (-0.5 * p * (1 + s * (half + tol + 4 * U * logs + 8 * U)) for s in (1, -1))
    for part, kept in (zip(x.split(1), mask.split(1)) if tile else zip(x.T.split(1 << 20), mask.T.split(1 << 20))):
        y, k = (part[0], kept[0]) if tile else (part.T, kept.T)
        for a in range(0, n, 4096):
            z, lo, hi = y[a:a + 4096].float(), low[a:a + 4096, None].float(), high[a:a + 4096, None].float()
            # (the bounds' own rounding to fp32: u more)
            assert torch.where(k[a:a + 4096], (z >= lo * (1 + 2 * U)) & (z <= hi * (1 - 2 * U)), z == 0).all()


def test_many_long_rows():
    """The last rows of 70001 of 65536 words, past 2^32 scores, against float64."""
    import torch

    import paper_2603_08957_amd as tre

    n, vocab = 70001, 65536
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GiB of GPU memory wanted")
    for tile in (0, 128):
        x = torch.empty((vocab // tile, n, tile) if tile else (n, vocab), dtype=torch.bfloat16, device="cuda").normal_()
        ids = torch.randint(0, vocab, (n,), device="cuda")
        r = tre.log_probs(x, ids, top=3, entropy=True)
        at = torch.tensor([0, 1, 32767, 65535, 65536, 65537, 69999, 70000])
        rows = rows_of(x[:, at] if tile else x[at]).double().cpu().numpy()
        some = tre.LogProbs(*(t[at] for t in vars(r).values()))
        keep = ids[at].cpu().numpy()
        Chain(rows, keep, 1.0, tile, "bf16").check(some, keep, 3, True)
        del x, r
