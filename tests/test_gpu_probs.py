"""Log probabilities of scores and their gradient on the GPU, against float64.

With u = 2^-24: a difference x - m and its product with the scale (itself two
products) are off by 4 u of d = scale (x - m) at most, so e^d by 4 u |d| + 2 u (the
base-2 exponential's unit in the last place) of itself.  A sum over c words takes
fewer than c + 16 additions and products in a row, each off by u.  So s is off by
e_s = (c + 18 + 4 A) u of itself, A being the mean of |d| under p, and t by
e_s + 4 u max|d e^d ...| likewise: the bounds below take e_s of t's magnitude too.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def types():
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16}


def scores_of(rng, n, vocab, tile, dtype, spread=3.0, strided=False):
    """Scores on the GPU and their rows [n, vocab] in float64."""
    import torch

    T = types()[dtype]
    rows = torch.from_numpy((rng.standard_normal((n, vocab)) * spread).astype(np.float32)).to(T)
    return place(rows, tile, strided), rows.double().numpy()


def place(rows, tile, strided=False):
    import torch

    n, vocab = rows.shape
    x = rows.view(n, vocab // tile, tile).transpose(0, 1).contiguous() if tile else rows
    if not strided:
        return x.cuda()
    if tile:
        buf = torch.full((x.shape[0] + 1, n + 2, tile + 3), 77.0, dtype=rows.dtype)
        view = buf.cuda()[1:, 1:n + 1, 2:tile + 2]
    else:
        buf = torch.full((n + 1, vocab + 5), 77.0, dtype=rows.dtype)
        view = buf.cuda()[:n, 3:vocab + 3]
    view.copy_(x)
    return view


def rows_of(x):
    return x if x.dim() == 2 else x.transpose(0, 1).reshape(x.shape[1], -1)


class Reference:
    def __init__(self, x, ids, scale):
        scale = np.float64(np.float32(scale))
        n, vocab = x.shape
        self.m = x.max(1)
        self.empty = np.isneginf(self.m)
        m = np.where(self.empty, 0, self.m)
        with np.errstate(all="ignore"):
            self.d = (x - m[:, None]) * scale
            e = np.exp(self.d)
            s = e.sum(1)
            self.logs = np.log(s)
            self.p = np.where(self.empty[:, None], 0, e / np.where(s == 0, 1, s)[:, None])
            dd = np.where(e > 0, self.d, 0)
            self.mean = (self.p * -dd).sum(1)          # A
            self.square = (self.p * dd ** 2).sum(1)
            self.entropy = np.where(self.empty, 0, self.logs + self.mean)
            self.lse = np.where(self.empty, -np.inf, scale * m + self.logs)
            # 1.25 times the lowest fp32 value, -4.25e38, has no fp32 value but -inf
            self.lse = np.where(np.abs(self.lse) > np.finfo(np.float32).max, np.sign(self.lse) * np.inf, self.lse)
            self.logp = np.where(self.empty[:, None], -np.inf, self.d - self.logs[:, None])
        self.scale, self.vocab = scale, vocab
        self.keep = None if ids is None else (ids >= 0) & (ids < vocab)
        if ids is not None:
            at = np.where(self.keep, ids, 0)
            self.log_prob = np.where(self.keep, self.logp[np.arange(n), at], 0)
            self.d_id = np.where(self.keep, self.d[np.arange(n), at], 0)
        self.e_s = (vocab + 18 + 4 * self.mean) * U

    def check(self, r, ids, top, entropy):
        def near(got, want, tol, what):
            got = got.cpu().double().numpy()
            assert np.array_equal(np.isneginf(got), np.isneginf(want)), what
            ok = np.isfinite(want)
            assert np.all(np.abs(got[ok] - want[ok]) <= np.broadcast_to(tol, want.shape)[ok]), (what, np.abs(got - want)[ok].max())

        with np.errstate(invalid="ignore"):
            logs = np.abs(np.where(self.empty, 0, self.logs))
            assert np.array_equal(r.stats[:, 0].cpu().double().numpy(), self.m)
            near(r.stats[:, 1], self.logs, self.e_s + 4 * U * logs, "log of the sum")
            size = np.abs(np.where(self.empty, 0, self.m)) * self.scale + logs
            near(r.lse, self.lse, self.e_s + 6 * U * size, "lse")
            if ids is not None:
                near(r.log_prob, self.log_prob, self.e_s + 6 * U * (logs + np.abs(np.where(np.isfinite(self.d_id), self.d_id, 0))), "log_prob")
            else:
                assert r.log_prob is None
            if entropy:
                # t: each term off by its exponential's 4 u |d| + 3 u and d's 4 u; then the sum
                tol = self.e_s * (1 + 2 * self.mean) + U * (4 * self.square + 8 * self.mean) + 6 * U * (logs + self.mean)
                near(r.entropy, self.entropy, tol, "entropy")
                assert (r.entropy.cpu() >= 0).all()
            else:
                assert r.entropy is None
            if top:
                order = np.stack([np.lexsort((np.arange(self.vocab), -row)) for row in self.d])[:, :top]
                assert np.array_equal(r.top_ids.cpu().numpy(), order)
                lp = np.take_along_axis(self.logp, order, 1)
                d = np.take_along_axis(self.d, order, 1)
                near(r.top_log_probs, lp, self.e_s[:, None] + 6 * U * (logs[:, None] + np.abs(np.where(np.isfinite(d), d, 0))), "top")
            else:
                assert r.top_ids is None and r.top_log_probs is None


SIZES = [(1, 1, 0), (3, 7, 0), (2, 8, 1), (5, 60, 20), (4, 64, 64), (3, 1000, 0), (2, 1001, 7), (7, 4096, 128), (1, 5000, 250),
         (2, 16397, 0), (33, 8200, 100), (1, 70001, 0), (3, 40960, 128), (600, 20000, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,tile", SIZES)
def test_log_probs(n, vocab, tile, dtype):
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(n * 31 + vocab)
    for k, (top, entropy, scale, strided) in enumerate([(0, False, 1.0, False), (min(5, vocab), True, 0.7, True),
                                                        (min(64, vocab), False, 1.9, False), (1, True, 1.0, True)]):
        x, rows = scores_of(rng, n, vocab, tile, dtype, strided=strided)
        ids = rng.integers(0, vocab, n)
        ids[rng.random(n) < 0.2] = -3
        status = torch.zeros(1, dtype=torch.int64, device="cuda")
        dev = torch.from_numpy(ids).to(torch.int32 if k % 2 else torch.int64).cuda()
        r = tre.log_probs(x, dev, scale=scale, top=top, entropy=entropy, status=status)
        Reference(rows, ids, scale).check(r, ids, top, entropy)
        assert status.item() == 0
        again = tre.log_probs(x, dev, scale=scale, top=top, entropy=entropy)
        for a, b in zip(vars(r).values(), vars(again).values()):
            assert a is None and b is None or torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,tile", [(2047, 8250, 250), (2048, 8250, 250), (2051, 8193, 0)])
def test_many_rows(n, vocab, tile, dtype):
    """A wavefront to each of many rows, four to one of fewer."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(n + vocab)
    x, rows = scores_of(rng, n, vocab, tile, dtype, strided=True)
    ids = rng.integers(0, vocab, n)
    want = Reference(rows, ids, 0.7)
    for top, entropy in ((0, True), (9, True)):
        r = tre.log_probs(x, torch.from_numpy(ids).cuda(), scale=0.7, top=top, entropy=entropy)
        want.check(r, ids, top, entropy)
    again = tre.log_probs(x, torch.from_numpy(ids).cuda(), scale=0.7, top=9, entropy=True)
    for a, b in zip(vars(r).values(), vars(again).values()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,tile", [(1, 300, 0), (12, 515, 103), (12, 9000, 0), (3, 33000, 250), (12, 40000, 0)])
def test_rows_of_few_words(n, vocab, tile, dtype):
    """-inf: masked words, rows of one word and of none; all scores alike; scores of one sign of zero and the other."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(vocab)
    rows = torch.from_numpy((rng.standard_normal((n, vocab)) * 2).astype(np.float32)).to(types()[dtype])
    rows[torch.from_numpy(rng.random((n, vocab)) < 0.6)] = -math.inf
    cases = [lambda r: r.fill_(-math.inf), lambda r: r.fill_(1.5), lambda r: r.fill_(-math.inf)[vocab - 1:].fill_(-2.0),
             lambda r: r.copy_(torch.arange(vocab).float() / 64), lambda r: r.copy_(-torch.arange(vocab).float() / 64),
             lambda r: r.copy_((torch.arange(vocab) % 2).float() * -0.0), lambda r: r.fill_(torch.finfo(r.dtype).min),
             lambda r: r.fill_(-math.inf)[1:3].fill_(3.0), lambda r: r.fill_(-0.0)[vocab // 2:].fill_(0.0)]
    for at in range(0, len(cases), n):
        for i, f in enumerate(cases[at:at + n]):
            f(rows[i])
        ids = rng.integers(0, vocab, n)
        x = place(rows, tile)
        for top in (0, 3, 64):
            r = tre.log_probs(x, torch.from_numpy(ids).cuda(), scale=1.25, top=top, entropy=True)
            Reference(rows.double().numpy(), ids, 1.25).check(r, ids, top, True)
        # without gradient from words that cannot come, and none in a row of none
        g = torch.ones(n, device="cuda")
        dx = rows_of(tre.log_probs_grad(x, r.stats, torch.from_numpy(ids).cuda(), g, g, g, r.entropy, scale=1.25, dtype=torch.float32))
        ref = Reference(rows.double().numpy(), ids, 1.25)
        check_grad(dx, ref, ids, np.ones(n), np.ones(n), np.ones(n), "f32")


def test_nan_and_inf():
    import torch

    import paper_2603_08957_amd as tre

    for n, vocab in ((4, 100), (4, 9000), (1, 50000)):
        rng = np.random.default_rng(vocab)
        for bad in (math.nan, math.inf):
            x, _ = scores_of(rng, n, vocab, 0, "f32")
            x[0, vocab // 3] = bad
            ids = torch.arange(n, device="cuda")
            r = tre.log_probs(x, ids, top=2, entropy=True)
            for t in (r.log_prob, r.lse, r.entropy, r.top_log_probs):
                assert t[0].isnan().all() and t[1:].isfinite().all()
            g = torch.ones(n, device="cuda")
            dx = tre.log_probs_grad(x, r.stats, ids, g)
            assert dx[0].isnan().all() and dx[1:].isfinite().all()
        x[0] = math.nan  # ranks as -inf: words in their order
        assert tre.log_probs(x, top=3).top_ids[0].tolist() == [0, 1, 2]


def check_grad(dx, ref, ids, g, gl, gh, dtype):
    """p is off by e_s + 4 u (|d| + |log s|) + 2 u of itself; the factor by a few u of the terms' magnitudes."""
    n, vocab = ref.p.shape
    p = ref.p
    logp = np.where(p > 0, ref.logp, 0)
    h = ref.entropy[:, None]
    keep = ref.keep if ref.keep is not None else np.zeros(n, bool)
    g = np.where(keep, g, 0)
    want = p * (gl - g)[:, None] - gh[:, None] * p * (logp + h)
    size = p * ((np.abs(gl) + np.abs(g))[:, None] + np.abs(gh)[:, None] * (np.abs(logp) + h))
    one = np.zeros((n, vocab))
    one[np.arange(n)[keep & ~ref.empty], ids[keep & ~ref.empty]] = 1
    want, size = want + one * g[:, None], size + one * np.abs(g)[:, None]
    want *= ref.scale
    logs = np.where(ref.empty, 0, np.abs(ref.logs))[:, None]
    d = np.abs(np.where(np.isfinite(ref.d), ref.d, 0))
    # log s and the entropy come as the forward pass left them, off by e_s and its tolerance
    off = 3 * ref.e_s[:, None] * (1 + h + np.where(p > 0, np.abs(logp), 0)) + U * (12 * (d + logs) + 24) + U * 8 * ref.square[:, None]
    tol = size * ref.scale * off + np.abs(gh)[:, None] * p * ref.scale * off
    got = dx.cpu().double().numpy()
    # an exponential below 2^-126 is 0: off by so much times the factor that it meets, |log p| + H among it, which is above
    # 87 there (with every gradient 1, 2 + 87 + H of 2^-126 is more than 2^-120)
    small = 2.0 ** -126 * ref.scale * ((np.abs(gl) + np.abs(g))[:, None] + np.abs(gh)[:, None] * (d + logs + h))
    bad = np.abs(got - want) > tol + HALF[dtype] * (np.abs(want) + tol) + small
    assert not bad.any() and np.isfinite(got).all(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n,vocab,tile", SIZES)
def test_log_probs_grad(n, vocab, tile, dtype, out):
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(n * 7 + vocab)
    T = types()
    for k, which in enumerate(["p", "plh", "l", "h", "ph"]):
        scale = (1.0, 0.6)[k % 2]
        x, rows = scores_of(rng, n, vocab, tile, dtype, strided=k % 2 == 1)
        ids = rng.integers(0, vocab, n)
        ids[rng.random(n) < 0.2] = -1
        gs = [torch.from_numpy(rng.standard_normal(n).astype(np.float32) * (c in which)).cuda() for c in "plh"]
        dev = torch.from_numpy(ids).to(torch.int64 if k % 2 else torch.int32).cuda()
        r = tre.log_probs(x, dev, scale=scale, entropy=True)
        kw = {name: g for name, g, c in zip(("grad_log_prob", "grad_lse", "grad_entropy"), gs, "plh") if c in which}
        dx = tre.log_probs_grad(x, r.stats, dev, entropy=r.entropy, scale=scale, dtype=T[out], **kw)
        assert dx.shape == x.shape and dx.dtype == T[out]
        ref = Reference(rows, ids, scale)
        check_grad(rows_of(dx), ref, ids, *(g.double().cpu().numpy() for g in gs), out)
        # into a layout of its own, whose other elements stay
        buf = torch.full((x.shape[0] + 1, *x.shape[1:-1], x.shape[-1] + 3), 5.0, dtype=T[out], device="cuda")
        own = buf[1:, ..., 2:x.shape[-1] + 2]
        tre.log_probs_grad(x, r.stats, dev, entropy=r.entropy, scale=scale, out=own, **kw)
        assert torch.equal(own, dx)
        own.fill_(5.0)
        assert (buf == 5.0).all()
        if dtype == out:  # in place
            assert tre.log_probs_grad(x, r.stats, dev, entropy=r.entropy, scale=scale, out=x, **kw) is x
            assert torch.equal(x, dx)


def test_grad_against_differences():
    """f(x + h v) - f(x - h v) over 2 h of the forward pass in float64 stands for the formula's derivative; the kernel's gradient
    along v agrees to the difference's own error, h^2 / 6 times the third derivative (below 8 for softmax terms and |v| <= 1,
    scale 1) and 2^-50 / h of cancellation, plus fp32's 2^-20."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(5)
    n, vocab = 6, 50
    x, rows = scores_of(rng, n, vocab, 10, "f32", spread=1.0)
    ids = rng.integers(0, vocab, n)
    g, gl, gh = rng.standard_normal((3, n)).astype(np.float32)
    dev = torch.from_numpy(ids).cuda()
    r = tre.log_probs(x, dev, entropy=True)
    dx = rows_of(tre.log_probs_grad(x, r.stats, dev, *(torch.from_numpy(t).cuda() for t in (g, gl, gh)), entropy=r.entropy))
    v = rng.uniform(-1, 1, (n, vocab))

    def loss(y):
        f = Reference(y, ids, 1.0)
        return g * f.log_prob + gl * f.lse + gh * f.entropy

    h = 1e-4
    diff = (loss(rows + h * v) - loss(rows - h * v)) / (2 * h)
    got = (dx.cpu().double().numpy() * v).sum(1)
    assert np.all(np.abs(got - diff) <= (np.abs(g) + np.abs(gl) + np.abs(gh)) * (8 * h * h / 6 * vocab + 2.0 ** -50 / h * 64 + vocab * 2.0 ** -20))


def test_words_out_of_range():
    import torch

    import paper_2603_08957_amd as tre

    x = torch.randn(3, 500, device="cuda")
    status = torch.zeros(1, dtype=torch.int64, device="cuda")
    ids = torch.tensor([499, 500, 2 ** 40], device="cuda")
    r = tre.log_probs(x, ids, status=status)
    assert status.item() == tre.tre.STATUS_CODE["TRE_E_KEYRANGE"]
    assert r.log_prob[1:].tolist() == [0.0, 0.0] and r.log_prob[0] != 0
    status.zero_()
    dx = tre.log_probs_grad(x, r.stats, ids, torch.ones(3, device="cuda"), status=status)
    assert status.item() == tre.tre.STATUS_CODE["TRE_E_KEYRANGE"] and not dx[1:].any() and dx[0].any()


def test_rows_without_gradient_are_not_read():
    import torch

    import paper_2603_08957_amd as tre

    x = torch.randn(4, 3000, device="cuda")
    x[1] = math.nan
    ids = torch.tensor([5, -1, -1, 7], device="cuda")
    r = tre.log_probs(x, ids)
    dx = tre.log_probs_grad(x, r.stats, ids, torch.ones(4, device="cuda"))
    assert not dx[1:3].any() and dx[0].isfinite().all() and dx[0].any() and dx[3].any()
    r = tre.log_probs(x, ids, entropy=True)
    assert r.entropy[1].isnan()
    gh = torch.tensor([1.0, 0, 0, 1], device="cuda")
    dx = tre.log_probs_grad(x, r.stats, ids, torch.ones(4, device="cuda"), grad_entropy=gh, entropy=r.entropy)
    assert not dx[1:3].any() and dx[0].isfinite().all() and dx[0].any() and dx[3].any()


@pytest.mark.parametrize("n", [0, 1])
def test_no_tokens(n):
    import torch

    import paper_2603_08957_amd as tre

    x = torch.randn(n, 40, device="cuda")
    ids = torch.zeros(n, dtype=torch.int64, device="cuda")
    r = tre.log_probs(x, ids, top=2, entropy=True)
    assert r.log_prob.shape == (n,) and r.top_ids.shape == (n, 2) and r.stats.shape == (n, 2)
    assert tre.log_probs_grad(x, r.stats, ids, torch.ones(n, device="cuda")).shape == (n, 40)
    assert tre.log_probs(x, top=2).top_ids.shape == (n, 2)


def test_streams_graphs_and_devices():
    """A captured pair of calls, replayed with the program's own work between; a caller's stream."""
    import torch

    import paper_2603_08957_amd as tre

    x = torch.randn(5, 30000, device="cuda")
    ids = torch.randint(0, 30000, (5,), device="cuda")
    g = torch.randn(5, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r = tre.log_probs(x, ids, top=7, entropy=True, stream=s)
    dx = tre.log_probs_grad(x, r.stats, ids, g, grad_entropy=g, entropy=r.entropy, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    want = tre.log_probs(x, ids, top=7, entropy=True)
    for a, b in zip(vars(r).values(), vars(want).values()):
        assert torch.equal(a, b)
    assert torch.equal(dx, tre.log_probs_grad(x, want.stats, ids, g, grad_entropy=g, entropy=want.entropy))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = tre.log_probs(x, ids, top=7, entropy=True)
        dx = tre.log_probs_grad(x, r.stats, ids, g, grad_entropy=g, entropy=r.entropy)
    for _ in range(4):
        x.copy_(torch.randn(5, 30000, device="cuda"))
        ids.copy_(torch.randint(0, 30000, (5,), device="cuda"))
        graph.replay()
        want = tre.log_probs(x, ids, top=7, entropy=True)
        torch.cuda.synchronize()
        for a, b in zip(vars(r).values(), vars(want).values()):
            assert torch.equal(a, b)
        assert torch.equal(dx, tre.log_probs_grad(x, want.stats, ids, g, grad_entropy=g, entropy=want.entropy))


def test_tiles_of_a_score_einsum():
    """Tokens' rows, their scores, loss and gradients over one table, as a model's last layer has them: against float64 autograd.

    The scores are products of bf16 values with fp32 sums over 64 terms, off by 65 u of the magnitudes' sum, a; they carry over
    to probabilities as factors e^(2 max a), and so into the gradients, which take 40 or 500 additions more."""
    import torch

    import paper_2603_08957_amd as tre

    n, vocab, d, tile = 40, 500, 64, 20
    torch.manual_seed(3)
    table = (torch.randn(vocab, d) / 4).bfloat16()
    ids = torch.randint(0, vocab, (n,))
    ids[::7] = -1
    words = torch.randint(0, vocab, (n,))
    words[3] = -1
    plan = tre.Plan("nd,vd->nv", "v", {"v": vocab, "n": n, "d": d}, {"v": tile}, "bf16")
    by_x = tre.Plan("nv,vd->nd", "v", {"v": vocab, "n": n, "d": d}, {"v": tile}, "bf16")
    keys = torch.arange(vocab // tile, dtype=torch.int32, device="cuda").view(-1, 1)
    dev = table.cuda()
    x = tre.lookup(dev, ids.cuda())
    y = tre.einsum(plan, None, x.view(1, -1), keys, dev.view(vocab // tile, -1))
    tiles = y.w_tiles.view(-1, n, tile)
    r = tre.log_probs(tiles, words.cuda(), top=3, entropy=True)
    g = torch.full((n,), -1.0 / n, device="cuda")
    dy = tre.log_probs_grad(tiles, r.stats, words.cuda(), g, dtype=torch.bfloat16)
    dx = tre.einsum(by_x, keys, dy.view(vocab // tile, -1), keys, dev.view(vocab // tile, -1)).w_tiles.view(n, d)
    dt = tre.lookup_grad(dx, ids.cuda(), vocab)

    t = table.double()
    xr = torch.where(ids[:, None] >= 0, t[ids.clamp_min(0)], 0.0)
    z = xr @ t.T
    lp = torch.log_softmax(z, 1)
    a = 65 * U * float((xr.abs() @ t.abs().T).max())
    want = torch.where(words >= 0, lp[torch.arange(n), words.clamp_min(0)], 0.0)
    tol = 2 * a + (vocab + 60) * U + 8 * U * float(lp.abs().max())
    assert (r.log_prob.cpu().double() - want).abs().max() <= tol
    assert (r.entropy.cpu().double() + (lp.exp() * lp).sum(1)).abs().max() <= tol * (2 + float(lp.abs().max()))
    assert (r.top_log_probs.cpu().double() - lp.topk(3, 1)[0]).abs().max() <= tol
    gz = lp.exp() * torch.where(words >= 0, 1.0 / n, 0.0)[:, None]
    gz[torch.arange(n)[words >= 0], words[words >= 0]] -= 1.0 / n
    gx = gz @ t
    off = (gz.abs() * (2.0 ** -8 + 2 * tol + 600 * U)) @ t.abs() + 2 * tol / n
    assert ((dx.cpu().double() - gx).abs() <= off).all()
    gt = torch.zeros(vocab, d, dtype=torch.double).index_add_(0, ids[ids >= 0], gx[ids >= 0])
    ot = torch.zeros(vocab, d, dtype=torch.double).index_add_(0, ids[ids >= 0], off[ids >= 0] + 40 * U * gx[ids >= 0].abs())
    assert ((dt.cpu().double() - gt).abs() <= ot + 41 * U).all()


def test_refusals():
    import torch

    import paper_2603_08957_amd as tre

    def refused(wanted, f, *a, **kw):
        with pytest.raises(tre.TreError) as e:
            f(*a, **kw)
        assert e.value.status == wanted

    x = torch.randn(4, 60, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    refused("TRE_E_SHAPE", tre.log_probs, x.T)
    refused("TRE_E_SHAPE", tre.log_probs, x[:, :0])
    refused("TRE_E_SHAPE", tre.log_probs, x.view(2, 2, 3, 20))
    refused("TRE_E_DTYPE", tre.log_probs, x.half())
    refused("TRE_E_SHAPE", tre.log_probs, x, ids[:3])
    refused("TRE_E_SHAPE", tre.log_probs, x.view(4, 3, 20), ids)  # (tiles of three tokens)
    refused("TRE_E_SHAPE", tre.log_probs, x, ids.repeat(2)[::2])
    refused("TRE_E_DTYPE", tre.log_probs, x, ids.float())
    refused("TRE_E_ARG", tre.log_probs, x, ids.cpu())
    refused("TRE_E_SHAPE", tre.log_probs, x, ids, top=61)
    refused("TRE_E_SHAPE", tre.log_probs, torch.randn(4, 80, device="cuda"), ids, top=65)
    refused("TRE_E_SHAPE", tre.log_probs, x, ids, top=-1)
    for scale in (0.0, -1.0, math.nan, math.inf):
        refused("TRE_E_ARG", tre.log_probs, x, ids, scale=scale)
    refused("TRE_E_DTYPE", tre.log_probs, x, ids, status=torch.zeros(1, device="cuda"))
    long = torch.randn(1, 1 << 20, device="cuda")
    assert tre.log_probs_workspace_bytes(1, 1 << 20) > 0
    refused("TRE_E_WORKSPACE", tre.log_probs, long, ws=torch.empty(256, dtype=torch.uint8, device="cuda")[:16])
    refused("TRE_E_ARG", tre.log_probs, long, ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[8:])
    ws = tre.alloc_workspace(tre.log_probs_workspace_bytes(1, 1 << 20, top=3))
    assert torch.equal(tre.log_probs(long, top=3, ws=ws).top_ids, tre.log_probs(long, top=3).top_ids)

    r = tre.log_probs(x, ids, entropy=True)
    g = torch.ones(4, device="cuda")
    refused("TRE_E_ARG", tre.log_probs_grad, x, r.stats, ids)
    refused("TRE_E_ARG", tre.log_probs_grad, x, r.stats, None, g)
    refused("TRE_E_ARG", tre.log_probs_grad, x, r.stats, ids, grad_entropy=g)
    refused("TRE_E_SHAPE", tre.log_probs_grad, x, r.stats[:, 0], ids, g)
    refused("TRE_E_DTYPE", tre.log_probs_grad, x, r.stats.double(), ids, g)
    refused("TRE_E_SHAPE", tre.log_probs_grad, x, r.stats, ids, g.repeat(2)[::2])
    refused("TRE_E_DTYPE", tre.log_probs_grad, x, r.stats, ids, g.double())
    refused("TRE_E_ARG", tre.log_probs_grad, x, r.stats, ids, g.cpu())
    refused("TRE_E_DTYPE", tre.log_probs_grad, x, r.stats, ids, g, dtype=torch.float16)
    refused("TRE_E_SHAPE", tre.log_probs_grad, x, r.stats, ids, g, out=torch.empty(4, 61, device="cuda"))
    refused("TRE_E_SHAPE", tre.log_probs_grad, x, r.stats, ids, g, dtype=torch.bfloat16, out=torch.empty(4, 60, device="cuda"))
    refused("TRE_E_SHAPE", tre.log_probs_grad, x, r.stats, ids, g, out=torch.empty(1, 60, device="cuda").expand(4, 60))
    refused("TRE_E_SHAPE", tre.log_probs_grad, x, r.stats, ids, g, out=torch.empty(60, 4, device="cuda").T)
    # in place, but laid out otherwise
    buf = torch.randn(4, 120, device="cuda")
    refused("TRE_E_ARG", tre.log_probs_grad, buf[:, :60], r.stats, ids, g, out=buf.view(8, 60)[:4])


def test_scores_that_all_tokens_share():
    """Rows at a stride of zero are read as they are."""
    import torch

    import paper_2603_08957_amd as tre

    x = torch.randn(1, 5000, device="cuda")
    ids = torch.arange(6, device="cuda")
    r = tre.log_probs(x.expand(6, 5000), ids, top=4)
    want = tre.log_probs(x.repeat(6, 1), ids, top=4)
    for a, b in zip(vars(r).values(), vars(want).values()):
        assert a is None and b is None or torch.equal(a, b)
    g = torch.ones(6, device="cuda")
    assert torch.equal(tre.log_probs_grad(x.expand(6, 5000), r.stats, ids, g), tre.log_probs_grad(x.repeat(6, 1), r.stats, ids, g))
