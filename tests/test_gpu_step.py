"""The gradient's norm and AdamW steps of many tensors on the GPU, against numpy.

With u = 2^-24: moments are fp32 products and sums in a stated order, so their bits are the oracle's, and so are 8-bit codes.
What is taken off a weight is a product of lr, m c1 and the reciprocal of sqrt(v c2) + eps: c1, c2, lr and eps rounded (u each,
c2 halved by the root), a root and a reciprocal good to one unit (2 u each), five products and a sum: under 14 u of it.  The
weight's own factor and product take 2 u, the last sum one more u of the result.
"""
import math

import numpy as np
import pytest

from oracle import moments

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def types():
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16}


def make(rng, sizes, dtype, spread, shift=0):
    """Tensors on the GPU (the first element `shift` elements off a wide boundary) with guards around them, and their values."""
    import torch

    got = []
    for n in sizes:
        x = torch.from_numpy((rng.standard_normal(n) * spread).astype(np.float32)).to(dtype)
        buf = torch.full((n + 16 + shift,), 9.0, dtype=dtype, device="cuda")
        view = buf[8 + shift:8 + shift + n]
        view.copy_(x)
        got.append((buf, view))
    return got


def values(tensors):
    return [t.float().cpu().numpy().reshape(-1) for t in tensors]


def flat(parts):
    """Values of tensors in the order of the moments, whole blocks of 32."""
    return np.concatenate([np.pad(p, (0, -len(p) % 32)) for p in parts] or [np.zeros(0, np.float32)]).astype(np.float32)


def guards_hold(tensors):
    for buf, view in tensors:
        at = view.storage_offset()
        assert (buf[:at] == 9.0).all() and (buf[at + view.numel():] == 9.0).all()


class Model:
    """Weights and moments stepped by the oracle."""

    def __init__(self, params, bits, dtypes):
        self.p, self.dtypes = params, dtypes
        n = len(flat(params))
        self.bits = bits
        self.m = self.v = np.zeros(n, np.float32)

    def step(self, grads, t, lr, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0, scale=1.0, seed=None):
        """Returns (wanted weights, tolerance) per tensor; the moments become those that are kept."""
        m, v = moments.step32(self.m, self.v, flat(grads), beta1, beta2, scale)
        n = len(m)
        r = moments.chance(n, seed, t) if seed is not None else (None, None, None)
        at, out = 0, []
        for p, dt in zip(self.p, self.dtypes):
            k = len(p)
            want, off = moments.weights64(p, m[at:at + k], v[at:at + k], t, float(np.float32(lr)), beta1, beta2, float(np.float32(eps)), decay)
            tol = 14 * U * off + 2 * U * np.abs(p) + U * np.abs(want)
            if dt == "bf16":
                tol = tol + (2.0 ** -8 if seed is None else 2.0 ** -7) * (np.abs(want) + tol)
            out.append((want, tol))
            at += (k + 31) // 32 * 32
        if self.bits == 8:
            self.state = moments.pack(m, v, r[:2])
            m, v = (x.astype(np.float32) for x in moments.unpack(self.state))
        self.m, self.v = m, v
        return out


SIZES = [[1], [31, 32, 33], [5, 0, 4097, 1, 129, 1024, 2000, 64], [20000, 3, 4096, 8191], [7] * 200, [70001, 1]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pdt,gdt", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("mixed", "mixed")])
@pytest.mark.parametrize("which", range(len(SIZES)))
def test_adamw(which, pdt, gdt, bits):
    import torch

    import paper_2603_08957_amd as tre

    sizes = SIZES[which]
    for seed in (None, 12345678901):
        rng = np.random.default_rng(which)
        T = types()
        pd = [pdt if pdt != "mixed" else ("f32", "bf16")[i % 2] for i in range(len(sizes))]
        gd = [gdt if gdt != "mixed" else ("f32", "bf16")[i // 2 % 2] for i in range(len(sizes))]
        params = [make(rng, [n], T[d], 0.05, i % 4)[0] for i, (n, d) in enumerate(zip(sizes, pd))]
        views = [v for _, v in params]
        state = tre.adamw_state(views, bits)
        assert state.numel() == (2 * len(flat(values(views))) if bits == 32 else len(flat(values(views))) * 33 // 16)
        model = Model(values(views), bits, pd)
        for t in (1, 2, 3):
            grads = [make(rng, [n], T[d], 10.0 ** rng.integers(-6, 2), (i + t) % 3)[0] for i, (n, d) in enumerate(zip(sizes, gd))]
            if t == 2 and sizes[0] > 1:
                grads[0][1].zero_()
            gviews = [v for _, v in grads]
            step, lr, scale = t, 1e-2, 0.3
            if t == 3:  # on the device
                step, lr, scale = torch.tensor([t], device="cuda"), torch.tensor(1e-2, device="cuda"), torch.tensor([0.3], device="cuda")
            tre.adamw(views, gviews, state, step, lr, beta2=0.99, weight_decay=0.1, grad_scale=scale, seed=seed)
            wanted = model.step(values(gviews), t, 1e-2, beta2=0.99, decay=0.1, scale=0.3, seed=seed)
            if bits == 32:
                m, v = (x.cpu().numpy() for x in tre.adamw_moments(state))
            else:
                assert np.array_equal(state.cpu().numpy(), model.state)
                m, v = (x.cpu().numpy() for x in tre.adamw_moments(state))
                mb, vb = (x.float().cpu().numpy() for x in tre.adamw_moments(state, dtype=torch.bfloat16))
                assert np.array_equal(m, mb) and np.array_equal(v, vb)
            assert np.array_equal(m, model.m) and np.array_equal(v, model.v)
            for got, (want, tol) in zip(values(views), wanted):
                assert np.all(np.abs(got - want) <= tol), (t, np.abs(got - want).max())
            guards_hold(params)
            guards_hold(grads)
            model.p = values(views)  # (each step against its own start)


@pytest.mark.parametrize("bits", [32, 8])
def test_many_launches(bits):
    """More tensors than a launch's arguments hold; all of them in one call as each for itself."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(4)
    sizes = [int(n) for n in rng.integers(0, 300, 250)]
    params = [torch.randn(n, device="cuda") for n in sizes]
    grads = [torch.randn(n, device="cuda") for n in sizes]
    alone = [p.clone() for p in params]
    state = tre.adamw_state(params, bits)
    for t in (1, 2):
        tre.adamw(params, grads, state, t, 1e-3)
    for p, q, g in zip(params, alone, grads):
        s = tre.adamw_state([q], bits)
        for t in (1, 2):
            tre.adamw([q], [g], s, t, 1e-3)
        assert torch.equal(p, q)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 1e30])
def test_gradients_that_are_not_finite(value):
    """8-bit blocks with such a moment hold NaN; their neighbours what they would hold without."""
    import torch

    import paper_2603_08957_amd as tre

    params = [torch.ones(200, device="cuda") for _ in range(2)]
    grads = [torch.full((200,), 0.5, device="cuda") for _ in range(2)]
    grads[1][70] = value
    state = tre.adamw_state(params[:1], 8)
    other = state.clone()
    tre.adamw(params[:1], grads[:1], state, 1, 1e-3)
    tre.adamw(params[1:], grads[1:], other, 1, 1e-3)
    m, v = tre.adamw_moments(state)
    m1, v1 = tre.adamw_moments(other)
    hit = torch.zeros(224, dtype=torch.bool, device="cuda")
    hit[64:96] = True
    assert v1[hit].isnan().all() and (m1[hit].isnan().all() or value == 1e30)
    assert torch.equal(m[~hit], m1[~hit]) and torch.equal(v[~hit], v1[~hit])
    assert torch.equal(params[0][96:], params[1][96:]) and torch.equal(params[0][:70], params[1][:70])


def test_small_and_large_moments():
    """Blocks from the least to nearly the largest fp32 value: codes are the oracle's, whose range the kernel's denormals have too."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(8)
    for seed in (None, 3):
        size = 10.0 ** rng.uniform(-44, 18, 100).repeat(32)
        g = torch.from_numpy((rng.standard_normal(3200) * size).astype(np.float32)).cuda()
        p = torch.zeros(3200, device="cuda")
        state = tre.adamw_state([p], 8)
        model = Model([np.zeros(3200)], 8, ["f32"])
        for t in (1, 2):
            tre.adamw([p], [g], state, t, 0.0, seed=seed)
            model.step([g.cpu().numpy()], t, 0.0, seed=seed)
            assert np.array_equal(state.cpu().numpy(), model.state)
            assert np.array_equal(tre.adamw_moments(state)[1].cpu().numpy(), model.v)


def test_chance_is_right_on_average():
    """The mean of n moments rounded by chance is off by five of its deviations, half a step / sqrt(n), at most (and by the
    place's 2^-20); nearest rounding is off by the place itself.  The same seed and step give the same, others do not."""
    import torch

    import paper_2603_08957_amd as tre

    n = 1 << 18
    p, g = torch.full((n,), 1.0, dtype=torch.bfloat16, device="cuda"), torch.full((n,), 1.03, device="cuda")
    g[::32] = 1.9  # the block's largest
    states = []
    for seed, t in ((5, 1), (5, 1), (6, 1), (5, 2)):
        q, state = p.clone(), tre.adamw_state([p], 8)
        tre.adamw([q], [g], state, t, 1e-3, beta1=0.0, beta2=0.5, seed=seed)
        m, v = tre.adamw_moments(state)
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        keep[::32] = False
        step = 2.0 ** -3
        assert abs(m[keep].double().mean().item() - 1.03) < 5 * step / 2 / 500 + step * 2.0 ** -19
        want = 0.5 * float(np.float32(1.03)) ** 2
        assert abs(v[keep].double().mean().item() - want) < 5 * 2.0 ** -4 / 2 / 500 + 2.0 ** -20
        # weights: 1 - lr (m / sqrt(v c2)) lies between two bf16 values
        off = 1e-3 / math.sqrt(0.5 / (1 - 0.5 ** t))
        assert abs(q[keep].double().mean().item() - (1 - off)) < 5 * 2.0 ** -8 / 2 / 500 + 1e-6
        states.append((state, q))
    assert torch.equal(states[0][0], states[1][0]) and torch.equal(states[0][1], states[1][1])
    for s, q in states[2:]:
        assert not torch.equal(states[0][0], s) and not torch.equal(states[0][1], q)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", [[1], [0], [0, 5, 0], [4097], [3, 100000, 17, 1 << 20], [11] * 300, [8192 * 4096 + 77]])
def test_grad_norm(sizes, dtype):
    """Sums in 64 bits, one root, one rounding to fp32; the factor one division and one rounding."""
    import torch

    import paper_2603_08957_amd as tre

    rng = np.random.default_rng(len(sizes))
    T = types()
    if sum(sizes) > 1 << 22:
        each = [torch.randn(n, device="cuda").to(T["bf16" if dtype == "bf16" else "f32"]) for n in sizes]
    else:
        each = [make(rng, [n], T[dtype if dtype != "mixed" else ("f32", "bf16")[i % 2]], 3.0, i % 3)[0][1] for i, n in enumerate(sizes)]
    want = math.sqrt(sum(float(t.double().square().sum()) for t in each))
    for most in (None, 0.01, 1e9, 0.0):
        out = tre.grad_norm(each, max_norm=most)
        assert torch.equal(out, tre.grad_norm(each, max_norm=most))
        norm, factor = out.double().tolist()
        assert abs(norm - want) <= (U + 2.0 ** -45) * want
        ref = 1.0 if most is None else min(1.0, float(np.float32(most)) / (want + 1e-6))
        assert abs(factor - ref) <= (U + 2.0 ** -45) * ref


@pytest.mark.parametrize("value", [1e30, math.inf, math.nan, 3e38])
def test_norm_of_large_values(value):
    import torch

    import paper_2603_08957_amd as tre

    each = [torch.ones(100, device="cuda"), torch.full((2,), value, device="cuda")]
    norm, factor = tre.grad_norm(each, max_norm=1.0).tolist()
    want = math.sqrt(2) * float(np.float32(value))
    if want <= float(np.finfo(np.float32).max):
        assert abs(norm - want) <= 2 * U * want and abs(factor * want - 1) <= 4 * U
    else:
        assert not math.isfinite(norm) and math.isnan(factor)


def test_no_step_after_a_norm_that_is_not_finite():
    import torch

    import paper_2603_08957_amd as tre

    params = [torch.randn(1000, device="cuda"), torch.randn(50, 3, device="cuda").bfloat16()]
    grads = [torch.randn(1000, device="cuda"), torch.randn(50, 3, device="cuda")]
    for bits in (8, 32):
        state = tre.adamw_state(params, bits)
        tre.adamw(params, grads, state, 1, 1e-2, grad_scale=tre.grad_norm(grads, 1.0)[1:])
        was = [t.clone() for t in (*params, state)]
        bad = [grads[0].clone(), grads[1]]
        bad[0][7] = math.inf
        tre.adamw(params, bad, state, 2, 1e-2, grad_scale=tre.grad_norm(bad, 1.0)[1:])
        assert all(torch.equal(a, b) for a, b in zip(was, (*params, state)))


def test_streams_and_graphs():
    """Clipping and a step captured once and replayed: the step's number, rate and gradients are the replay's own."""
    import torch

    import paper_2603_08957_amd as tre

    torch.manual_seed(1)
    shapes = [(300, 40), (17,), (4096,), (5, 5, 5)]
    for bits, seed in ((32, None), (8, None), (8, 9)):
        params = [torch.randn(s, device="cuda") for s in shapes]
        twin = [p.clone() for p in params]
        grads = [torch.zeros(s, device="cuda") for s in shapes]
        state, tstate = tre.adamw_state(params, bits), tre.adamw_state(twin, bits)
        step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step += 1
            clip = tre.grad_norm(grads, 1.0)
            tre.adamw(params, grads, state, step, lr, weight_decay=0.1, grad_scale=clip[1:], seed=seed)
        step.zero_()
        s = torch.cuda.Stream()
        for t in range(1, 5):
            for g in grads:
                g.copy_(torch.randn_like(g))
            lr.fill_(1e-2 / t)
            graph.replay()
            s.wait_stream(torch.cuda.current_stream())
            c = tre.grad_norm(grads, 1.0, stream=s)
            # (the host's step and rate: the same but for the rate's rounding, so the device's is taken)
            tre.adamw(twin, grads, tstate, t, lr, weight_decay=0.1, grad_scale=c[1:], seed=seed, stream=s)
            torch.cuda.current_stream().wait_stream(s)
            torch.cuda.synchronize()
            assert torch.equal(state, tstate) and step.item() == t
            for p, q in zip(params, twin):
                assert (p - q).abs().max() <= 8 * U * q.abs().max()
                p.copy_(q)


def test_refusals():
    import torch

    import paper_2603_08957_amd as tre

    def refused(status, f, *a, **kw):
        with pytest.raises(tre.TreError) as e:
            f(*a, **kw)
        assert e.value.status == status

    p, g = [torch.zeros(40, 3, device="cuda")], [torch.zeros(40, 3, device="cuda")]
    state = tre.adamw_state(p)
    refused("TRE_E_SHAPE", tre.adamw, p, [g[0].view(3, 40)], state, 1, 1e-3)
    refused("TRE_E_SHAPE", tre.adamw, p, g + g, state, 1, 1e-3)
    refused("TRE_E_SHAPE", tre.adamw, p, [g[0].view(3, 40).T], state, 1, 1e-3)
    refused("TRE_E_SHAPE", tre.adamw, p, g, state[:-64], 1, 1e-3)
    refused("TRE_E_DTYPE", tre.adamw, p, g, state.double(), 1, 1e-3)
    refused("TRE_E_DTYPE", tre.adamw, [p[0].double()], g, state, 1, 1e-3)
    refused("TRE_E_DTYPE", tre.adamw, p, g, state, torch.ones(1, device="cuda"), 1e-3)
    refused("TRE_E_SHAPE", tre.adamw, p, g, state, torch.ones(2, dtype=torch.int64, device="cuda"), 1e-3)
    refused("TRE_E_ARG", tre.adamw, p, g, state, torch.ones(1, dtype=torch.int64), 1e-3)
    refused("TRE_E_ARG", tre.adamw, p, [g[0].cpu()], state, 1, 1e-3)
    refused("TRE_E_ARG", tre.adamw, p, g, state, 0, 1e-3)
    refused("TRE_E_ARG", tre.adamw, p + p, g + g, tre.adamw_state(p + g), 1, 1e-3)
    refused("TRE_E_ARG", tre.adamw, p, [None], state, 1, 1e-3)
    refused("TRE_E_ARG", tre.adamw_state, p, 16)
    refused("TRE_E_SHAPE", tre.grad_norm, [p[0].T])
    refused("TRE_E_DTYPE", tre.grad_norm, [p[0].half()])
    refused("TRE_E_WORKSPACE", tre.grad_norm, p, ws=torch.empty(256, dtype=torch.uint8, device="cuda")[:8])
    refused("TRE_E_SHAPE", tre.adamw_moments, torch.zeros(65, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("bits,seed", [(32, None), (8, None), (8, 1)])
def test_a_table_is_trained(bits, seed):
    """Rows, scores, loss, gradients, clipping and a step, as a program that trains a table runs them; the first step's gradient of
    the table against float64's (bounds: the scores' sums of 32 terms, then 200 or 30 more)."""
    import torch

    import paper_2603_08957_amd as tre

    n, vocab, d, tile = 30, 200, 32, 20
    torch.manual_seed(2)
    table = torch.randn(vocab, d, device="cuda") / 4
    ids, words = (torch.randint(0, vocab, (n,), device="cuda") for _ in range(2))
    ext, til = {"v": vocab, "n": n, "d": d}, {"v": tile}
    scores = tre.Plan("nd,vd->nv", "v", ext, til, "f32")
    by_x, by_w = tre.Plan("nv,vd->nd", "v", ext, til, "f32"), tre.Plan("nv,nd->vd", "v", ext, til, "f32")
    keys = torch.arange(vocab // tile, dtype=torch.int32, device="cuda").view(-1, 1)
    state = tre.adamw_state([table], bits)
    start = table.double().cpu()
    for t in range(1, 4):
        x = tre.lookup(table, ids)
        w = table.view(vocab // tile, -1)
        tiles = tre.einsum(scores, None, x.view(1, -1), keys, w).w_tiles.view(-1, n, tile)
        r = tre.log_probs(tiles, words)
        dy = tre.log_probs_grad(tiles, r.stats, words, torch.full((n,), -1.0 / n, device="cuda")).view(vocab // tile, -1)
        dx = tre.einsum(by_x, keys, dy, keys, w).w_tiles.view(n, d)
        grad = tre.einsum(by_w, keys, dy, None, x.view(1, -1)).w_tiles.view(vocab, d)
        tre.lookup_grad(dx, ids, vocab, out=grad, accumulate=True)
        if t == 1:
            ref = start.clone().requires_grad_()
            rows = ref[ids.cpu()]
            loss = -torch.log_softmax(rows @ ref.T, 1)[torch.arange(n), words.cpu()].mean()
            loss.backward()
            z = float((rows.detach().abs() @ start.abs().T).max())
            rel = 2 * (33 * U * z) + (vocab + 60) * U + (vocab + n + 40) * U
            p = torch.softmax(rows.detach() @ start.T, 1) / n
            size = p + torch.nn.functional.one_hot(words.cpu(), vocab) / n
            bound = size.T @ rows.detach().abs()
            bound = bound.index_add(0, ids.cpu(), size @ start.abs())
            assert ((grad.cpu().double() - ref.grad).abs() <= 2 * rel * bound + U).all()
            assert (r.log_prob.double().mean().cpu() + loss.detach()).abs() <= rel + 8 * U * 10
        before = table.clone()
        tre.adamw([table], [grad], state, t, 1e-2, weight_decay=0.01, grad_scale=tre.grad_norm([grad], 1.0)[1:], seed=seed)
        assert not torch.equal(before, table) and table.isfinite().all()
