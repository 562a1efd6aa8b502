"""Timed cases of the operators at the end of a model held as tile relations:
what it answers with, the gradient that goes back into it, and the step that
its weights take.

  log_probs       of scores, as rows or as the tiles of a score EinSum: log
                  probabilities of given tokens, log of the sum, entropy and top
                  alternatives (`log_probs`)
  log_probs_grad  the gradient of these by the scores (`log_probs_grad`)
  grad_norm       the norm of many tensors together and the factor that clips
                  it (`grad_norm`)
  adamw           one AdamW step over many tensors, the moments in 32 or 8 bits
                  (`adamw`), and 8-bit moments read back (`adamw_moments`)

8-bit moments: blocks of 32 consecutive elements of a tensor share a power of
two 2^e, e = floor(log2 of the largest) - 7 (at least -127), stored as the byte
e + 127.  Times it, the first moment is a sign and a 7-bit code c, the second an
8-bit code c, of which c / 8 = E is the exponent and c % 8 = f the fraction:
(1 + f / 8) 2^(E - bias), or f / 8 2^(1 - bias) for E = 0, with bias 7 and 23.
They are rounded to the nearest code (ties to the even one) or, with a seed, up
with the probability that the place between two codes has; a second moment that
is not zero takes code 1 at least.  A tensor's moments begin at a multiple of 32
elements; the buffer holds all first moments' codes, all second ones', then the
bytes e + 127 of both.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def listed():
    return [
        # one decoding step: the next token's log probability and alternatives out of the score tiles
        {"name": "answer_1", "kind": "logp", "n": 1, "vocab": 32768, "tile": 128, "hidden": 0, "dtype": "f32", "top": 20,
         "entropy": False, "scale": 1.0, "pad": 0.0},
        # a small served batch; vocabulary and tiles as they come, the last columns no words, a temperature
        {"name": "answer_13_ragged", "kind": "logp", "n": 13, "vocab": 50250, "tile": 250, "hidden": 193, "dtype": "f32", "top": 5,
         "entropy": True, "scale": 1.25, "pad": 0.0},
        # given texts scored, with alternatives for every token
        {"name": "score_2048_top", "kind": "logp", "n": 2048, "vocab": 32768, "tile": 128, "hidden": 0, "dtype": "bf16", "top": 8,
         "entropy": False, "scale": 1.0, "pad": 0.0},
        # the loss of a training batch, padded
        {"name": "loss_8192_bf16", "kind": "logp", "n": 8192, "vocab": 32768, "tile": 0, "hidden": 0, "dtype": "bf16", "top": 0,
         "entropy": True, "scale": 1.0, "pad": 0.1},
        # the gradient of a few short sequences by the score tiles
        {"name": "loss_grad_512_f32", "kind": "logp_grad", "n": 512, "vocab": 4096, "tile": 128, "hidden": 0, "dtype": "f32",
         "out": "f32", "entropy": False, "lse": False, "scale": 1.0, "pad": 0.0},
        # the gradient of a padded training batch, entropy and the log of the sum in its loss
        {"name": "loss_grad_8192_bf16", "kind": "logp_grad", "n": 8192, "vocab": 32768, "tile": 128, "hidden": 0, "dtype": "bf16",
         "out": "bf16", "entropy": True, "lse": True, "scale": 1.0, "pad": 0.1},
        # the gradients of a small model's layers
        {"name": "norm_60_small", "kind": "norm", "tensors": 60, "total": 300000, "mix": 1, "dtype": "f32", "clip": 1.0},
        # the gradients of a large model
        {"name": "norm_300_large", "kind": "norm", "tensors": 300, "total": 400000000, "mix": 2, "dtype": "bf16", "clip": 1.0},
        # the smallest step: a small model's layers
        {"name": "adamw_60_small", "kind": "adamw", "tensors": 60, "total": 300000, "mix": 1, "param": "f32", "grad": "f32",
         "bits": 32, "seed": -1, "step": 10, "device": False},
        # a large model's step as it is usual: everything in fp32
        {"name": "adamw_134m_f32", "kind": "adamw", "tensors": 200, "total": 134000000, "mix": 3, "param": "f32", "grad": "f32",
         "bits": 32, "seed": -1, "step": 1000, "device": False},
        # the same with moments in 8 bits, step and rate on the device
        {"name": "adamw_67m_8bit", "kind": "adamw", "tensors": 100, "total": 67000000, "mix": 4, "param": "f32", "grad": "bf16",
         "bits": 8, "seed": -1, "step": 1000, "device": True},
        # everything short: bf16 weights and 8-bit moments, both rounded by chance
        {"name": "adamw_67m_short", "kind": "adamw", "tensors": 333, "total": 67000000, "mix": 5, "param": "bf16", "grad": "bf16",
         "bits": 8, "seed": 77, "step": 3, "device": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logp", "logp", "logp_grad", "norm", "adamw", "adamw"])
    if kind in ("logp", "logp_grad"):
        cols = rng.choice([0, 128, 250, _log(rng, 8, 400)])
        vocab = _log(rng, 100, 60000)
        vocab = cols * max(1, vocab // cols) if cols else vocab
        case = {"kind": kind, "n": _log(rng, 1, min(8192, 200000000 // vocab)), "vocab": vocab, "tile": cols,
                "hidden": rng.choice([0, rng.randrange(vocab // 4)]), "dtype": rng.choice(["f32", "bf16"])}
        if kind == "logp":
            case["top"] = rng.choice([0, 1, rng.randint(2, 64)])
            case["n"] = min(case["n"], 60000000 // vocab) if case["top"] else case["n"]
        else:
            case["out"], case["lse"] = rng.choice(["f32", "bf16"]), rng.choice([False, True])
        return {**case, "entropy": rng.choice([False, True]), "scale": rng.choice([1.0, rng.uniform(0.5, 2.0)]),
                "pad": rng.choice([0.0, 0.1])}
    tensors = _log(rng, 1, 400)
    if kind == "norm":
        return {"kind": kind, "tensors": tensors, "total": _log(rng, 2000, 300000000), "mix": rng.randrange(1 << 20),
                "dtype": rng.choice(["f32", "bf16"]), "clip": rng.choice([0.5, 1e6])}
    bits = rng.choice([32, 8])
    return {"kind": kind, "tensors": tensors, "total": _log(rng, 2000, 100000000 if bits == 32 else 50000000),
            "mix": rng.randrange(1 << 20), "param": rng.choice(["f32", "bf16"]), "grad": rng.choice(["f32", "bf16"]),
            "bits": bits, "seed": rng.choice([-1, rng.randrange(1 << 40)]), "step": _log(rng, 1, 100000),
            "device": rng.choice([False, True])}


# ------------------------------------------------------------------ inputs

_TYPE = {"f32": F32, "bf16": BF16}
_SIZE = {"f32": 4, "bf16": 2}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rows(x):
    """Tiles [tiles, n, cols] as rows [n, vocab]."""
    return x if x.dim() == 2 else x.transpose(0, 1).reshape(x.shape[1], -1)


def _tiles(c, y):
    """Rows [n, vocab] in the layout of the case's scores."""
    return y.view(c["n"], -1, c["tile"]).transpose(0, 1).contiguous() if c["tile"] else y


def _scores(c, g):
    """Scores of a spread that a trained model's have, the hidden words' -inf."""
    shape = (c["vocab"] // c["tile"], c["n"], c["tile"]) if c["tile"] else (c["n"], c["vocab"])
    x = torch.randn(shape, generator=g, device=DEV, dtype=F32).mul_(2.5)
    if c["hidden"]:
        first = c["vocab"] - c["hidden"]
        word = torch.arange(c["vocab"], device=DEV)
        x.masked_fill_(word.view(-1, 1, c["tile"]) >= first if c["tile"] else word >= first, -math.inf)
    return x.to(_TYPE[c["dtype"]])


def _tokens(c, g):
    """Tokens of which the k-th most frequent comes about 1 / k as often as the
    first; a share `pad` of them is -1 (no token)."""
    words = c["vocab"] - c["hidden"]
    u = torch.rand((c["n"],), generator=g, device=DEV, dtype=F64)
    ids = (float(words + 1) ** u).long().sub_(1).clamp_(0, words - 1)
    if c["pad"]:
        ids[torch.rand((c["n"],), generator=g, device=DEV) < c["pad"]] = -1
    return ids


def _sizes(c):
    """Elements of each tensor: a few large ones and many small, odd numbers of them."""
    r = random.Random(c["mix"])
    w = [math.exp(r.gauss(0.0, 1.5)) for _ in range(c["tensors"])]
    return [max(1, int(c["total"] * x / sum(w))) for x in w]


def _room(n):
    return (n + 31) // 32 * 32


class _Many:
    """Tensors of these sizes, each beginning at a multiple of 32 elements of one
    buffer, with zeros between."""

    def __init__(self, sizes, dtype, g, spread):
        at, self.total = [], 0
        for n in sizes:
            at.append(self.total)
            self.total += _room(n)
        self.flat = torch.randn((self.total,), generator=g, device=DEV, dtype=F32).mul_(spread).to(dtype)
        ends = torch.tensor([a + n for a, n in zip(at, sizes)], device=DEV)
        gap = ends[:, None] + torch.arange(32, device=DEV)
        limit = torch.tensor(at[1:] + [self.total], device=DEV)
        self.flat[gap[gap < limit[:, None]]] = 0
        self.each = [self.flat[a:a + n] for a, n in zip(at, sizes)]


# ---------------------------------------------------------------- log_probs

def _logp_inputs(c, seed):
    g = _gen(seed)
    return _scores(c, g), _tokens(c, g)


def _logp_prepare(c, seed):
    x, ids = _logp_inputs(c, seed)
    return {"c": c, "x": x, "ids": ids}


def _logp_run(s):
    c, ids = s["c"], s["ids"]
    if own:
        import paper_2603_08957_amd as tre

        r = tre.log_probs(s["x"], ids, scale=c["scale"], top=c["top"], entropy=c["entropy"])
        out = {"log_prob": r.log_prob, "lse": r.lse, "stats": r.stats}
        if c["entropy"]:
            out["entropy"] = r.entropy
        if c["top"]:
            out["top_ids"], out["top_log_probs"] = r.top_ids, r.top_log_probs
        return out
    x = _rows(s["x"]).float()
    m = x.amax(1, keepdim=True)
    d = (x - m) * c["scale"]
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    logs = torch.log(total)
    out = {"log_prob": torch.where(ids >= 0, (d.gather(1, ids.clamp_min(0)[:, None]) - logs)[:, 0], 0.0),
           "lse": (m * c["scale"] + logs)[:, 0], "stats": torch.cat([m, logs], 1)}
    if c["entropy"]:
        out["entropy"] = (logs - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total)[:, 0]
    if c["top"]:
        # the order of the values, and of places among equal ones, as one whole number
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -2147483648 - bits, bits) * 4294967296 - torch.arange(c["vocab"], device=DEV)
        at = -(order.topk(c["top"], 1)[0] % -4294967296)
        out["top_ids"], out["top_log_probs"] = at.int(), d.gather(1, at) - logs
    return out


def _logp_exact(c, seed):
    x, ids = _logp_inputs(c, seed)
    z = _rows(x).double() * c["scale"]
    lse = torch.logsumexp(z, 1)
    top = _rows(x).amax(1).double()
    out = {"log_prob": torch.where(ids >= 0, z[torch.arange(c["n"], device=DEV), ids.clamp_min(0)] - lse, 0.0), "lse": lse,
           "stats": torch.stack([top, lse - top * c["scale"]], 1)}
    z -= lse[:, None]
    if c["top"]:
        out["top_ids"], out["top_log_probs"] = None, z.topk(c["top"], 1)[0]
    if c["entropy"]:
        out["entropy"] = -(torch.exp(z) * z.clamp_min(-1e4)).sum(1)
    return out


def _logp_work(c):
    n = c["n"] * c["vocab"]
    return {"bytes": n * _SIZE[c["dtype"]] + c["n"] * (8 + 16 + 4 * c["entropy"] + 8 * c["top"]),
            "flops": n * (5 + 2 * c["entropy"])}


# ----------------------------------------------------------- log_probs_grad

def _logp_grad_inputs(c, seed):
    g = _gen(seed)
    x, ids = _scores(c, g), _tokens(c, g)
    grads = torch.randn((3, c["n"]), generator=g, device=DEV, dtype=F32) / c["n"]
    keep = (ids >= 0).float()  # (a padded row has no part in the loss)
    return x, ids, grads[0] * keep, grads[1] * keep if c["lse"] else None, grads[2] * keep if c["entropy"] else None


def _logp_grad_prepare(c, seed):
    x, ids, g, gl, gh = _logp_grad_inputs(c, seed)
    # what the forward pass left
    z = _rows(x).double()
    m = z.amax(1)
    z = z.sub_(m[:, None]).mul_(c["scale"])
    logs = torch.logsumexp(z, 1)
    z = z.sub_(logs[:, None]).clamp_min_(-1e4)
    s = {"c": c, "x": x, "ids": ids, "g": g, "gl": gl, "gh": gh, "stats": torch.stack([m, logs], 1).float()}
    s["entropy"] = -(torch.exp(z).mul_(z)).sum(1).float() if c["entropy"] else None
    return s


def _logp_grad_run(s):
    c, ids = s["c"], s["ids"]
    if own:
        import paper_2603_08957_amd as tre

        return tre.log_probs_grad(s["x"], s["stats"], ids, grad_log_prob=s["g"], grad_lse=s["gl"], grad_entropy=s["gh"],
                                  entropy=s["entropy"], scale=c["scale"], dtype=_TYPE[c["out"]])
    x = _rows(s["x"]).float()
    lp = (x - s["stats"][:, :1]) * c["scale"] - s["stats"][:, 1:]
    p = torch.exp(lp)
    dz = p * ((s["gl"] if c["lse"] else 0.0) - s["g"])[:, None]
    if c["entropy"]:
        dz -= torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0) * s["gh"][:, None]
    dz.scatter_add_(1, ids.clamp_min(0)[:, None], torch.where(ids >= 0, s["g"], 0.0)[:, None])
    return _tiles(c, (dz * c["scale"]).to(_TYPE[c["out"]]))


def _logp_grad_exact(c, seed):
    x, ids, g, gl, gh = _logp_grad_inputs(c, seed)
    lp = torch.log_softmax(_rows(x).double() * c["scale"], 1)
    p = torch.exp(lp)
    dz = -p * g[:, None].double()
    rows = (ids >= 0).nonzero()[:, 0]
    dz[rows, ids[rows]] += g[rows].double()
    if gl is not None:
        dz += p * gl[:, None]
    if gh is not None:
        lp.clamp_min_(-1e4)
        h = -(p * lp).sum(1, keepdim=True)
        dz -= gh[:, None] * p * (lp + h)
    return _tiles(c, dz * c["scale"])


def _logp_grad_work(c):
    n = c["n"] * c["vocab"]
    return {"bytes": n * ((1 - c["pad"]) * _SIZE[c["dtype"]] + _SIZE[c["out"]]) + c["n"] * (20 + 4 * c["lse"] + 8 * c["entropy"]),
            "flops": n * (5 + 2 * c["entropy"])}


# ---------------------------------------------------------------- grad_norm

def _norm_prepare(c, seed):
    many = _Many(_sizes(c), _TYPE[c["dtype"]], _gen(seed), 1e-3)
    return {"c": c, "flat": many.flat, "each": many.each}


def _norm_run(s):
    c = s["c"]
    if own:
        import paper_2603_08957_amd as tre

        return tre.grad_norm(s["each"], max_norm=c["clip"])
    norm = s["flat"].double().square().sum().sqrt()
    return torch.stack([norm, (c["clip"] / (norm + 1e-6)).clamp_max(1.0)]).float()


def _norm_exact(c, seed):
    norm = torch.linalg.vector_norm(_Many(_sizes(c), _TYPE[c["dtype"]], _gen(seed), 1e-3).flat, dtype=F64)
    return torch.stack([norm, torch.minimum(c["clip"] / (norm + 1e-6), torch.ones_like(norm))])


def _norm_work(c):
    n = sum(_sizes(c))
    return {"bytes": n * _SIZE[c["dtype"]] + 8, "flops": 2 * n}


# -------------------------------------------------------------------- adamw

B1, B2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 3e-4, 0.1
_W = 0xFFFFFFFF


def _chance(n, seed, step):
    """20, 20 and 16 random bits of each of n elements: a hash of (seed, step,
    element), three rounds of shifts and products in 32 bits."""
    i = torch.arange(n, device=DEV, dtype=torch.int64)
    k0 = ((seed & _W) + step * 0x9E3779B1) & _W
    h = (((i & _W) ^ k0) * 0x6A09E667) & _W
    h ^= h >> 15
    h = (h + (seed >> 32 & _W) + (i >> 32) * 0xBB67AE85) & _W
    h = (h * 0xBB67AE85) & _W
    h ^= h >> 13
    y = (h * 0x3C6EF373) & _W
    y ^= y >> 16
    return h >> 12, y >> 12, (h ^ (y << 4)) & 0xFFFF


def _two_to(e):
    """2^e of whole numbers from -127 to 127, exactly."""
    return torch.where(e > -127, e + 127 << 23, 1 << 22).int().view(F32)


def _encode(x, bias, chance):
    """Codes of the magnitudes of x [blocks, 32] and the bytes of the blocks' powers of two."""
    a = x.abs()
    byte = ((a.amax(1).view(torch.int32) >> 23) - 7).clamp_min(0)
    y = a * _two_to(127 - byte)[:, None]
    u = y.view(torch.int32)
    low = (y * 2.0 ** (bias + 2)).clamp_max(8.0)  # in steps of the codes below 8
    if chance is None:
        high = (u + 0x7FFFF + (u >> 20 & 1)) >> 20
        low = torch.round(low).int()
    else:
        r = chance.view(-1, 32).int()
        high = (u + r) >> 20
        low = ((low * 2.0 ** 20).int() + r) >> 20
    return torch.where(y >= 2.0 ** (1 - bias), high - ((127 - bias) << 3), low), byte


def _decode(code, byte, bias):
    c = code.view(-1, 32).int()
    e, f = c >> 3, (c & 7).float()
    y = torch.where(e > 0, (1 + f / 8) * _two_to(e - bias), f * 2.0 ** (-2 - bias))
    return (y * _two_to(byte.int() - 127)[:, None]).view(-1)


def _moments_of(state):
    n = state.numel() * 16 // 33
    q, q2, b, b2 = state.split([n, n, n // 32, n // 32])
    m = _decode(q & 127, b, 7)
    return torch.where(q > 127, -m, m), _decode(q2, b2, 23)


def _state_of(m, v, chance):
    rm, rv = chance[:2] if chance else (None, None)
    cm, bm = _encode(m.view(-1, 32), 7, rm)
    cv, bv = _encode(v.view(-1, 32), 23, rv)
    cv = torch.where(v.view(-1, 32) > 0, cv.clamp_min(1), cv)
    cm = cm + torch.where(m.view(-1, 32) < 0, 128, 0)
    return torch.cat([t.reshape(-1).to(torch.uint8) for t in (cm, cv, bm, bv)])


def _adamw_inputs(c, seed):
    """Weights, gradients and the moments that earlier steps left, in 32 bits."""
    g = _gen(seed)
    sizes = _sizes(c)
    p, grad = _Many(sizes, _TYPE[c["param"]], g, 0.02), _Many(sizes, _TYPE[c["grad"]], g, 1e-3)
    live = (grad.flat != 0).float()
    m = torch.randn((p.total,), generator=g, device=DEV, dtype=F32).mul_(3e-4) * live
    v = torch.rand((p.total,), generator=g, device=DEV, dtype=F32).add_(0.2).mul_(1e-6) * live
    factor = torch.full((1,), 0.7310586, device=DEV)  # as clipping gives it
    return p, grad, m, v, factor


def _adamw_prepare(c, seed):
    p, grad, m, v, factor = _adamw_inputs(c, seed)
    s = {"c": c, "p": p.flat, "params": p.each, "g": grad.flat, "grads": grad.each, "k": factor,
         "state": torch.cat([m, v]) if c["bits"] == 32 else _state_of(m, v, None), "step": c["step"], "lr": LR}
    if c["device"]:
        s["step"], s["lr"] = torch.tensor([c["step"]], device=DEV), torch.tensor([LR], device=DEV)
    return s


def _adamw_run(s):
    c, state = s["c"], s["state"]
    short = c["bits"] == 8
    if own:
        import paper_2603_08957_amd as tre

        tre.adamw(s["params"], s["grads"], state, s["step"], s["lr"], beta1=B1, beta2=B2, eps=EPS, weight_decay=DECAY,
                  grad_scale=s["k"], seed=c["seed"] if c["seed"] >= 0 else None)
        m, v = tre.adamw_moments(state, dtype=BF16) if short else state.chunk(2)
        return {"p": s["p"], "m": m, "v": v}
    chance = _chance(state.numel() * 16 // 33 if short else state.numel() // 2, c["seed"], c["step"]) if c["seed"] >= 0 else None
    m, v = _moments_of(state) if short else state.chunk(2)
    g = s["g"].float() * s["k"]
    m = m * B1 + g * (1 - B1)
    v = v * B2 + g * g * (1 - B2)
    lr = s["lr"]
    if c["device"]:
        c1, c2 = ((1 - torch.exp(s["step"].double() * math.log(b))).float() for b in (B1, B2))
    else:
        c1, c2 = 1 - B1 ** c["step"], 1 - B2 ** c["step"]
    p = s["p"].float() * (1 - lr * DECAY) - lr * (m / c1) / ((v / c2).sqrt() + EPS)
    if chance and c["param"] == "bf16":
        p = ((p.view(torch.int32) + chance[2].int()) >> 16 << 16).view(F32)
    s["p"].copy_(p)
    state.copy_(_state_of(m, v, chance) if short else torch.cat([m, v]))
    m, v = _moments_of(state) if short else state.chunk(2)
    return {"p": s["p"], "m": m.to(BF16) if short else m, "v": v.to(BF16) if short else v}


def _exact_8bit(x, bias, chance):
    """The values that 8-bit codes keep of magnitudes x, in 64 bits."""
    b = x.view(-1, 32)
    top = b.amax(1, keepdim=True)
    unit = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 7)
    y = b / unit
    step = torch.exp2(torch.floor(torch.log2(y.clamp_min(2.0 ** (1 - bias)))) - 3)
    q = torch.round(y / step) if chance is None else torch.floor(y / step + chance.view(-1, 32) * 2.0 ** -20)
    return (q * step * unit).view(-1), (step * unit).view(-1)


def _adamw_exact(c, seed):
    p, grad, m, v, factor = _adamw_inputs(c, seed)
    chance = _chance(p.total, c["seed"], c["step"]) if c["seed"] >= 0 else (None, None, None)
    short = c["bits"] == 8
    m, v = m.double(), v.double()

    def least(v, chance):  # second moments do not go to zero
        kept, step = _exact_8bit(v, 23, chance)
        return torch.where(v > 0, torch.maximum(kept, step), kept)

    if short:  # (what earlier steps left was kept in 8 bits too)
        m, v = _exact_8bit(m.abs(), 7, None)[0] * m.sign(), least(v, None)
    g = grad.flat.double() * factor.double()
    m = B1 * m + (1 - B1) * g
    v = B2 * v + (1 - B2) * g ** 2
    lr = float(torch.tensor(LR, dtype=F32)) if c["device"] else LR
    w = p.flat.double()
    w -= lr * DECAY * w + lr * (m / (1 - B1 ** c["step"])) / (torch.sqrt(v / (1 - B2 ** c["step"])) + EPS)
    if short:
        m, v = _exact_8bit(m.abs(), 7, chance[0])[0] * m.sign(), least(v, chance[1])
    return {"p": w, "m": m, "v": v}


def _adamw_work(c):
    n = sum(_sizes(c))
    moments = 16 if c["bits"] == 32 else 4 * 33 / 32 + 2 * 33 / 32 + 4  # (read and written; 8 bits: and read back in bf16)
    return {"bytes": n * (2 * _SIZE[c["param"]] + _SIZE[c["grad"]] + moments), "flops": 15 * n}


# ------------------------------------------------------------------------

_KINDS = {
    "logp": (_logp_prepare, _logp_run, _logp_exact, _logp_work),
    "logp_grad": (_logp_grad_prepare, _logp_grad_run, _logp_grad_exact, _logp_grad_work),
    "norm": (_norm_prepare, _norm_run, _norm_exact, _norm_work),
    "adamw": (_adamw_prepare, _adamw_run, _adamw_exact, _adamw_work),
}


def prepare(case, seed):
    return _KINDS[case["kind"]][0](case, seed)


def run(state):
    return _KINDS[state["c"]["kind"]][1](state)


def exact(case, seed):
    return _KINDS[case["kind"]][2](case, seed)


def work(case):
    return _KINDS[case["kind"]][3](case)
