"""Timed cases of the 4-bit tile and table operators: what a program that
trains or serves a model held as tile relations calls, over the range of sizes,
layouts and types it calls them with.

  round        tiles quantised to microscaled 4-bit blocks (`mx_quantize`) and
               read back (`mx_dequantize`): activations, weights, graph tiles
  token        the scores of a few rows against a table of 4-bit tiles, as one
               decoding step has them: rows quantised, then one EinSum
  blocks       block-sparse times dense matrix, both in 4-bit tiles
  dense        a large dense product, the rows quantised in the call
  train        a linear layer's step in 4-bit tiles: product and both
               gradients, every operand quantised along what it contracts
  lookup       rows of a table by token (`lookup`), scaled; the table in fp32,
               bf16 or 4-bit tiles
  lookup_grad  the table's gradient, rows summed by token (`lookup_grad`)

A 4-bit block is 32 consecutive values along the contracted labels that share
a power of two, 2^(floor(log2 max) - 2), and are rounded to the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times it (ties to the even code, 6 at most).
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def listed():
    return [
        # a weight matrix taken into 4 bits, contracted label last
        {"name": "quantize_rows_bf16", "kind": "round", "tiles": 64, "rows": 256, "k": 8192, "order": "rk", "dtype": "bf16"},
        # many tiles of a graph's adjacency or of a layer off the 32 grid, the contracted label first
        {"name": "quantize_columns_f32", "kind": "round", "tiles": 2000, "rows": 96, "k": 100, "order": "kr", "dtype": "f32"},
        # one decoding step: the scores of one token over the vocabulary
        {"name": "token_1", "kind": "token", "n": 1, "vocab": 32768, "d": 4096, "tile": 128},
        # a small served batch; widths and vocabulary as they come
        {"name": "token_13_ragged", "kind": "token", "n": 13, "vocab": 50250, "d": 1000, "tile": 250},
        # 5% dense 128-blocks times a wide dense matrix
        {"name": "blocks_16384", "kind": "blocks", "n": 16384, "cols": 1024, "block": 128, "density": 0.05},
        # the largest product: a long prompt through a wide layer
        {"name": "dense_8192", "kind": "dense", "n": 8192, "d": 8192, "v": 8192, "tile": 256},
        # a training step of one layer
        {"name": "train_4096", "kind": "train", "n": 4096, "d": 2048, "v": 8192, "tile": 256},
        # the smallest call: the next token of a few sequences
        {"name": "lookup_8_f32", "kind": "lookup", "n": 8, "vocab": 4096, "d": 767, "table": "f32", "out": "f32", "pad": 0.0},
        # the tokens of a training batch, padded
        {"name": "lookup_131072_bf16", "kind": "lookup", "n": 131072, "vocab": 32768, "d": 4096, "table": "bf16",
         "out": "bf16", "pad": 0.1},
        # a prompt's rows out of the 4-bit tiles that the scores are taken against too
        {"name": "lookup_8192_mxfp4", "kind": "lookup", "n": 8192, "vocab": 32768, "d": 4096, "table": "mxfp4", "tile": 128,
         "out": "bf16", "pad": 0.0},
        # the gradient of a few short sequences: many launches against little data
        {"name": "lookup_grad_512_f32", "kind": "lookup_grad", "n": 512, "vocab": 4096, "d": 767, "grad": "f32", "out": "f32",
         "pad": 0.0},
        # a training batch: some tokens make up a tenth of it, most come once or never
        {"name": "lookup_grad_65536_bf16", "kind": "lookup_grad", "n": 65536, "vocab": 32768, "d": 4096, "grad": "bf16",
         "out": "f32", "pad": 0.1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["round", "token", "blocks", "dense", "train", "lookup", "lookup_grad"])
    if kind == "round":
        rows, k = _log(rng, 1, 300), _log(rng, 1, 8192)
        return {"kind": kind, "tiles": max(1, _log(rng, 1000, 100000000) // (rows * k)), "rows": rows, "k": k,
                "order": rng.choice(["rk", "kr"]), "dtype": rng.choice(["f32", "bf16"])}
    if kind == "token":
        tile = rng.choice([16, 64, 128, 256, _log(rng, 10, 300)])
        return {"kind": kind, "n": _log(rng, 1, 64), "vocab": tile * _log(rng, 4, max(5, 100000 // tile)),
                "d": rng.choice([64, 512, 2048, _log(rng, 17, 4096)]), "tile": tile}
    if kind == "blocks":
        block = rng.choice([64, 128, _log(rng, 17, 200)])
        return {"kind": kind, "n": block * _log(rng, 8, 100), "cols": rng.choice([128, 512, _log(rng, 17, 1100)]),
                "block": block, "density": rng.uniform(0.02, 0.15)}
    if kind == "dense":
        tile = rng.choice([64, 128, 256, _log(rng, 17, 300)])
        return {"kind": kind, "n": tile * _log(rng, 1, max(2, 4000 // tile)), "d": _log(rng, 32, 6000),
                "v": tile * _log(rng, 1, max(2, 6000 // tile)), "tile": tile}
    if kind == "train":
        tile = rng.choice([64, 128, 256, _log(rng, 30, 300)])
        return {"kind": kind, "n": tile * _log(rng, 1, max(2, 3000 // tile)), "d": _log(rng, 32, 3000),
                "v": tile * _log(rng, 1, max(2, 4000 // tile)), "tile": tile}
    n, d = _log(rng, 1, 60000), _log(rng, 8, 4096)
    vocab = _log(rng, 100, 60000)
    if kind == "lookup":
        table = rng.choice(["f32", "bf16", "mxfp4"])
        case = {"kind": kind, "n": n, "vocab": vocab, "d": d, "table": table, "out": rng.choice(["f32", "bf16"]),
                "pad": rng.choice([0.0, 0.1])}
        if table == "mxfp4":
            case["tile"] = _log(rng, 1, 256)
            case["vocab"] = case["tile"] * max(1, vocab // case["tile"])
        return case
    return {"kind": kind, "n": n, "vocab": vocab, "d": d, "grad": rng.choice(["f32", "bf16"]),
            "out": rng.choice(["f32", "bf16"]), "pad": rng.choice([0.0, 0.1])}


# ------------------------------------------------------------------ inputs

_TYPE = {"f32": F32, "bf16": BF16}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _values(shape, dtype, g, spread=0.0):
    """N(0, 1) values; `spread` > 0: every row of the last dimension has a size
    of its own, as activations have."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=F32)
    if spread:
        x *= torch.exp(spread * torch.randn(shape[:-1] + (1,), generator=g, device=DEV, dtype=F32))
    return x.to(_TYPE[dtype])


def _tokens(c, g):
    """Tokens of which the k-th most frequent comes about 1 / k as often as the
    first; a share `pad` of them is -1 (no token)."""
    u = torch.rand((c["n"],), generator=g, device=DEV, dtype=torch.float64)
    ids = (float(c["vocab"] + 1) ** u).long().sub_(1).clamp_(0, c["vocab"] - 1)
    if c["pad"]:
        ids[torch.rand((c["n"],), generator=g, device=DEV) < c["pad"]] = -1
    return ids


def _keys(*cols):
    return torch.stack(cols, dim=1).to(torch.int32).contiguous()


def _range(n):
    return _keys(torch.arange(n, device=DEV))


def _block_keys(c, g):
    """Keys (i, j) of the non-zero blocks, sorted, one on the diagonal at least."""
    nb = c["n"] // c["block"]
    hit = torch.rand((nb, nb), generator=g, device=DEV) < c["density"]
    hit.fill_diagonal_(True)
    return _keys(*hit.nonzero(as_tuple=True))


# ------------------------------------------------- the plain forms' numbers

def _mx(x):
    """Values of x (any shape, fp32) quantised in blocks of 32 of the last dimension."""
    k = x.shape[-1]
    b = torch.nn.functional.pad(x.float(), (0, -k % 32)).unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(-127, 127)  # frexp: top = m 2^e, 0.5 <= m < 1
    y = torch.ldexp(b, -e)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(y / step) * step).clamp(-6, 6)
    return torch.ldexp(q, e).flatten(-2)[..., :k]


def _mx_t(x):
    """The same in blocks of the dimension before the last."""
    return _mx(x.transpose(-1, -2)).transpose(-1, -2)


def _exact_mx(x):
    """The definition, in 64 bits: the nearest of the eight values times the block's power of two."""
    k = x.shape[-1]
    b = torch.nn.functional.pad(x.double(), (0, -k % 32)).unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    scale = torch.where(top > 0, torch.exp2(torch.floor(torch.log2(top.clamp_min(1e-300))) - 2), torch.ones_like(top))
    y = b / scale
    a = y.abs()
    # halves between neighbours, each belonging to the neighbour whose code is even
    q = torch.zeros_like(a)
    for low, value, closed in ((0.25, 0.5, False), (0.75, 1.0, True), (1.25, 1.5, False), (1.75, 2.0, True),
                               (2.5, 3.0, False), (3.5, 4.0, True), (5.0, 6.0, False)):
        q = torch.where(a >= low if closed else a > low, value, q)
    return (torch.copysign(q, y) * scale).flatten(-2)[..., :k]


def _exact_mx_t(x):
    return _exact_mx(x.transpose(-1, -2)).transpose(-1, -2)


# --------------------------------------------------- own: plans and buffers

class _Call:
    """One EinSum over 4-bit tiles with its workspace and output buffers, kept
    by the program that runs it again and again."""

    def __init__(self, plan, n_u, n_v, pairs, keys):
        import paper_2603_08957_amd as tre

        self.tre, self.plan = tre, plan
        self.ws = tre.alloc_workspace(plan.workspace_bytes(n_u, n_v, pairs))
        _, bound, ok = tre.output_bounds(plan, n_u, n_v, self.ws.numel())
        self.counts = torch.zeros(4, dtype=torch.int64, device=DEV) if ok and bound == keys else None
        self.keys = torch.empty((keys, max(plan.key_arity[2], 1)), dtype=torch.int32, device=DEV)
        self.tiles = torch.empty((keys, plan.tile_elems[2]), dtype=BF16 if plan.w_bf16 else F32, device=DEV)

    def __call__(self, uk, ut, vk, vt):
        if self.counts is not None:
            self.tre.execute_async(self.plan, uk, ut, vk, vt, self.keys, self.tiles, self.ws, self.counts)
        else:
            self.tre.execute(self.plan, uk, ut, vk, vt, self.keys, self.tiles, self.ws)
        return self.keys, self.tiles


# -------------------------------------------------------------------- round

def _round_inputs(c, seed):
    shape = (c["tiles"], c["rows"], c["k"]) if c["order"] == "rk" else (c["tiles"], c["k"], c["rows"])
    return _values(shape, c["dtype"], _gen(seed), 1.0)


def _round_prepare(c, seed):
    s = {"c": c, "x": _round_inputs(c, seed)}
    if own:
        import paper_2603_08957_amd as tre

        u = "ik" if c["order"] == "rk" else "ki"
        s["plan"] = tre.Plan(f"{u},jk->ij", "i", {"i": c["tiles"] * c["rows"], "j": 16, "k": c["k"]}, {"i": c["rows"]},
                             "mxfp4")
    return s


def _round_run(s):
    x = s["x"]
    if own:
        import paper_2603_08957_amd as tre

        q = tre.mx_quantize(s["plan"], "u", x.flatten(1))
        return tre.mx_dequantize(s["plan"], "u", q, dtype=x.dtype).view(x.shape)
    return (_mx(x) if s["c"]["order"] == "rk" else _mx_t(x)).contiguous().to(x.dtype)


def _round_exact(c, seed):
    x = _round_inputs(c, seed)
    return (_exact_mx(x) if c["order"] == "rk" else _exact_mx_t(x)).contiguous()


def _round_work(c):
    n = c["tiles"] * c["rows"] * c["k"]
    eb = 2 if c["dtype"] == "bf16" else 4
    return {"bytes": n * 2 * eb + 2 * c["tiles"] * c["rows"] * _row(c["k"]), "flops": 4 * n}


def _row(k):
    """Bytes of k values in 4 bits: 16 of codes and one of scale for each block."""
    return 17 * ((k + 31) // 32)


# -------------------------------------------------------------------- token

def _token_inputs(c, seed):
    g = _gen(seed)
    return (_values((c["n"], c["d"]), "bf16", g, 0.5), _values((c["vocab"], c["d"]), "bf16", g))


def _token_prepare(c, seed):
    x, w = _token_inputs(c, seed)
    nt = c["vocab"] // c["tile"]
    s = {"c": c, "x": x, "keys": _range(nt)}
    if own:  # the table is laid out once, when the model is loaded
        import paper_2603_08957_amd as tre

        s["plan"] = tre.Plan("vd,nd->nv", "v", {"v": c["vocab"], "n": c["n"], "d": c["d"]}, {"v": c["tile"]}, "mxfp4")
        s["w"] = tre.mx_quantize(s["plan"], "u", w.view(nt, -1))
        s["call"] = _Call(s["plan"], nt, 1, nt, nt)
    else:
        s["w"] = _mx(w)
    return s


def _token_run(s):
    c, x = s["c"], s["x"]
    if own:
        import paper_2603_08957_amd as tre

        keys, tiles = s["call"](s["keys"], s["w"], None, tre.mx_quantize(s["plan"], "v", x.view(1, -1)))
        return {"keys": keys, "tiles": tiles}
    y = _mx(x) @ s["w"].T
    return {"keys": s["keys"].clone(), "tiles": y.view(c["n"], -1, c["tile"]).transpose(0, 1).flatten(1)}


def _token_exact(c, seed):
    x, w = _token_inputs(c, seed)
    y = _exact_mx(x) @ _exact_mx(w).T
    return {"keys": None, "tiles": y.view(c["n"], -1, c["tile"]).transpose(0, 1).flatten(1)}


def _token_work(c):
    return {"bytes": c["vocab"] * _row(c["d"]) + 2 * c["n"] * c["d"] + 4 * c["n"] * c["vocab"] + 8 * (c["vocab"] // c["tile"]),
            "flops": 2 * c["n"] * c["vocab"] * c["d"]}


# ------------------------------------------------------------------- blocks

def _blocks_inputs(c, seed):
    g = _gen(seed)
    keys = _block_keys(c, g)
    return (keys, _values((keys.shape[0], c["block"], c["block"]), "bf16", g),
            _values((c["n"] // c["block"], c["block"], c["cols"]), "bf16", g, 0.5))


def _blocks_prepare(c, seed):
    keys, a, b = _blocks_inputs(c, seed)
    nb, t = c["n"] // c["block"], c["block"]
    s = {"c": c, "keys": keys, "b": b}
    if own:  # the sparse matrix is laid out once
        import paper_2603_08957_amd as tre

        s["plan"] = tre.Plan("ij,jk->ik", "ij", {"i": c["n"], "j": c["n"], "k": c["cols"]}, {"i": t, "j": t}, "mxfp4")
        s["a"] = tre.mx_quantize(s["plan"], "u", a.flatten(1))
        s["bk"] = _range(nb)
        s["call"] = _Call(s["plan"], keys.shape[0], nb, keys.shape[0], nb)
    else:
        s["a"] = _mx(a)
    return s


def _blocks_run(s):
    c, keys, b = s["c"], s["keys"], s["b"]
    nb = c["n"] // c["block"]
    if own:
        import paper_2603_08957_amd as tre

        wk, tiles = s["call"](keys, s["a"], s["bk"], tre.mx_quantize(s["plan"], "v", b.flatten(1)))
        return {"keys": wk, "tiles": tiles}
    p = torch.bmm(s["a"], _mx_t(b)[keys[:, 1].long()].contiguous())
    w = torch.zeros((nb, c["block"], c["cols"]), device=DEV).index_add_(0, keys[:, 0].long(), p)
    return {"keys": _range(nb), "tiles": w.flatten(1)}


def _blocks_exact(c, seed):
    keys, a, b = _blocks_inputs(c, seed)
    nb = c["n"] // c["block"]
    w = torch.zeros((nb, c["block"], c["cols"]), device=DEV, dtype=torch.float64)
    av, bv = _exact_mx(a), _exact_mx_t(b).contiguous()
    for at in range(0, keys.shape[0], 256):
        i, j = keys[at:at + 256, 0].long(), keys[at:at + 256, 1].long()
        w.index_add_(0, i, torch.bmm(av[at:at + 256], bv[j]))
    return {"keys": None, "tiles": w.flatten(1)}


def _blocks_work(c):
    nb, t = c["n"] // c["block"], c["block"]
    pairs = nb + c["density"] * nb * (nb - 1)
    return {"bytes": pairs * (t * _row(t) + 8) + c["n"] * c["cols"] * (2 + 4), "flops": 2 * pairs * t * t * c["cols"]}


# -------------------------------------------------------------------- dense

def _dense_inputs(c, seed):
    g = _gen(seed)
    return (_values((c["n"], c["d"]), "bf16", g, 0.5), _values((c["v"], c["d"]), "bf16", g))


def _grid(a, b):
    """Keys (i, j) of a full grid."""
    return _keys(torch.arange(a, device=DEV).repeat_interleave(b), torch.arange(b, device=DEV).repeat(a))


def _cut(y, rows, cols):
    """A matrix as tiles [rows x cols], one row of tiles after the other."""
    return y.view(y.shape[0] // rows, rows, y.shape[1] // cols, cols).transpose(1, 2).flatten(0, 1).flatten(1)


def _dense_prepare(c, seed):
    x, w = _dense_inputs(c, seed)
    t = c["tile"]
    nn, nv = c["n"] // t, c["v"] // t
    s = {"c": c, "x": x}
    if own:  # the weights are laid out once
        import paper_2603_08957_amd as tre

        s["plan"] = tre.Plan("nd,vd->nv", "nv", {"n": c["n"], "v": c["v"], "d": c["d"]}, {"n": t, "v": t}, "mxfp4",
                             w_bf16=True)
        s["xk"], s["wk"] = _range(nn), _range(nv)
        s["w"] = tre.mx_quantize(s["plan"], "v", w.view(nv, -1))
        s["call"] = _Call(s["plan"], nn, nv, nn * nv, nn * nv)
    else:
        s["w"] = _mx(w)
    return s


def _dense_run(s):
    c, x = s["c"], s["x"]
    t = c["tile"]
    if own:
        import paper_2603_08957_amd as tre

        q = tre.mx_quantize(s["plan"], "u", x.view(c["n"] // t, -1))
        keys, tiles = s["call"](s["xk"], q, s["wk"], s["w"])
        return {"keys": keys, "tiles": tiles}
    y = _mx(x) @ s["w"].T
    return {"keys": _grid(c["n"] // t, c["v"] // t), "tiles": _cut(y.to(BF16), t, t)}


def _dense_exact(c, seed):
    x, w = _dense_inputs(c, seed)
    return {"keys": None, "tiles": _cut(_exact_mx(x) @ _exact_mx(w).T, c["tile"], c["tile"])}


def _dense_work(c):
    return {"bytes": 2 * c["n"] * c["d"] + c["v"] * _row(c["d"]) + 2 * c["n"] * c["v"], "flops": 2 * c["n"] * c["v"] * c["d"]}


# -------------------------------------------------------------------- train

def _train_inputs(c, seed):
    g = _gen(seed)
    return (_values((c["n"], c["d"]), "bf16", g, 0.5), _values((c["v"], c["d"]), "bf16", g),
            _values((c["n"], c["v"]), "bf16", g, 0.5))


def _train_prepare(c, seed):
    x, w, dy = _train_inputs(c, seed)
    t = c["tile"]
    nn, nv = c["n"] // t, c["v"] // t
    s = {"c": c, "x": x, "w": w, "dy": _cut(dy, t, t)}
    if own:
        import paper_2603_08957_amd as tre

        ext, til = {"n": c["n"], "v": c["v"], "d": c["d"]}, {"n": t, "v": t}
        s["y"] = tre.Plan("nd,vd->nv", "nv", ext, til, "mxfp4", w_bf16=True)
        s["dx"] = tre.Plan("nv,vd->nd", "nv", ext, til, "mxfp4", w_bf16=True)
        s["dw"] = tre.Plan("nv,nd->vd", "nv", ext, til, "mxfp4")
        s["xk"], s["wk"], s["yk"] = _range(nn), _range(nv), _grid(nn, nv)
        s["calls"] = (_Call(s["y"], nn, nv, nn * nv, nn * nv), _Call(s["dx"], nn * nv, nv, nn * nv, nn),
                      _Call(s["dw"], nn * nv, nn, nn * nv, nv))
    return s


def _train_run(s):
    c, x, w, dy = s["c"], s["x"], s["w"], s["dy"]
    t = c["tile"]
    nn, nv = c["n"] // t, c["v"] // t
    if own:
        import paper_2603_08957_amd as tre

        q, xt, wt = tre.mx_quantize, x.view(nn, -1), w.view(nv, -1)
        y, dx, dw = s["calls"]
        _, yt = y(s["xk"], q(s["y"], "u", xt), s["wk"], q(s["y"], "v", wt))
        _, dxt = dx(s["yk"], q(s["dx"], "u", dy), s["wk"], q(s["dx"], "v", wt))
        _, dwt = dw(s["yk"], q(s["dw"], "u", dy), s["xk"], q(s["dw"], "v", xt))
        return {"y": yt, "dx": dxt.view(c["n"], -1), "dw": dwt.view(c["v"], -1)}
    g = dy.view(nn, nv, t, t).transpose(1, 2)
    y = _mx(x) @ _mx(w).T
    # (blocks of 32 start anew in every tile of the contracted label)
    gn, wn = _mx(g).reshape(c["n"], -1), _mx_t(w.view(nv, t, -1)).reshape(c["v"], -1)
    gv, xv = _mx_t(g.transpose(1, 2)).transpose(1, 2).reshape(c["n"], -1), _mx_t(x.view(nn, t, -1)).reshape(c["n"], -1)
    return {"y": _cut(y.to(BF16), t, t), "dx": (gn @ wn).to(BF16), "dw": gv.T @ xv}


def _train_exact(c, seed):
    x, w, dy = _train_inputs(c, seed)
    t = c["tile"]
    nn, nv = c["n"] // t, c["v"] // t
    y = _exact_mx(x) @ _exact_mx(w).T
    gn = _exact_mx(dy.view(c["n"], nv, t)).reshape(c["n"], -1)
    gv = _exact_mx_t(dy.view(nn, t, -1)).reshape(c["n"], -1)
    dx = gn @ _exact_mx_t(w.view(nv, t, -1)).reshape(c["v"], -1)
    dw = gv.T @ _exact_mx_t(x.view(nn, t, -1)).reshape(c["n"], -1)
    return {"y": _cut(y, t, t), "dx": dx, "dw": dw}


def _train_work(c):
    n, d, v = c["n"], c["d"], c["v"]
    return {"bytes": 2 * (n * d + v * d + n * v) + 2 * (n * v + n * d) + 4 * v * d, "flops": 6 * n * d * v}


# ------------------------------------------------------------------- lookup

def _lookup_inputs(c, seed):
    g = _gen(seed)
    return _tokens(c, g), _values((c["vocab"], c["d"]), "f32" if c["table"] == "f32" else "bf16", g)


def _lookup_prepare(c, seed):
    ids, table = _lookup_inputs(c, seed)
    s = {"c": c, "ids": ids, "table": table, "scale": math.sqrt(c["d"])}
    if c["table"] == "mxfp4" and own:  # the table is laid out once, when the model is loaded
        import paper_2603_08957_amd as tre

        s["plan"] = tre.Plan("vd,nd->nv", "v", {"v": c["vocab"], "n": 16, "d": c["d"]}, {"v": c["tile"]}, "mxfp4")
        s["table"] = tre.mx_quantize(s["plan"], "u", table.view(c["vocab"] // c["tile"], -1))
    elif c["table"] == "mxfp4":
        s["table"] = _mx(table)
    return s


def _lookup_run(s):
    c, ids = s["c"], s["ids"]
    if own:
        import paper_2603_08957_amd as tre

        mx = {"plan": s["plan"], "operand": "u"} if c["table"] == "mxfp4" else {}
        return tre.lookup(s["table"], ids, scale=s["scale"], dtype=_TYPE[c["out"]], **mx)
    rows = s["table"][ids.clamp_min(0)].float() * s["scale"]
    return torch.where(ids[:, None] >= 0, rows, 0.0).to(_TYPE[c["out"]])


def _lookup_exact(c, seed):
    ids, table = _lookup_inputs(c, seed)
    if c["table"] == "mxfp4":
        table = _exact_mx(table)
    rows = table[ids.clamp_min(0)].double() * math.sqrt(c["d"])
    rows[ids < 0] = 0
    return rows


def _distinct(c):
    """The mean number of different tokens among n."""
    k = torch.arange(c["vocab"], dtype=torch.float64)
    p = torch.log((k + 2) / (k + 1)) / math.log(c["vocab"] + 1)
    return float(-torch.expm1(c["n"] * (1 - c["pad"]) * torch.log1p(-p)).sum())


def _lookup_work(c):
    row = _row(c["d"]) if c["table"] == "mxfp4" else c["d"] * (4 if c["table"] == "f32" else 2)
    out = c["d"] * (4 if c["out"] == "f32" else 2)
    return {"bytes": _distinct(c) * row + c["n"] * (out + 8), "flops": c["n"] * c["d"]}


# -------------------------------------------------------------- lookup_grad

def _lookup_grad_inputs(c, seed):
    g = _gen(seed)
    return _tokens(c, g), _values((c["n"], c["d"]), c["grad"], g, 0.5)


def _lookup_grad_prepare(c, seed):
    ids, grad = _lookup_grad_inputs(c, seed)
    s = {"c": c, "ids": ids, "grad": grad, "scale": math.sqrt(c["d"])}
    if own:  # a training program keeps the gradient's buffer and the workspace
        import paper_2603_08957_amd as tre

        s["out"] = torch.empty((c["vocab"], c["d"]), dtype=_TYPE[c["out"]], device=DEV)
        s["ws"] = tre.alloc_workspace(tre.lookup_grad_workspace_bytes(c["n"], c["vocab"], c["d"]))
    return s


def _lookup_grad_run(s):
    c, ids, grad = s["c"], s["ids"], s["grad"]
    if own:
        import paper_2603_08957_amd as tre

        return tre.lookup_grad(grad, ids, c["vocab"], scale=s["scale"], out=s["out"], ws=s["ws"])
    rows = torch.where(ids[:, None] >= 0, grad.float(), 0.0)
    total = torch.zeros((c["vocab"], c["d"]), device=DEV).index_add_(0, ids.clamp_min(0), rows)
    return (total * s["scale"]).to(_TYPE[c["out"]])


def _lookup_grad_exact(c, seed):
    ids, grad = _lookup_grad_inputs(c, seed)
    keep = ids >= 0
    total = torch.zeros((c["vocab"], c["d"]), dtype=torch.float64, device=DEV)
    return total.index_add_(0, ids[keep], grad[keep].double()) * math.sqrt(c["d"])


def _lookup_grad_work(c):
    gb = 4 if c["grad"] == "f32" else 2
    ob = 4 if c["out"] == "f32" else 2
    return {"bytes": c["n"] * ((1 - c["pad"]) * c["d"] * gb + 8) + c["vocab"] * c["d"] * ob, "flops": c["n"] * c["d"]}


# ------------------------------------------------------------------------

_KINDS = {
    "round": (_round_prepare, _round_run, _round_exact, _round_work),
    "token": (_token_prepare, _token_run, _token_exact, _token_work),
    "blocks": (_blocks_prepare, _blocks_run, _blocks_exact, _blocks_work),
    "dense": (_dense_prepare, _dense_run, _dense_exact, _dense_work),
    "train": (_train_prepare, _train_run, _train_exact, _train_work),
    "lookup": (_lookup_prepare, _lookup_run, _lookup_exact, _lookup_work),
    "lookup_grad": (_lookup_grad_prepare, _lookup_grad_run, _lookup_grad_exact, _lookup_grad_work),
}


def prepare(case, seed):
    return _KINDS[case["kind"]][0](case, seed)


def run(state):
    return _KINDS[state["c"]["kind"]][1](state)


def exact(case, seed):
    return _KINDS[case["kind"]][2](case, seed)


def work(case):
    return _KINDS[case["kind"]][3](case)
