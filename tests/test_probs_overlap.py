"""A gradient of log probabilities that overlaps what it is computed from is refused, on the CPU: layouts of few elements, whose
bytes are listed.  Calls that are not refused find no GPU here."""
import random

import pytest

BASE = 1 << 20  # (nothing is read there: no GPU)


@pytest.fixture(scope="module")
def call():
    import torch

    import paper_2603_08957_amd as tre

    if torch.cuda.is_available():
        pytest.skip("addresses of nothing")
    L, S = tre.lib(), tre.tre.STATUS

    def f(n, tiles, cols, x, x_bytes, x_strides, out, out_bytes, out_strides, stats=BASE << 1, ids=BASE << 2, by=BASE << 3):
        return S[L.tre_log_probs_grad(BASE + x, x_bytes == 2, n, tiles * cols, cols, *x_strides, stats, ids, 8, 1.0, by, None, None, None,
                                      BASE + out, out_bytes == 2, *out_strides, None, None)]

    return f


def bytes_of(at, n, tiles, cols, size, strides):
    return {at + (i * strides[0] + t * strides[1] + c) * size + b
            for i in range(n) for t in range(tiles) for c in range(cols) for b in range(size)}


def strides_of(r, n, tiles, cols, apart):
    """(row, tile): rows of a tile or tiles of a row side by side, with gaps or without; scores may share places."""
    gap, far = r.choice([0, 0, 1, cols, 3 * cols + 1]), r.choice([0, 0, 2, 7 * cols])
    inner = cols + gap
    if r.random() < 0.5:
        s = (inner, inner * n + far)
    else:
        s = (inner * tiles + far, inner)
    if not apart and r.random() < 0.3:
        s = (r.choice([0, 1, s[0]]), r.choice([0, s[1]]))
    return s


def test_overlaps(call):
    r = random.Random(4)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        n, tiles, cols = r.randint(1, 4), r.randint(1, 4), r.randint(1, 5)
        xb, ob = r.choice([2, 4]), r.choice([2, 4])
        os = strides_of(r, n, tiles, cols, True)
        kind = r.choice(["whole", "same", "any"])
        xs = strides_of(r, n, tiles, cols, False)
        if kind == "whole":
            xs = r.choice([(cols, cols * n), (cols * tiles, cols), (0, cols), (0, 0)])
        elif kind == "same" and (os[0] * ob % xb or os[1] * ob % xb):
            continue
        elif kind == "same":
            xs = (os[0] * ob // xb, os[1] * ob // xb)
        x, out = 4 * r.randint(100, 140), 4 * r.randint(100, 140)
        if x == out:
            continue
        common = bool(bytes_of(x, n, tiles, cols, xb, xs) & bytes_of(out, n, tiles, cols, ob, os))
        got = call(n, tiles, cols, x, xb, xs, out, ob, os)
        assert got in ("TRE_E_ARG", "TRE_E_DEVICE")
        if common and kind != "any":
            assert got == "TRE_E_ARG", (n, tiles, cols, x, xb, xs, out, ob, os)
        if not common:
            assert got == "TRE_E_DEVICE", (n, tiles, cols, x, xb, xs, out, ob, os)
        if kind != "any":
            seen[common] += 1
    assert min(seen.values()) > 500


def test_values_of_tokens_inside_the_gradient(call):
    """Statistics in a gap of the gradient's rows are apart, in a row they are not."""
    n, cols = 3, 8
    for at, bad in ((32, False), (28, True), (0, True), (56, True), (60, True), (-24, False), (-20, True), (164, False), (159 // 4 * 4, True)):
        # rows of 32 bytes every 64; 24 bytes of statistics
        assert call(n, 1, cols, -4096, 4, (8, 0), 0, 4, (16, 0), stats=BASE + at) == ("TRE_E_ARG" if bad else "TRE_E_DEVICE"), at
    assert call(n, 1, cols, -4096, 4, (8, 0), 0, 4, (16, 0), ids=BASE + 32) == "TRE_E_DEVICE"
    assert call(n, 1, cols, -4096, 4, (8, 0), 0, 4, (16, 0), ids=BASE + 48) == "TRE_E_ARG"
    assert call(n, 1, cols, -4096, 4, (8, 0), 0, 4, (16, 0), by=BASE + 52) == "TRE_E_DEVICE"
    assert call(n, 1, cols, -4096, 4, (8, 0), 0, 4, (16, 0), by=BASE + 56) == "TRE_E_ARG"


def test_large_layouts(call):
    """Two halves of one buffer's rows, and a row that is not its own half."""
    n, vocab = 1 << 20, 1 << 20
    far = dict(stats=1 << 56, ids=1 << 56, by=1 << 56)
    for xb, ob in ((4, 4), (2, 4), (4, 2)):
        xs, os = (8 * vocab // xb, 0), (8 * vocab // ob, 0)
        assert call(n, 1, vocab, 0, xb, xs, 4 * vocab, ob, os, **far) == "TRE_E_DEVICE"
        assert call(n, 1, vocab, 4 * vocab, xb, xs, 0, ob, os, **far) == "TRE_E_DEVICE"
        assert call(n, 1, vocab, 0, xb, xs, xb * vocab - 4, ob, os, **far) == "TRE_E_ARG"
        assert call(n, 1, vocab, ((n - 1) << 23) + ob * vocab - 4, xb, xs, 0, ob, os, **far) == "TRE_E_ARG"
        assert call(n, 1, vocab, n << 23, xb, xs, 0, ob, os, **far) == "TRE_E_DEVICE"
