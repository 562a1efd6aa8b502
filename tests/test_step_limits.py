"""Limits of the training step's arguments and codes, on the CPU."""
import ctypes
import subprocess
from array import array

import numpy as np
import pytest

from oracle import moments
from paper_2603_08957_amd import build


@pytest.fixture(scope="module")
def tre():
    import paper_2603_08957_amd as t

    t.lib()
    return t


A = 1 << 20  # an address that nothing reads


def test_adamw_refuses_an_eps_whose_reciprocal_is_infinite(tre):
    """1 / eps of an fp32 eps below 2^-126 is taken as infinite, and a weight without moments would become 0 * inf."""
    L, S = tre.lib(), tre.tre.STATUS

    def call(eps):
        o = tre.tre.AdamwOptions(lr=1e-3, beta1=0.9, beta2=0.99, eps=eps, grad_scale=1.0, step=1, bits=32)
        sizes, one, at = array("q", [0]), array("i", [0]), array("q", [A])
        a, b, c = (ctypes.c_void_p(x.buffer_info()[0]) for x in (at, one, sizes))
        return S[L.tre_adamw(1, a, b, a, b, c, A, ctypes.byref(o), None)]  # (no elements: refused or nothing to do)

    assert [call(e) for e in (2.0 ** -127, 1e-40, 2.0 ** -126 * (1 - 2.0 ** -20), 0.0, -1.0)] == ["TRE_E_ARG"] * 5
    assert [call(e) for e in (2.0 ** -126, 1e-30, 1e-8)] == ["TRE_OK"] * 3


def test_codes_of_second_moments_convert_no_value_that_has_no_whole_number(tmp_path):
    """The kernel's own code, built for the host with a trap at a conversion of a float outside the integers' range, against
    the table: every power of two from the denormals up to 128 with random fractions, codes themselves and their middles,
    infinity and NaN."""
    main = tmp_path / "codes.cpp"
    main.write_text("""
#include "codes.h"
#include <cstdio>
int main(int, char** a) {
    FILE *in = fopen(a[1], "rb"), *out = fopen(a[2], "wb");
    struct { float y; uint32_t word; } x;
    while (fread(&x, 8, 1, in) == 1) {
        const uint32_t c[2] = {tre::second_code<false>(x.y, x.word), tre::second_code<true>(x.y, x.word)};
        fwrite(c, 8, 1, out);
    }
    return fclose(out);
}
""")
    exe = tmp_path / "codes"
    r = subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I", build.CSRC,
                        "-Xarch_host", "-fsanitize=float-cast-overflow", "-Xarch_host", "-fsanitize-trap=float-cast-overflow",
                        str(main), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    rng = np.random.default_rng(3)
    t = moments.table(23)[:249]
    y = np.concatenate([rng.uniform(1, 2, (158, 40)) * 2.0 ** np.arange(-150, 8)[:, None], np.tile(t[:-1], (40, 1)).T,
                        np.tile((t[:-1] + t[1:]) / 2, (40, 1)).T]).reshape(-1).astype(np.float32)
    y = np.concatenate([y, np.zeros(-len(y) % 31, np.float32)]).reshape(-1, 31)
    y = np.concatenate([np.full((len(y), 1), 255.5, np.float32), y], 1).reshape(-1)  # (blocks whose power of two is 1)
    word = rng.integers(0, 1 << 32, len(y), dtype=np.uint32)
    odd = np.array([np.inf, np.nan, 256.4], np.float32)
    pairs = np.zeros(len(y) + len(odd), [("y", "f4"), ("word", "u4")])
    pairs["y"], pairs["word"][:len(y)] = np.concatenate([y, odd]), word
    pairs.tofile(tmp_path / "in")
    r = subprocess.run([str(exe), str(tmp_path / "in"), str(tmp_path / "out")])
    assert r.returncode == 0, f"ended with {r.returncode}"
    got = np.fromfile(tmp_path / "out", np.uint32).reshape(-1, 2)[:len(y)]
    nearest, b = moments.encode(y, 23)
    chance, _ = moments.encode(y, 23, (word >> 12).astype(int))
    assert (b == 127).all()
    # (the kernel brings a value that is not zero up to code 1 outside)
    least = (y > 0).astype(int)
    assert np.array_equal(np.maximum(got[:, 0], least), nearest)
    assert np.array_equal(np.maximum(got[:, 1], least), chance)
