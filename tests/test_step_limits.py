"""Limits of the training step's arguments and codes, on the CPU."""
import ctypes
from array import array

import pytest


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
