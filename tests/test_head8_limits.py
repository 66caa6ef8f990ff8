"""Limits of the 8-bit head's operators that their host code has to see: workspaces of calls with several groups of matrices, and
arguments past the range of what they are computed in."""
import ctypes

import pytest

from paper_1404_1869_amd import densenet as D
from test_head8_abi import back, muon, scores


def muon_bytes(*shapes, **kw):
    """The workspace that matrices of these shapes ask for together."""
    t = (D.dn_muon_tensor * len(shapes))()
    for e, (rows, cols) in zip(t, shapes):
        e.p = e.g = e.m = 4096
        e.rows, e.cols, e.rate = rows, cols, 1.0
    k = D.dn_muon_params(0.02, 0.95, 0.0, 1.0, 1e-7)
    for c in k.coefficients:
        c[:] = (3.4445, -4.775, 2.0315)
    k.steps, k.nesterov = 5, 1
    need = ctypes.c_size_t()
    assert D.lib().densenet_muon(t, len(shapes), D.DN_F32, D.DN_F32, D.DN_BF16, ctypes.byref(k), None, 0, ctypes.byref(need), None) == D.DN_OK
    return need.value


def test_matrices_past_a_launch_share_its_workspace():
    """Matrices that no workgroup holds go 32 to a launch, whose workspace the next launch takes again: the largest counts."""
    wide, tall, small = (130, 140), (141, 131), (100, 100)
    assert muon_bytes(small, small) == D.DN_NO_WORKSPACE
    one, many = muon_bytes(wide), muon_bytes(*[wide, tall] * 16)
    assert D.DN_NO_WORKSPACE < one < many
    assert muon_bytes(*[wide, tall] * 16, wide) == many and muon_bytes(*[wide, tall] * 160) == many
    assert muon_bytes(*[small, wide, tall, small] * 160) == many  # (small ones go to launches of their own)
    big = muon_bytes((2000, 3000))
    assert big > many
    assert muon_bytes(*[wide, tall] * 16, (2000, 3000)) == big  # the larger launch is the last one
    first = muon_bytes((2000, 3000), *[wide, tall] * 15, wide)
    assert first > many
    assert muon_bytes((2000, 3000), *[small] * 100, *[wide, tall] * 32) == first  # or the first, with 31 others
    same = muon_bytes(*[wide] * 32)
    assert muon(rows=130, cols=140, count=33, size=same - 1) == D.DN_E_BUFFER_TOO_SMALL


@pytest.mark.parametrize("kw", [dict(lr=1e39), dict(grad_scale=-1e39), dict(rate=1e39), dict(lr=1e30, weight_decay=1e30), dict(lr=1e30, rate=1e30),
                                dict(lr=1e-30, rate=-1e300)])
def test_muon_refuses_what_fp32_does_not_hold(kw):
    """Parameters that are finite, and infinite where the step is computed: the weights would be NaN."""
    need = ctypes.c_size_t()
    assert muon(work=None, need=ctypes.byref(need)) == D.DN_OK
    assert muon(work=None, need=ctypes.byref(need), **kw) == D.DN_E_INVALID_ARG and D.last_error()


def test_scores_refuse_a_scale_whose_base_2_exponents_overflow():
    """x log2(e) is what exponentials take: with a scale past 2^128 ln 2 equal logits would have a lse of NaN."""
    need = ctypes.c_size_t()
    for scale, status in ((2.0 ** 127, D.DN_OK), (3e38, D.DN_E_INVALID_ARG)):
        assert scores(work=None, need=ctypes.byref(need), scale=scale) == status
        assert back(n=0, x=None, dx=None, lse=None, scale=scale) == status
