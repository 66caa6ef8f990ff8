"""Limits of the head's entry points, on a machine without a GPU: what a launch or a workspace could not hold is refused on the
host, and what is held in pieces needs a workspace of one piece."""
import ctypes

import pytest

from paper_1404_1869_amd import densenet as D

P = ctypes.c_void_p(4096)  # never read: every call ends on the host


def loss(n, C, V, dt, need, work=None):
    return D.lib().densenet_softmax_loss(P, C, P, C, P, n, C, V, dt, P, P, work, 0, ctypes.byref(need), None)


def loss_back(n, C, V, dt, need, work=None):
    return D.lib().densenet_softmax_loss_backward(P, C, P, C, P, P, None, 1.0, n, C, V, dt, P, C, P, C, work, 0, ctypes.byref(need), None)


@pytest.mark.parametrize("dt", [D.DN_F32, D.DN_BF16])
def test_gradient_refuses_what_no_launch_holds(dt):
    need = ctypes.c_size_t()
    assert loss_back((1 << 30) - 256, 8, 10, dt, need) == D.DN_OK
    assert loss_back((1 << 30) - 255, 8, 10, dt, need) == D.DN_E_TOO_LARGE and D.last_error()
    assert loss_back(1 << 20, 1 << 18, 300, dt, need) == D.DN_E_TOO_LARGE   # 2^24 tiles of dh
    assert loss_back(300, 1 << 18, 1 << 20, dt, need) == D.DN_E_TOO_LARGE   # of dw
    assert loss_back((1 << 20) - 128, 1 << 18, 300, dt, need) == D.DN_OK


@pytest.mark.parametrize("dt", [D.DN_F32, D.DN_F16, D.DN_BF16])
@pytest.mark.parametrize("C,V", [(8, 10), (16, 100), (8, 3000)])
def test_many_rows_need_the_workspace_of_a_piece(dt, C, V):
    """From 2^22 rows on the forward pass goes in pieces."""
    need = ctypes.c_size_t()
    assert loss(1 << 22, C, V, dt, need) == D.DN_OK
    most = need.value
    for n in ((1 << 24) + 3, (1 << 26) + 5, (1 << 31) - 256):
        assert loss(n, C, V, dt, need) == D.DN_OK and 0 < need.value <= 2.1 * most


def test_a_piece_of_few_rows_has_its_own_workspace():
    """2^22 - 128 rows a piece: some rows more are two pieces of half of them, and every piece's needs are met."""
    need = ctypes.c_size_t()
    sizes = []
    for n in ((1 << 22) - 128, (1 << 22) - 127, (1 << 21), 64):
        assert loss(n, 8, 3000, D.DN_F32, need) == D.DN_OK
        sizes.append(need.value)
    assert sizes[1] <= sizes[0] * 1.01 and sizes[1] >= sizes[2] * 0.99


def test_gradients_of_no_rows_ask_for_a_workspace():
    """A null workspace is a size query, so a call that has dw or dgamma to write must not be told that it needs none."""
    need = ctypes.c_size_t(0)
    assert loss_back(0, 8, 10, D.DN_BF16, need) == D.DN_OK and need.value > 0
    need.value = 0
    assert D.lib().densenet_rms_norm_backward(P, 8, D.DN_F32, P, 8, None, 0, None, 0, 8, D.DN_F32, 1e-6, P, 8, P, None, 0,
                                              ctypes.byref(need), None) == D.DN_OK and need.value > 0


@pytest.mark.parametrize("option", ["--words", "--boxes", "--steps"])
def test_example_refuses_nothing_to_do(option, capsys):
    pytest.importorskip("torch")
    from paper_1404_1869_amd import region_head
    with pytest.raises(SystemExit) as e:
        region_head.main([option, "0"])
    assert e.value.code == 2 and "at least 1" in capsys.readouterr().err
