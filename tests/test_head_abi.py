"""The head's entry points on a machine without a GPU: size queries, and bad arguments refused on the host before any
device work, with a status and a message."""
import ctypes

import pytest

from paper_1404_1869_amd import densenet as D

P = ctypes.c_void_p(4096)   # never read: every call below ends on the host
ODD = ctypes.c_void_p(4097)


def norm(x=P, xs=64, res=None, rs=0, gamma=None, n=4, C=64, dt=D.DN_F32, eps=1e-6, s=None, ss=0, y=P, ys=64, ydt=D.DN_F32, block=0,
         scale=None):
    return D.lib().densenet_rms_norm(x, xs, res, rs, gamma, n, C, dt, eps, s, ss, y, ys, ydt, block, scale, None)


def norm_back(dy=P, ds=64, ddt=D.DN_F32, s=P, ss=64, e=None, es=0, gamma=None, n=4, C=64, dt=D.DN_F32, eps=1e-6, dx=P, xs=64, dg=P,
              ws=P, size=1 << 30, need=None):
    return D.lib().densenet_rms_norm_backward(dy, ds, ddt, s, ss, e, es, gamma, n, C, dt, eps, dx, xs, dg, ws, size, need, None)


def loss(h=P, hs=64, w=P, ws=64, lab=P, n=4, C=64, V=100, dt=D.DN_BF16, out=P, lse=P, work=P, size=1 << 40, need=None):
    return D.lib().densenet_softmax_loss(h, hs, w, ws, lab, n, C, V, dt, out, lse, work, size, need, None)


def loss_back(h=P, hs=64, w=P, ws=64, lab=P, lse=P, dl=None, n=4, C=64, V=100, dt=D.DN_BF16, dh=P, dhs=64, dw=P, dws=64, work=P,
              size=1 << 40, need=None):
    return D.lib().densenet_softmax_loss_backward(h, hs, w, ws, lab, lse, dl, 1.0, n, C, V, dt, dh, dhs, dw, dws, work, size, need, None)


def adamw(n=1000, block=0, blocks=4, count=1, p=4096, g=4096, copy=None, pdt=D.DN_F32, gdt=D.DN_F32, cdt=D.DN_BF16, m=P, v=P, ms=P, vs=P,
          params=True, table=True, **kw):
    t = (D.dn_adamw_tensor * max(1, count))()
    t[0].p, t[0].g, t[0].copy, t[0].n, t[0].block = p, g, copy, n, block
    k = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0, step=1, seed=0, state_bits=32)
    k.update(kw)
    q = D.dn_adamw_params(*(k[f] for f, _ in D.dn_adamw_params._fields_))
    return D.lib().densenet_adamw(t if table else None, count, pdt, gdt, cdt, ctypes.byref(q) if params else None, m, v, ms, vs, blocks,
                                  None)


INV, LARGE, SMALL, UNS = D.DN_E_INVALID_ARG, D.DN_E_TOO_LARGE, D.DN_E_BUFFER_TOO_SMALL, D.DN_E_UNSUPPORTED


@pytest.mark.parametrize("call,kw,status", [
    (norm, dict(x=None), INV), (norm, dict(y=None), INV), (norm, dict(x=ODD), INV), (norm, dict(xs=63), INV), (norm, dict(ys=10), INV),
    (norm, dict(res=P, rs=1), INV), (norm, dict(s=P, ss=5), INV), (norm, dict(n=-1), INV), (norm, dict(C=0), INV),
    (norm, dict(C=32769, xs=40000, ys=40000), LARGE), (norm, dict(dt=3), UNS), (norm, dict(ydt=4), UNS), (norm, dict(eps=-1.0), INV),
    (norm, dict(eps=float("nan")), INV), (norm, dict(block=32), INV), (norm, dict(scale=P), INV), (norm, dict(ydt=D.DN_F8), INV),
    (norm, dict(ydt=D.DN_F8, scale=P, block=48), UNS), (norm, dict(gamma=ODD), INV), (norm, dict(n=1 << 31), LARGE),
    (norm_back, dict(dy=None), INV), (norm_back, dict(s=None), INV), (norm_back, dict(dx=None), INV), (norm_back, dict(ddt=3), UNS),
    (norm_back, dict(e=P, es=3), INV), (norm_back, dict(size=8), SMALL), (norm_back, dict(ws=ctypes.c_void_p(4100)), INV),
    (norm_back, dict(dg=ODD), INV), (norm_back, dict(eps=float("inf")), INV), (norm_back, dict(C=40000, ss=40000), LARGE),
    (loss, dict(h=None), INV), (loss, dict(w=None), INV), (loss, dict(lab=None), INV), (loss, dict(out=None), INV), (loss, dict(lse=None), INV),
    (loss, dict(hs=10), INV), (loss, dict(ws=10), INV), (loss, dict(V=0), INV), (loss, dict(C=0), INV), (loss, dict(n=-5), INV),
    (loss, dict(dt=3), UNS), (loss, dict(h=ODD), INV), (loss, dict(size=4), SMALL), (loss, dict(C=1 << 22, hs=1 << 22, ws=1 << 22), LARGE),
    (loss, dict(n=1 << 30, V=1 << 30), LARGE),
    (loss_back, dict(lse=None), INV), (loss_back, dict(dh=None), INV), (loss_back, dict(dw=None), INV), (loss_back, dict(dhs=63), INV),
    (loss_back, dict(dws=0), INV), (loss_back, dict(size=4), SMALL), (loss_back, dict(dw=ODD), INV), (loss_back, dict(dt=7), UNS),
    (adamw, dict(params=False), INV), (adamw, dict(table=False), INV), (adamw, dict(count=-1), INV), (adamw, dict(p=None), INV),
    (adamw, dict(g=None), INV), (adamw, dict(n=-1), INV), (adamw, dict(n=1025), INV), (adamw, dict(block=1), INV), (adamw, dict(block=-1), INV),
    (adamw, dict(p=4098), INV), (adamw, dict(copy=4097), INV), (adamw, dict(m=None), INV), (adamw, dict(v=ODD), INV), (adamw, dict(pdt=3), UNS),
    (adamw, dict(cdt=D.DN_F32), UNS), (adamw, dict(state_bits=16), UNS), (adamw, dict(state_bits=8, ms=None), INV),
    (adamw, dict(beta1=1.0), INV), (adamw, dict(beta2=-0.1), INV), (adamw, dict(eps=0.0), INV), (adamw, dict(eps=1e-60), INV),
    (adamw, dict(step=0), INV), (adamw, dict(lr=float("nan")), INV), (adamw, dict(grad_scale=float("inf")), INV),
    (adamw, dict(blocks=-1), INV), (adamw, dict(n=1 << 62), INV),
])
def test_refuses(call, kw, status):
    assert call(**kw) == status
    assert D.last_error()


def test_nothing_to_do():
    assert norm(n=0, x=None, y=None) == D.DN_OK
    assert loss(n=0, h=None, lab=None, out=None, lse=None) == D.DN_OK
    assert norm_back(n=0, dy=None, s=None, dx=None, dg=None) == D.DN_OK
    assert adamw(count=0) == D.DN_OK and adamw(n=0, p=None, g=None) == D.DN_OK


def test_size_queries():
    need = ctypes.c_size_t(77)
    assert norm_back(ws=None, need=ctypes.byref(need), n=100000, C=100) == D.DN_OK
    assert 0 < need.value <= 4 * 4096 * 100 and need.value % (4 * 100) == 0
    assert loss(work=None, need=ctypes.byref(need), n=0) == D.DN_OK and need.value == 0
    # rows that the loads can take as they lie need no copy; odd ones and fp32 do
    big = dict(n=1000, C=1000, V=50000, work=None, need=ctypes.byref(need))
    assert loss(hs=1000, ws=1000, **big) == D.DN_OK
    plain = need.value
    assert loss(hs=1001, ws=1000, **big) == D.DN_OK and need.value >= plain + 2 * 1000 * 1000
    assert loss(hs=1000, ws=1000, w=ctypes.c_void_p(4098), **big) == D.DN_OK and need.value >= plain + 2 * 50000 * 1000
    assert loss(hs=1000, ws=1000, dt=D.DN_F32, **big) == D.DN_OK and need.value >= plain + 4 * 51000 * 1000   # two 16-bit parts
    # of few fp32 rows the words are read as they lie
    big["n"] = 64
    assert loss(hs=1000, ws=1000, dt=D.DN_F32, **big) == D.DN_OK and need.value < 50000 * 1000
    # the gradient's workspace does not grow with the whole n x V
    assert loss_back(n=1 << 16, C=64, V=1 << 18, work=None, need=ctypes.byref(need)) == D.DN_OK
    assert need.value < 2 * (1 << 34) / 8


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 64)
    for call in (lambda: D.densenet_rms_norm(x), lambda: D.densenet_softmax_loss(x, x, torch.zeros(4, dtype=torch.int64)),
                 lambda: D.densenet_rms_norm_backward(x, x), lambda: D.AdamWPlan([x], [x])):
        with pytest.raises(D.DenseNetError):
            call()
