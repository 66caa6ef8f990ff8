"""The head's operators (norm, softmax loss, AdamW) through the binding, against plain forms in 64 bits.

Tolerances.  unit(type) is half a unit in the last place relative to a value: 2^-24, 2^-11, 2^-8 for fp32, fp16, bf16 (and
2^-4 for e4m3); a stored result may be off by that, fp16's by 2^-25 near 0.  What is computed in 32 bits before it is bounded
from its terms: a sum of C products by (C / 8 + 16) 2^-24 of the sum of their magnitudes (eight or more are added at a
time), a reduction over a row's threads likewise.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}
EPS = 1e-6


@pytest.fixture(scope="module")
def D():
    from paper_1404_1869_amd import densenet
    assert torch.cuda.is_available()
    densenet.lib()
    return densenet


def rows(g, n, C, dt, pad=0, scale=1.0, offset=0):
    """[n][C] of normal values, rows C + pad apart, the first `offset` elements into its memory."""
    flat = (torch.randn(n * (C + pad) + offset, generator=g, device="cuda") * scale).to(DT[dt])
    return flat[offset:].view(n, C + pad)[:, :C]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def sum_err(C):
    return (C / 8 + 16) * 2.0 ** -24


def within(got, want, bound, what):
    got, want = got.double(), want.double()
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, by up to {float((off / bound).max()):.2f} bounds"


# ---------------------------------------------------------------------------------------------------------------------
# Norm
# ---------------------------------------------------------------------------------------------------------------------
NORM = [  # n, C, type, y type, residual, row padding, first element
    (1, 1, "f32", "f32", False, 0, 0), (1, 4096, "bf16", "bf16", True, 0, 0), (7, 8, "f16", "f32", True, 0, 0),
    (5, 511, "bf16", "f16", True, 1, 0), (9, 513, "f32", "bf16", False, 3, 1), (6, 1024, "f16", "f16", True, 8, 0),
    (3, 1025, "bf16", "bf16", True, 7, 3), (130, 2047, "f16", "f16", True, 0, 0), (4, 4097, "f32", "f16", False, 0, 2),
    (3, 9216, "f32", "bf16", False, 0, 0), (2, 12289, "bf16", "f32", True, 0, 0), (2, 16400, "f16", "bf16", False, 5, 0),
    (2, 32768, "f32", "f32", True, 0, 0), (1, 32767, "bf16", "bf16", False, 0, 1),
]


@pytest.mark.parametrize("n,C,dt,yt,res,pad,off", NORM)
def test_norm(D, n, C, dt, yt, res, pad, off):
    g = gen(n * 1000 + C)
    x, r = rows(g, n, C, dt, pad, 3.0, off), rows(g, n, C, dt, pad, 1.0, off) if res else None
    gamma = 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
    y, s, scale = D.densenet_rms_norm(x, gamma, residual=r, eps=EPS, out_dtype=D.DTYPES[yt])
    assert scale is None and (s is None) == (r is None) and y.dtype == DT[yt]
    a = x.double() + (r.double() if res else 0)
    want = a / (a.square().mean(1, keepdim=True) + EPS).sqrt() * gamma.double()
    within(y, want, (UNIT[yt] + sum_err(C)) * want.abs() + TINY[yt], "y")
    if res:
        within(s, a, UNIT[dt] * a.abs() * (1 + 2.0 ** -20) + 2.0 ** -24 * a.abs() + TINY[dt], "sum")
    # no gamma: ones; results in given memory, the sum over the input's own
    y2 = torch.empty_like(y)
    x2 = x.contiguous()
    D.densenet_rms_norm(x2, None, residual=r, eps=EPS, out_dtype=D.DTYPES[yt], out=y2, sum_out=x2)
    want = want / gamma.double()
    within(y2, want, (UNIT[yt] + sum_err(C)) * want.abs() + TINY[yt], "y without gamma")
    assert torch.equal(x2, s if res else x)


@pytest.mark.parametrize("n,C,dt,block,pad", [(3, 9216, "f32", 0, 0), (5, 1000, "bf16", 0, 3), (4, 1000, "bf16", 32, 0), (3, 513, "f16", 64, 1),
                                             (2, 9216, "f32", 128, 0), (6, 31, "f16", 32, 0), (1, 4100, "bf16", 128, 0),
                                             (2, 20000, "f16", 64, 0)])
def test_norm_in_8_bits(D, n, C, dt, block, pad):
    g = gen(C + block)
    x, gamma = rows(g, n, C, dt, pad, 2.0), 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
    x[-1, :C // 2] = 0  # blocks of zeros
    y, _, scale = D.densenet_rms_norm(x, gamma, eps=EPS, out_dtype=D.DN_F8, block=block)
    a = x.double()
    want = a / (a.square().mean(1, keepdim=True) + EPS).sqrt() * gamma.double()
    b = block or C
    k = -(-C // b)
    top = torch.nn.functional.pad(want, (0, k * b - C)).view(n, k, b).abs().amax(2)
    within(scale, top / 448, (sum_err(C) + 2.0 ** -22) * top / 448, "scale")
    wide = scale.double().repeat_interleave(b, 1)[:, :C]
    within(y.double() * wide, want, (2.0 ** -4 + sum_err(C)) * want.abs() + wide * 2.0 ** -10 * (1 + 2.0 ** -10), "values")
    assert float(y[-1, :C // 2].float().abs().max()) == 0 if C > 1 else True


def test_norm_zero_rows_and_special_values(D):
    x = torch.zeros(4, 100, device="cuda")
    x[1], x[2, 3], x[3, 5] = 1.0, float("nan"), float("inf")
    y, _, _ = D.densenet_rms_norm(x, eps=EPS)
    assert torch.equal(y[0], torch.zeros_like(y[0])) and bool(y[2].isnan().all())
    assert bool(y[3, 5].isnan()) and float(y[3, :5].abs().max()) == 0
    within(y[1], torch.ones(100, device="cuda"), torch.tensor(1e-6, device="cuda"), "ones")
    q, _, k = D.densenet_rms_norm(x, eps=EPS, out_dtype=D.DN_F8)
    assert float(k[0]) == 0 and float(q[0].float().abs().max()) == 0
    assert bool(q[2].float().isnan().all()) and bool(q[3, 5].float().isnan())
    q, _, k = D.densenet_rms_norm(torch.full((1, 64), 1e-30, device="cuda"), eps=1.0, out_dtype=D.DN_F8, block=32)
    within(q.double() * k.double().repeat_interleave(32, 1), torch.full((1, 64), 1e-30, device="cuda"),
           torch.tensor(1e-36, device="cuda"), "small values")
    e = torch.empty(0, 100, device="cuda")
    y, s, _ = D.densenet_rms_norm(e, residual=e)
    assert y.shape == (0, 100) and s.shape == (0, 100)


def plain_norm_back(s, dy, gamma, dsum):
    a = dy * gamma
    q = 1 / (s.square().mean(1, keepdim=True) + EPS).sqrt()
    dx = q * (a - s * q * q * (a * s).mean(1, keepdim=True))
    # magnitudes of what is summed: of dx, and of dgamma
    big = q * (a.abs() + s.abs() * q * q * (a * s).abs().mean(1, keepdim=True))
    if dsum is not None:
        dx, big = dx + dsum, big + dsum.abs()
    return dx, (dy * s * q).sum(0), big, (dy * s * q).abs().sum(0)


@pytest.mark.parametrize("n,C,dt,yt,res,pad", [(1, 1, "f32", "f32", False, 0), (3, 8, "bf16", "bf16", True, 0), (2000, 500, "f32", "bf16", True, 3),
                                              (4100, 24, "f16", "f32", False, 0), (33, 1000, "bf16", "f16", True, 0),
                                              (1500, 2047, "f16", "f16", True, 1), (1025, 4096, "bf16", "bf16", True, 8),
                                              (40, 9216, "f32", "f32", False, 0), (5, 16385, "bf16", "f32", True, 0),
                                              (3, 32768, "f32", "bf16", False, 0)])
def test_norm_gradient(D, n, C, dt, yt, res, pad):
    g = gen(n + C)
    s, dy = rows(g, n, C, dt, pad, 2.0), rows(g, n, C, yt, pad)
    dsum = rows(g, n, C, dt, pad) if res else None
    gamma = 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
    dx, dgamma = D.densenet_rms_norm_backward(dy, s, gamma, dsum=dsum, eps=EPS)
    want, wg, big, bigg = plain_norm_back(s.double(), dy.double(), gamma.double(), None if dsum is None else dsum.double())
    within(dx, want, UNIT[dt] * want.abs() + 4 * sum_err(C) * big + TINY[dt], "dx")
    within(dgamma, wg, (sum_err(C) + sum_err(n)) * bigg + 1e-37, "dgamma")
    again = D.densenet_rms_norm_backward(dy, s, gamma, dsum=dsum, eps=EPS)
    assert torch.equal(dx, again[0]) and torch.equal(dgamma, again[1])


def test_norm_gradient_against_differences(D):
    g = gen(5)
    s, dy, u = (rows(g, 6, 300, "f32") for _ in range(3))
    gamma = 1 + 0.3 * torch.randn(300, generator=g, device="cuda")
    dx, dgamma = D.densenet_rms_norm_backward(dy, s, gamma, eps=EPS)

    def f(x, w):
        return ((x / (x.square().mean(1, keepdim=True) + EPS).sqrt() * w) * dy.double()).sum()
    t, x, w = 1e-4, s.double(), gamma.double()
    slope = (f(x + t * u.double(), w) - f(x - t * u.double(), w)) / (2 * t)
    assert abs(float((dx.double() * u.double()).sum() - slope)) < 1e-4 * float((dx * u).abs().sum())
    uw = u[0].double()
    slope = (f(x, w + t * uw) - f(x, w - t * uw)) / (2 * t)
    assert abs(float((dgamma.double() * uw).sum() - slope)) < 1e-4 * float((dgamma * u[0]).abs().sum())


def test_norm_gradient_of_no_rows_is_zero(D):
    e = torch.empty(0, 100, device="cuda")
    dx, dgamma = D.densenet_rms_norm_backward(e, e, None, dgamma=torch.full((100,), 7.0, device="cuda"))
    assert dx.shape == (0, 100) and float(dgamma.abs().max()) == 0


# ---------------------------------------------------------------------------------------------------------------------
# Softmax loss
# ---------------------------------------------------------------------------------------------------------------------
def loss_case(n, C, V, dt, pad=0, masked=0.2, offset=0, size=1.0):
    g = gen(n * 7 + C * 3 + V)
    h, w = rows(g, n, C, dt, pad, size, offset), rows(g, V, C, dt, pad, 2.0 / math.sqrt(C), offset)
    labels = torch.randint(0, V, (n,), generator=g, device="cuda")
    labels = torch.where(torch.rand(n, generator=g, device="cuda") < masked, -1, labels)
    if n > 2 and masked:
        labels[0], labels[1], labels[2] = V - 1, V, -100  # the last word; two labels past the vocabulary
    return h, w, labels


def plain_loss(h, w, labels, dt):
    """Loss, lse and the error bound of a logit of each row."""
    V = w.shape[0]
    logits = h.double() @ w.double().T
    has = (labels >= 0) & (labels < V)
    lse = torch.logsumexp(logits, 1)
    at = logits.gather(1, labels.clamp(0, V - 1)[:, None])[:, 0]
    # fp32: three parts leave out 2^-23 of a product, and their sum takes six products in turn
    err = (6 * sum_err(h.shape[1]) if dt == "f32" else sum_err(h.shape[1])) * (h.double().abs() @ w.double().abs().T).amax(1)
    return torch.where(has, lse - at, 0.0), torch.where(has, lse, 0.0), logits, has, err


LOSS = [  # n, C, V, type, row padding, first element
    (1, 1, 1, "f32", 0, 0), (1, 8, 5, "bf16", 0, 0), (3, 64, 128, "f16", 0, 0), (1, 4096, 2000, "bf16", 0, 0), (17, 65, 1000, "bf16", 0, 0),
    (32, 72, 257, "f16", 8, 0), (33, 200, 129, "bf16", 3, 1), (64, 128, 30011, "bf16", 0, 0), (65, 31, 4000, "f16", 0, 0),
    (300, 96, 777, "bf16", 0, 8), (257, 1000, 513, "f32", 0, 0), (40, 9216, 100, "f32", 0, 0), (2100, 40, 30000, "f16", 0, 0),
    (700, 520, 20001, "bf16", 0, 0), (5, 33, 100003, "f32", 1, 0), (2049, 264, 6000, "f32", 0, 0),
]


@pytest.mark.parametrize("n,C,V,dt,pad,off", LOSS)
def test_loss(D, n, C, V, dt, pad, off):
    h, w, labels = loss_case(n, C, V, dt, pad, offset=off)
    loss, lse = D.densenet_softmax_loss(h, w, labels)
    want, wl, _, has, err = plain_loss(h, w, labels, dt)
    tol = 2 * err + 2.0 ** -21 * (wl.abs() + 16)
    within(lse, wl, tol, "lse")
    within(loss, want, 2 * tol, "loss")
    assert float(loss[~has].abs().sum()) == 0 and float(lse[~has].abs().sum()) == 0


BACK = LOSS + [(1500, 1100, 3000, "bf16", 0, 0), (4096, 264, 5003, "f16", 0, 0), (130, 2048, 40000, "bf16", 0, 0)]


@pytest.mark.parametrize("per_row", [False, True])
@pytest.mark.parametrize("n,C,V,dt,pad,off", BACK)
def test_loss_gradient(D, n, C, V, dt, pad, off, per_row):
    h, w, labels = loss_case(n, C, V, dt, pad, offset=off)
    want, wl, logits, has, err = plain_loss(h, w, labels, dt)
    dloss = torch.randn(n, generator=gen(3), device="cuda") * 1e-3 if per_row else None
    dh, dw = D.densenet_softmax_loss_backward(h, w, labels, wl.float(), dloss=dloss, scale=0.5)
    p = torch.exp(logits - torch.logsumexp(logits, 1, keepdim=True))
    c = 0.5 * torch.where(has, dloss.double() if per_row else 1.0 / max(1, int(has.sum())), 0.0)
    g = p.clone()
    g.scatter_add_(1, labels.clamp(0, V - 1)[:, None], -torch.ones_like(g[:, :1]))
    g, p = g * c[:, None], p * c.abs()[:, None]
    # g: its rounding (fp32: three parts, 2^-23 left out; fp16: 2^-25 near 0, of values 2^10 times as large), and the
    # exponent's error, 2 err of the logits and the rounding of lse and of the exponent's argument
    top = c.abs().max()
    ge = (2.0 ** -22 if dt == "f32" else UNIT[dt]) * g.abs() + p * (2 * err + 2.0 ** -22 * (wl.abs() + 40))[:, None]
    ge = ge + (2.0 ** -34 * top if dt == "f16" else 1e-30)
    many = 6 if dt == "f32" else 1
    hz = torch.where(has[:, None], h.double(), 0.0)
    for got, want, terms, wrong, K, what in ((dh, g @ w.double(), g.abs() @ w.double().abs(), ge @ w.double().abs(), V, "dh"),
                                             (dw, g.T @ hz, g.abs().T @ hz.abs(), ge.T @ hz.abs(), n, "dw")):
        within(got, want, UNIT[dt] * want.abs() * 1.01 + wrong + many * sum_err(K) * terms + TINY[dt], what)
    assert not bool(dh[~has].any())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_masked_rows_reach_nothing(D, dt):
    h, w, labels = loss_case(200, 136, 900, dt)
    has = (labels >= 0) & (labels < 900)
    loss, lse = D.densenet_softmax_loss(h, w, labels)
    dh, dw = D.densenet_softmax_loss_backward(h, w, labels, lse)
    h2 = h.clone()
    h2[~has] = torch.tensor([float("nan"), float("inf"), -3e38, 1.0], device="cuda").to(h.dtype).repeat(34)
    loss2, lse2 = D.densenet_softmax_loss(h2, w, labels)
    dh2, dw2 = D.densenet_softmax_loss_backward(h2, w, labels, lse2)
    for a, b in ((loss, loss2), (lse, lse2), (dh, dh2), (dw, dw2)):
        assert torch.equal(a, b)
    # no row at all has a label
    labels = torch.full_like(labels, -1)
    loss, lse = D.densenet_softmax_loss(h2, w, labels)
    dh, dw = D.densenet_softmax_loss_backward(h2, w, labels, lse)
    assert not any(bool(t.any()) for t in (loss, lse, dh, dw))
    # no rows: dw is 0
    dw.fill_(7)
    D.densenet_softmax_loss_backward(h[:0], w, labels[:0], lse[:0], dw=dw)
    assert not bool(dw.any())


def test_loss_extreme_logits(D):
    """Logits of +-20000 (exponentials past fp32's range without the maximum), and words of -infinity, the type's lowest
    value and NaN in 16 bits."""
    h = torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16)
    h[:, 0] = torch.tensor([1.0, -1.0, 0.0, 1.0])
    w = torch.zeros(300, 64, device="cuda", dtype=torch.bfloat16)
    w[:, 0] = torch.linspace(-20000, 20000, 300)
    labels = torch.tensor([299, 0, 5, 100], device="cuda")
    loss, lse = D.densenet_softmax_loss(h, w, labels)
    want, wl, _, _, err = plain_loss(h, w, labels, "bf16")
    within(lse, wl, err + 2.0 ** -21 * (wl.abs() + 16), "lse")
    within(loss, want, 2 * err + 2.0 ** -20 * (wl.abs() + 16), "loss")
    low = torch.tensor(-float("inf"), device="cuda", dtype=torch.bfloat16)
    for value in (low, torch.tensor(torch.finfo(torch.bfloat16).min, device="cuda", dtype=torch.bfloat16)):
        w2 = torch.randn(300, 8, generator=gen(1), device="cuda").bfloat16()
        h2 = torch.randn(2, 8, generator=gen(2), device="cuda").bfloat16()
        h2[:, 0] = 1
        w2[7, 0] = value  # a word that no row can reach
        lab = torch.tensor([3, 299], device="cuda")
        loss, lse = D.densenet_softmax_loss(h2, w2, lab)
        logits = (h2.double() @ w2.double().T)
        within(lse, torch.logsumexp(logits, 1), torch.tensor(1e-5, device="cuda"), "lse")
        dh, dw = D.densenet_softmax_loss_backward(h2, w2, lab, lse)
        assert not bool(dw[7].any())
    w2[7, 0] = float("nan")
    loss, lse = D.densenet_softmax_loss(h2, w2, lab)
    assert bool(lse.isnan().all()) and bool(loss.isnan().all())


def test_loss_gradient_against_differences(D):
    h, w, labels = loss_case(50, 120, 400, "f32")
    has = (labels >= 0) & (labels < 400)
    _, lse = D.densenet_softmax_loss(h, w, labels)
    dh, dw = D.densenet_softmax_loss_backward(h, w, labels, lse)

    def f(h, w):
        logits = h @ w.T
        at = logits.gather(1, labels.clamp(0, 399)[:, None])[:, 0]
        return (torch.logsumexp(logits, 1) - at)[has].mean()
    g, t = gen(9), 1e-4
    for x, d, call in ((h, dh, lambda x: f(x, w.double())), (w, dw, lambda x: f(h.double(), x))):
        u = torch.randn(x.shape, generator=g, device="cuda").double()
        slope = (call(x.double() + t * u) - call(x.double() - t * u)) / (2 * t)
        assert abs(float((d.double() * u).sum() - slope)) < 1e-4 * float((d.double() * u).abs().sum())


def test_loss_on_another_stream_and_again(D):
    h, w, labels = loss_case(300, 520, 5000, "bf16")
    _, lse = D.densenet_softmax_loss(h, w, labels)
    first = D.densenet_softmax_loss_backward(h, w, labels, lse)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        _, lse2 = D.densenet_softmax_loss(h, w, labels)
        other = D.densenet_softmax_loss_backward(h, w, labels, lse2)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(lse, lse2) and torch.equal(first[0], other[0]) and torch.equal(first[1], other[1])


# ---------------------------------------------------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------------------------------------------------
K = {"lr": 3e-3, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, "weight_decay": 0.1}


def adam_tensors(sizes, p, gt, seed=0, offset=0):
    g = gen(seed)
    make = lambda dt, s: [(torch.randn(n + offset, generator=g, device="cuda") * s).to(DT[dt])[offset:] for n in sizes]  # noqa: E731
    return make(p, 0.1), make(gt, 0.01)


def plain_step(p, g, m, v, step, gs):
    g = g * gs
    m = K["beta1"] * m + (1 - K["beta1"]) * g
    v = K["beta2"] * v + (1 - K["beta2"]) * g * g
    p = p * (1 - K["lr"] * K["weight_decay"]) - K["lr"] * (m / (1 - K["beta1"] ** step)) / ((v / (1 - K["beta2"] ** step)).sqrt() + K["eps"])
    return p, m, v


@pytest.mark.parametrize("p,gt,offset,copy", [("f32", "bf16", 0, "bf16"), ("f32", "f32", 1, "f16"), ("bf16", "bf16", 0, None),
                                             ("f16", "f32", 3, None), ("bf16", "f16", 1, "bf16")])
def test_adamw_32bit(D, p, gt, offset, copy):
    sizes = [1, 7, 255, 256, 257, 2048, 2049, 5000] + [3] * 80 + [100001, 0]
    params, grads = adam_tensors(sizes, p, gt, 1, offset)
    copies = [torch.zeros(n, device="cuda", dtype=DT[copy]) for n in sizes] if copy else None
    if copy:
        copies[3] = None
    plan = D.AdamWPlan(params, grads, copies=copies)
    assert plan.state_bits == 32
    want = [(a.double(), torch.zeros(n, device="cuda").double(), torch.zeros(n, device="cuda").double()) for a, n in zip(params, sizes)]
    for step in (1, 2, 3):
        D.densenet_adamw(plan, step=step, grad_scale=0.5, **K)
        # with 16-bit parameters the next step starts from the rounded ones
        want = [plain_step(a if step == 1 or p == "f32" else q, g.double(), m, v, step, 0.5)
                for (a, m, v), g, q in zip(want, grads, held if step > 1 else want)]  # noqa: F821
        held = [t.double() for t in params]
        for i, (a, m, v) in enumerate(want):
            n, b = sizes[i], plan.blocks[i] * 256
            within(plan.m[b:b + n], m, 2.0 ** -21 * (m.abs() + 0.01), f"m of tensor {i}")
            within(plan.v[b:b + n], v, 2.0 ** -21 * (v + 1e-6), f"v of tensor {i}")
            # a step moves by about lr: its own error is some units of fp32 of that
            within(params[i], a, UNIT[p] * a.abs() * 1.01 + 2.0 ** -19 * K["lr"] * 4 + 2.0 ** -22 * a.abs() + TINY[p], f"p of tensor {i}")
            if copy and copies[i] is not None:
                within(copies[i], params[i], UNIT[copy] * params[i].double().abs() + TINY[copy], f"copy of tensor {i}")


def chance(count, seed):
    x = (np.arange(count, dtype=np.uint64) * 0x9E3779B1 + seed) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x2C1B3C6D) & 0xFFFFFFFF
    x = ((x ^ (x >> 12)) * 0x297A2D39) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    return (x >> 16).astype(np.float64) / 65536, (x & 0xFFFF).astype(np.float64) / 65536


@pytest.mark.parametrize("p,gt,offset", [("f32", "bf16", 0), ("bf16", "f32", 1)])
def test_adamw_8bit(D, p, gt, offset):
    sizes = [1, 8, 255, 256, 257, 4100] + [9] * 75 + [30001]
    params, grads = adam_tensors(sizes, p, gt, 2, offset)
    grads[3].zero_()  # a block that stays 0
    plan = D.AdamWPlan(params, grads, state_bits=8)
    want_p = [t.double() for t in params]
    for step in (1, 2, 3):
        before = [(plan.m.double().view(-1, 256) * plan.m_scale.double()[:, None]).view(-1),
                  (plan.v.double().view(-1, 256) * plan.v_scale.double()[:, None]).view(-1).square()]
        D.densenet_adamw(plan, step=step, seed=17 + step, **K)
        cm, cv = chance(plan.m.numel(), 17 + step)
        for i, n in enumerate(sizes):
            b, k = plan.blocks[i] * 256, -(-n // 256)
            a, m, v = plain_step(want_p[i], grads[i].double(), before[0][b:b + n], before[1][b:b + n], step, 1.0)
            within(params[i], a, UNIT[p] * a.abs() * 1.01 + 2.0 ** -19 * K["lr"] * 4 + 2.0 ** -22 * a.abs(), f"p of tensor {i}")
            want_p[i] = params[i].double()
            for codes, scales, t, c in ((plan.m, plan.m_scale, m, cm), (plan.v, plan.v_scale, v.sqrt(), cv)):
                whole = torch.zeros(k * 256, device="cuda", dtype=torch.float64)
                whole[:n] = t
                top = whole.view(-1, 256).abs().amax(1)
                sc = scales[b // 256:b // 256 + k].double()
                within(sc, top / 448, 2.0 ** -20 * top / 448, f"scale of tensor {i}")
                x = whole.abs() / torch.where(top > 0, top / 448, 1.0).repeat_interleave(256)
                fine = (torch.frexp(x.clamp(min=2.0 ** -6))[1].long() - 4 + 1023 << 52).view(torch.float64)  # exact powers of two
                place = x / fine + torch.from_numpy(c[b:b + k * 256]).cuda()
                q = torch.floor(place) * fine
                if codes is plan.v:
                    q = torch.where(whole > 0, q.clamp(min=2.0 ** -9), q)
                got = codes[b:b + k * 256].double()
                same = got == q * torch.sign(whole)
                # fp32 may fall on the other side only where 64 bits lie within its error of the edge
                edge = (place - place.round()).abs() < 448 * 2.0 ** -19
                edge |= (x / fine - (x / fine).round()).abs() < 448 * 2.0 ** -19
                assert bool((same | edge).all()), f"tensor {i}: {int((~(same | edge)).sum())} codes"
                assert float(same.double().mean()) > 0.99
                assert not bool(got[n:].any())
    assert not bool(plan.m[plan.blocks[3] * 256:plan.blocks[3] * 256 + 256].double().any())


def test_adamw_8bit_keeps_small_changes_on_average(D):
    """A gradient ten times as large as its past moves sqrt(v) by less than half a code: to nearest, never; here the mean
    over many values follows within five of its standard deviations."""
    n = 1 << 16
    grads = [torch.full((n,), 1.0, device="cuda")]
    grads[0][::256] = 10.0  # each block's largest value, so the others' codes lie well inside the range
    params = [torch.zeros(n, device="cuda")]
    r = torch.full((n,), 0.1 * 0.95, device="cuda")
    r[::256] = 10.0
    scale = r.view(-1, 256).amax(1) / 448
    v = (r.view(-1, 256) / scale[:, None]).to(torch.float8_e4m3fn).view(-1)
    plan = D.AdamWPlan(params, grads, m=torch.zeros(n, device="cuda").to(torch.float8_e4m3fn), v=v, m_scale=torch.zeros(n // 256, device="cuda"),
                       v_scale=scale)
    old = float((v.float()[1]) * scale[0])
    D.densenet_adamw(plan, lr=0.0, step=1, beta2=0.9999, seed=5)
    want = math.sqrt(0.9999 * old * old + 1e-4)
    got = plan.v.double() * plan.v_scale.double().repeat_interleave(256)
    got = torch.cat([got.view(-1, 256)[:, 1:].reshape(-1)])
    assert len(got.unique()) == 2
    assert abs(float(got.mean()) - want) < 5 * float(got.std()) / math.sqrt(got.numel()) + 1e-6


def test_operators_refuse(D):
    x = torch.zeros(4, 32, device="cuda")
    h, w, lab = x.bfloat16(), torch.zeros(10, 32, device="cuda").bfloat16(), torch.zeros(4, dtype=torch.int64, device="cuda")
    plan = D.AdamWPlan([x], [x.clone()])
    for call in (
            lambda: D.densenet_rms_norm(x[0]), lambda: D.densenet_rms_norm(x.double()), lambda: D.densenet_rms_norm(x.T),
            lambda: D.densenet_rms_norm(x.cpu()), lambda: D.densenet_rms_norm(x, gamma=x[0, :5]), lambda: D.densenet_rms_norm(x, residual=h),
            lambda: D.densenet_rms_norm(x, block=32), lambda: D.densenet_rms_norm(x, out_dtype=D.DN_F8, block=16),
            lambda: D.densenet_rms_norm(x, out_dtype=9), lambda: D.densenet_rms_norm(x, eps=-1.0), lambda: D.densenet_rms_norm(x, eps=float("nan")),
            lambda: D.densenet_rms_norm(x, scale=x), lambda: D.densenet_rms_norm(torch.zeros(1, 32769, device="cuda")),
            lambda: D.densenet_rms_norm(x[:, :0]),
            lambda: D.densenet_rms_norm(x[:1].expand(4, 32)),
            lambda: D.densenet_rms_norm_backward(x, h, dsum=x), lambda: D.densenet_rms_norm_backward(x[:2], x),
            lambda: D.densenet_softmax_loss(h, w[:, :16], lab), lambda: D.densenet_softmax_loss(h, w.float(), lab),
            lambda: D.densenet_softmax_loss(h, w, lab.int()), lambda: D.densenet_softmax_loss(h, w, lab[:3]),
            lambda: D.densenet_softmax_loss(h, w[:0], lab), lambda: D.densenet_softmax_loss(h, w.cpu(), lab),
            lambda: D.densenet_softmax_loss_backward(h, w, lab, x[0, :3]), lambda: D.densenet_softmax_loss_backward(h, w, lab, lab),
            lambda: D.AdamWPlan([], []), lambda: D.AdamWPlan([x], []), lambda: D.AdamWPlan([x], [x[:2]]), lambda: D.AdamWPlan([x, h], [x, x]),
            lambda: D.AdamWPlan([x], [x], copies=[x.double()]), lambda: D.AdamWPlan([x], [x], state_bits=16),
            lambda: D.AdamWPlan([x], [x], m=x), lambda: D.densenet_adamw(plan, lr=1e-3, step=0), lambda: D.densenet_adamw(plan, lr=float("inf"), step=1),
            lambda: D.densenet_adamw(plan, lr=1e-3, step=1, beta1=1.0), lambda: D.densenet_adamw(plan, lr=1e-3, step=1, eps=0.0),
            lambda: plan.set_grads([x, x])):
        with pytest.raises(D.DenseNetError):
            call()
    assert float(x.abs().max()) == 0


# ---------------------------------------------------------------------------------------------------------------------
# Together: a head on region descriptors
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt,bits", [("bf16", 8), ("f32", 32)])
def test_region_head_learns(D, dt, bits):
    from paper_1404_1869_amd.region_head import RegionHead, image_descriptors
    desc = image_descriptors(150)
    assert desc.shape == (150, 9216)
    labels = torch.arange(150, device="cuda") % 90
    labels[5] = -1
    head = RegionHead(90, 9216, dtype=D.DTYPES[dt], state_bits=bits)
    # the first step's loss and gradients against the definition (w is still the fp32 start, rounded for the products)
    a = desc.double()
    y = (a / (a.square().mean(1, keepdim=True) + 1e-6).sqrt()).to(DT[dt])
    want, _, _, _, err = plain_loss(y, head.products, labels, dt)
    first = head.step(desc, labels)
    within(first, want, 4 * err + 2 * UNIT[dt] * (y.double().abs() @ head.w.double().abs().T).amax(1) + 1e-5, "loss")
    for _ in range(15):
        last = head.step(desc, labels)
    assert float(last.mean()) < 0.9 * math.log(90)  # a tenth below a head that knows nothing
    if dt != "f32":
        assert torch.equal(head.products, head.w.to(DT[dt]))
    codes, scale = head.store(desc)
    y = a / (a.square().mean(1, keepdim=True) + 1e-6).sqrt() * head.gamma.double()
    within(codes.double() * scale.double(), y, (2.0 ** -4 + 1e-3) * y.abs() + scale.double() * 2.0 ** -9, "stored")


def test_step_in_a_graph(D):
    """A training step's calls captured in a graph: every replay, with other work between, gives what eager calls give."""
    n, C, V = 130, 264, 1000
    g = gen(8)
    x, r = torch.empty(n, C, device="cuda"), torch.empty(n, C, device="cuda")
    w, labels = rows(g, V, C, "bf16", 0, 0.1), torch.randint(-1, V, (n,), generator=g, device="cuda")
    gamma = torch.ones(C, device="cuda")

    def step(plans):
        y, s, _ = D.densenet_rms_norm(x, gamma, residual=r, out_dtype=D.DN_BF16)
        loss, lse = D.densenet_softmax_loss(y, w, labels)
        dy, dw = D.densenet_softmax_loss_backward(y, w, labels, lse, dw=plans[0].grads[0])
        dx, _ = D.densenet_rms_norm_backward(dy, s, gamma, dgamma=plans[1].grads[0])
        for p in plans:
            D.densenet_adamw(p, lr=1e-3, step=1, seed=3)
        return loss, dx, dw
    make = lambda: (D.AdamWPlan([w.clone()], [torch.zeros_like(w)], state_bits=8), D.AdamWPlan([gamma.clone()], [torch.zeros_like(gamma)]))  # noqa: E731
    plans, eager = make(), make()
    x.normal_(generator=g), r.normal_(generator=g)
    step(make())  # warm up outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(plans)
    for _ in range(4):
        x.normal_(generator=g), r.normal_(generator=g)
        graph.replay()
        want = step(eager)
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        for p, q in zip(plans, eager):
            assert torch.equal(p.params[0], q.params[0]) and torch.equal(p.m.view(torch.uint8), q.m.view(torch.uint8))


def test_loss_past_32_bit_offsets(D):
    """Weights of more than 2^31 values: the words at the end count, and get their gradient, like those at the start."""
    n, C, V = 3, 8200, 262144
    assert V * C > 2 ** 31
    g = gen(4)
    h = torch.randn(n, C, generator=g, device="cuda").bfloat16()
    w = torch.empty(V, C, device="cuda", dtype=torch.bfloat16)
    for part in w.split(16384):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * (2 / math.sqrt(C)))
    labels = torch.tensor([V - 1, 5, V - 3], device="cuda")
    loss, lse = D.densenet_softmax_loss(h, w, labels)
    logits = torch.cat([h.double() @ part.double().T for part in w.split(16384)], 1)
    err = sum_err(C) * max(float((h.double().abs() @ part.double().abs().T).max()) for part in w[:65536].split(16384)) * 1.1
    want = torch.logsumexp(logits, 1)
    bound = torch.full_like(want, 2 * err + 2.0 ** -21 * 32)
    within(lse, want, bound, "lse")
    within(loss, want - logits.gather(1, labels[:, None])[:, 0], 2 * bound, "loss")
    dh, dw = D.densenet_softmax_loss_backward(h, w, labels, lse)
    p = (logits - want[:, None]).exp()
    p.scatter_add_(1, labels[:, None], -torch.ones_like(p[:, :1]))
    p /= n
    for rng in (slice(0, 50), slice(V - 50, V)):
        ref, terms = p[:, rng].T @ h.double(), p[:, rng].abs().T @ h.double().abs()
        within(dw[rng], ref, UNIT["bf16"] * ref.abs() * 1.01 + (UNIT["bf16"] + 4 * err + 1e-5) * terms, "dw")
    ref = sum(p[:, i:i + 16384] @ w[i:i + 16384].double() for i in range(0, V, 16384))
    terms = sum(p[:, i:i + 16384].abs() @ w[i:i + 16384].double().abs() for i in range(0, V, 16384))
    within(dh, ref, UNIT["bf16"] * ref.abs() * 1.01 + (UNIT["bf16"] + 4 * err + sum_err(V)) * terms, "dh")


FEW = [(3000, 264, 21, "bf16"), (700, 1000, 33, "f16"), (2500, 100, 64, "f32"), (300, 9216, 20, "f32"), (65, 130, 65, "f32"),
       (200, 72, 32, "f32"), (64, 257, 3000, "f32"), (33, 1024, 40, "bf16"), (500, 300, 2048, "f32"), (450, 96, 1500, "f32")]


@pytest.mark.parametrize("n,C,V,dt", FEW)
def test_few_words_or_rows(D, n, C, V, dt):
    """Shapes around those where the logits change tiles or the layout of fp32 operands: 32, 64 and 400 rows, 32 and 64 words."""
    test_loss(D, n, C, V, dt, 0, 0)
    test_loss_gradient(D, n, C, V, dt, 0, 0, True)
    test_loss_gradient(D, n, C, V, dt, 1, 1, False)


@pytest.mark.parametrize("n,C,V,dt", [(4200, 4096, 300, "bf16"), (2100, 4096, 40, "f32"), (40, 2048, 3000, "f32")])
def test_masked_rows_of_a_large_batch(D, n, C, V, dt):
    """As test_masked_rows_reach_nothing, where h is read as it lies unless a masked row holds an infinity or a NaN."""
    h, w, labels = loss_case(n, C, V, dt)
    has = (labels >= 0) & (labels < V)
    _, lse = D.densenet_softmax_loss(h, w, labels)
    dh, dw = D.densenet_softmax_loss_backward(h, w, labels, lse)
    for value in (float("nan"), float("-inf"), 1e4):
        h2 = h.clone()
        h2[int((~has).nonzero()[-1]), C - 1] = value
        dh2, dw2 = D.densenet_softmax_loss_backward(h2, w, labels, lse)
        assert torch.equal(dh, dh2) and torch.equal(dw, dw2)
    test_loss_gradient(D, n, C, V, dt, 0, 0, True)


def test_outputs_with_strides_leave_the_rest(D):
    """Results written into columns of wider buffers: the columns beside them stay as they were."""
    n, C, V = 70, 131, 300
    g = gen(6)
    x, r = rows(g, n, C, "bf16", 5), rows(g, n, C, "bf16", 2)
    wide = lambda rows_, dt: torch.full((rows_ + 1, C + 3), 7.0, device="cuda").to(dt)  # noqa: E731
    y, s, q, dx, dh, dw = (wide(k, torch.bfloat16) for k in (n, n, n, n, n, V))
    q = wide(n, torch.float8_e4m3fn)
    cut = lambda t, k=n: t[:k, 1:1 + C]  # noqa: E731
    D.densenet_rms_norm(x, residual=r, out=cut(y), sum_out=cut(s))
    D.densenet_rms_norm(x, residual=r, out=cut(q), out_dtype=D.DN_F8, block=32)
    D.densenet_rms_norm_backward(r, x, dx=cut(dx))
    w, labels = rows(g, V, C, "bf16", 4, 0.1), torch.randint(-1, V, (n,), generator=g, device="cuda")
    _, lse = D.densenet_softmax_loss(x, w, labels)
    D.densenet_softmax_loss_backward(x, w, labels, lse, dh=cut(dh), dw=cut(dw, V))
    a, b, _ = D.densenet_rms_norm(x, residual=r)
    c, _, _ = D.densenet_rms_norm(x, residual=r, out_dtype=D.DN_F8, block=32)
    e, _ = D.densenet_rms_norm_backward(r, x)
    h, v = D.densenet_softmax_loss_backward(x, w, labels, lse)
    for t, want in ((y, a), (s, b), (q, c), (dx, e), (dh, h), (dw, v)):
        k = want.shape[0]
        assert torch.equal(t[:k, 1:1 + C].float(), want.float())
        rest = t.float().clone()
        rest[:k, 1:1 + C] = 7
        assert bool((rest == 7).all())


@pytest.mark.parametrize("n,C,V,dt", [(1, 4096, 2000, "bf16"), (64, 1024, 30000, "f16"), (300, 96, 777, "bf16"), (1001, 300, 5003, "f32"),
                                      (200, 264, 3000, "f32"), (20, 512, 4000, "f32"), (3000, 264, 21, "f32"), (9000, 130, 500, "bf16"),
                                      (4200, 4096, 300, "bf16")])
def test_workspace_is_enough(D, n, C, V, dt):
    """The calls stay within the workspace that their size queries ask for."""
    import ctypes
    h, w, labels = loss_case(n, C, V, dt)
    L, code, st = D.lib(), D.DTYPES[dt], D._on(h.device)
    need = ctypes.c_size_t()
    out = [torch.empty(n, device="cuda") for _ in range(2)]
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    ops = (h.data_ptr(), C, w.data_ptr(), C, labels.data_ptr())
    dims = (n, C, V, code)
    calls = ((L.densenet_softmax_loss, (*ops, *dims, out[0].data_ptr(), out[1].data_ptr())),
             (L.densenet_softmax_loss_backward, (*ops, out[1].data_ptr(), None, 1.0, *dims, dh.data_ptr(), C, dw.data_ptr(), C)))
    for call, args in calls:
        D.check(call(*args, None, 0, ctypes.byref(need), st))
        work = torch.full((need.value + 4096,), 165, dtype=torch.uint8, device="cuda")
        D.check(call(*args, work.data_ptr(), need.value, ctypes.byref(need), st))
        assert bool((work[need.value:] == 165).all())
        assert call(*args, work.data_ptr(), need.value - 1, ctypes.byref(need), st) == D.DN_E_BUFFER_TOO_SMALL
    assert all(bool(t.isfinite().all()) for t in (*out, dh, dw))


@pytest.mark.parametrize("n,C,V", [(4, 64, 300), (4, 4096, 300), (200, 4096, 40), (300, 64, 5000), (300, 4096, 300)])
def test_loss_of_rows_that_are_sure(D, n, C, V):
    """Labels whose logits lead by 8 among logits of a hundred: the loss (about V e^-8) keeps its digits, in all paths of the
    join.  The logits are exact (one value of a row, integers and eighths), so the bound is the softmax's own: a few units of
    fp32 of the loss and of the exponentials, not of the logits."""
    h = torch.zeros(n, C, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros(V, C, device="cuda", dtype=torch.bfloat16)
    h[:, 0] = 8
    w[:, 0] = torch.randint(90, 97, (V,), generator=gen(1), device="cuda").bfloat16() / 8
    labels = torch.randint(0, V, (n,), generator=gen(2), device="cuda")
    labels[:] = labels[0]
    w[labels[0], 0] = 13  # 104, at least 8 above the others
    loss, _ = D.densenet_softmax_loss(h, w, labels)
    logits = h.double() @ w.double().T
    want = torch.logsumexp(logits, 1) - logits.gather(1, labels[:, None])[:, 0]
    assert 0 < float(want.min()) < 1
    within(loss, want, 2.0 ** -20 * (want + 0.1), "loss")


@pytest.mark.parametrize("drop", [0, 10, 16, 24])
def test_fp32_values_far_below_their_rows_largest(D, drop):
    """fp32 logits from two fp16 parts: a value of 2^-drop to 2^-(drop + 1) of its row's largest, which meets a zero weight,
    keeps 22 bits, or is off by half of fp16's smallest step, 2^-25, where the largest is scaled to 2^13 at least: 2^-38 of
    it.  Each product is off by that of either factor (w's one value is its row's largest)."""
    rel = max(2.0 ** -22, 2.0 ** (drop + 1 - 38))
    n, C, V = 100, 16, 200
    g = gen(drop)
    h, w = torch.zeros(n, C, device="cuda"), torch.zeros(V, C, device="cuda")
    h[:, 0] = 1 + torch.rand(n, generator=g, device="cuda")
    h[:, 5] = h[:, 0] * 2.0 ** -drop * (1 + torch.rand(n, generator=g, device="cuda")) / 2
    w[:, 5] = 2.0 ** drop * (20 + 40 * torch.rand(V, generator=g, device="cuda"))
    labels = torch.randint(0, V, (n,), generator=g, device="cuda")
    _, lse = D.densenet_softmax_loss(h, w, labels)
    logits = h.double() @ w.double().T
    want = torch.logsumexp(logits, 1)
    within(lse, want, (rel + 2.0 ** -22 + 2.0 ** -23) * 1.01 * logits.amax(1) + 2.0 ** -22 * want, "lse")


@pytest.mark.parametrize("n", [3, 100, 500])
def test_fp32_words_of_the_lowest_value(D, n):
    """A word masked by fp32's lowest value, in each layout of fp32 operands (as they lie, three parts, two and three): no row
    reaches it, and the gradients of the others are what they are without it."""
    C, V = 72, 200
    h, w, labels = loss_case(n, C, V, "f32", masked=0.0)
    h[:, 0] = 0.5
    labels[labels == 7] = 8
    keep = [v for v in range(V) if v != 7]
    w[7] = 0
    w[7, 0] = torch.finfo(torch.float32).min
    loss, lse = D.densenet_softmax_loss(h, w, labels)
    dh, dw = D.densenet_softmax_loss_backward(h, w, labels, lse)
    assert not bool(dw[7].any())
    want, wl, _, _, err = plain_loss(h, w[keep], labels - (labels > 7).long(), "f32")
    within(lse, wl, 2 * err + 2.0 ** -21 * (wl.abs() + 16), "lse")
    p = torch.exp(h.double() @ w.double().T - wl[:, None])
    p.scatter_add_(1, labels[:, None], -torch.ones_like(p[:, :1]))
    p /= n
    tol = 2 * err.max() + 2.0 ** -20
    within(dh, p @ w.double(), (tol + 6 * sum_err(V)) * (p[:, keep].abs() @ w[keep].double().abs()) + 1e-30, "dh")
    within(dw, p.T @ h.double(), (tol + 6 * sum_err(n)) * (p.abs().T @ h.double().abs()) + 1e-30, "dw")
