"""The head's operators where their numbers run out of range: weights of rows far apart or next to nothing, infinities among
words, batches that the gradient takes in pieces.  Against plain forms in 64 bits; tolerances as in test_gpu_head.py."""
import math

import pytest

torch = pytest.importorskip("torch")
import test_gpu_head as base  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}


@pytest.fixture(scope="module")
def D():
    from paper_1404_1869_amd import densenet
    assert torch.cuda.is_available()
    densenet.lib()
    return densenet


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dt="f32", scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(DT[dt])


def sum_err(k):
    return (k / 8 + 16) * 2.0 ** -24


def within(got, want, bound, what):
    got, want = got.double(), want.double()
    off = (got - want).abs()
    bad = int((~(off <= bound)).sum())
    assert bad == 0, f"{what}: {bad} of {off.numel()} off, by up to {float((off / bound).max()):.2f} bounds"


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("weight", [1e-45, 1e-38, 2.9e-36, 1e-30, 1.0, 1e30, 3e38])
def test_weights_of_any_size(D, dt, weight):
    """Rows' weights (dloss) from fp32's smallest to its largest value: gradients are finite, and those of weight 1 times it.
    `scale` brings them back where it can.  g: its rounding (fp16: 2^-25 of values 2^10 times the weights over the largest, or
    2^126 times the weights where that is less), and the exponent's error."""
    n, C, V = 70, 64, 100
    g = gen(1)
    h, w = normal(g, n, C, dt=dt), normal(g, V, C, dt=dt, scale=0.5)
    labels = torch.randint(0, V, (n,), generator=g, device="cuda")
    _, lse = D.densenet_softmax_loss(h, w, labels)
    part = torch.rand(n, generator=g, device="cuda") * 0.5 + 0.5
    part[3] = 1
    dloss = part * weight
    scale = max(1.2e-38, min(1e38, 1 / weight))
    c = dloss.double() * scale  # (as fp32 holds the weights: the smallest are 0 or one step)
    dh, dw = D.densenet_softmax_loss_backward(h, w, labels, lse, dloss=dloss, scale=scale)
    assert bool(dh.isfinite().all()) and bool(dw.isfinite().all())
    p = torch.exp(h.double() @ w.double().T - lse.double()[:, None]) * c[:, None]
    d = p.clone()
    d[torch.arange(n, device="cuda"), labels] -= c
    err = (6 if dt == "f32" else 1) * sum_err(C) * (h.double().abs() @ w.double().abs().T).amax(1)
    off = (2.0 ** -22 if dt == "f32" else UNIT[dt]) * d.abs() + p * (2 * err + 2.0 ** -22 * (lse.double().abs() + 40))[:, None]
    off = off + (2.0 ** -25 * max(2.0 ** -126 * scale, 2.0 ** -10 * float(c.max())) if dt == "f16" else 0)
    many = 6 if dt == "f32" else 1
    for got, a, b, e, k, what in ((dh, d, w.double(), off, V, "dh"), (dw, d.T, h.double(), off.T, n, "dw")):
        want = a @ b
        within(got, want, UNIT[dt] * want.abs() * 1.01 + e @ b.abs() + many * sum_err(k) * (a.abs() @ b.abs()) + TINY[dt], what)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_rows_of_light_weight_keep_their_gradient(D, dt):
    """Weights from 1 to 1e-7 in one call, a vocabulary of 20000 words with a common mean, so that what g's small values add
    up to is most of a row of dh.  Each row to its own size: half a unit of g, or half of fp16's smallest step of g times 2^14 over
    the largest weight.  A call for each decade, whose `scale` brings its rows into fp16's range."""
    n, C, V = 64, 64, 20000
    g = gen(5)
    w = (normal(g, V, C, scale=0.1) + normal(g, C)).to(DT[dt])
    h, labels = normal(g, n, C, dt=dt, scale=0.1), torch.randint(0, V, (n,), generator=g, device="cuda")
    dloss = torch.logspace(0, -7, n, device="cuda")
    _, lse = D.densenet_softmax_loss(h, w, labels)
    p = torch.exp(h.double() @ w.double().T - lse.double()[:, None]) * dloss.double()[:, None]
    d = p.clone()
    d[torch.arange(n, device="cuda"), labels] -= dloss.double()
    err = sum_err(C) * (h.double().abs() @ w.double().abs().T).amax(1)
    off = UNIT[dt] * d.abs() + p * (2 * err + 2.0 ** -22 * (lse.double().abs() + 40))[:, None]
    if dt == "f16":
        off = off + 2.0 ** -25 * 2.0 ** -14
    for decade in range(8):
        scale = 10.0 ** decade
        dh, _ = D.densenet_softmax_loss_backward(h, w, labels, lse, dloss=dloss, scale=scale)
        rows = (dloss * scale > 0.3) & (dloss * scale <= 3.001)
        want = d[rows] @ w.double() * scale
        bound = UNIT[dt] * want.abs() * 1.01 + scale * (off[rows] @ w.double().abs() + sum_err(V) * (d[rows].abs() @ w.double().abs())) + TINY[dt]
        within(dh[rows], want, bound, f"dh of weights around 1e-{decade}")


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_region_head_gradients(D, dt):
    """The first step's gradients of 2000 rows of 9216 over 20000 words, whose mean leaves values below fp16's smallest.  Off, as
    a whole, by some roundings of terms of either sign: eight of `dt`'s (fp32: of 2^-20)."""
    from paper_1404_1869_amd.region_head import RegionHead
    n, C, V = 2000, 9216, 20000
    desc = torch.relu(normal(gen(1), n, C, scale=2.0))
    labels = torch.randint(-1, V, (n,), generator=gen(2), device="cuda")
    head = RegionHead(V, C, dtype=D.DTYPES[dt], state_bits=32)
    y, _, _ = D.densenet_rms_norm(desc, head.gamma, eps=head.eps, out_dtype=D.DTYPES[dt])
    w, start = head.products.clone(), head.w.clone()
    head.step(desc, labels)
    has = labels >= 0
    p = torch.softmax(y.double() @ w.double().T, 1)
    p.scatter_add_(1, labels.clamp(min=0)[:, None], torch.full_like(p[:, :1], -1.0))
    p *= (has.double() / int(has.sum()))[:, None]
    dw = p.T @ y.double()
    s = desc.double()
    dgamma = ((p @ w.double()) * s / (s.square().mean(1, keepdim=True) + head.eps).sqrt()).sum(0)
    scale = getattr(head, "scale", 1.0)
    for got, want, what in ((head.dw, dw, "dw"), (head.dgamma, dgamma, "dgamma")):
        off = float((got.double() / scale - want).norm() / want.norm())
        assert off < 8 * max(UNIT[dt], 2.0 ** -20), f"{what} off by {off:.1e}"
    # and the optimiser takes the scale back: m = (1 - beta1) gradient
    m = head.plans[0].m[:V * C].view(V, C)
    assert float((m.double() / 0.1 - dw).norm() / dw.norm()) < 8 * max(UNIT[dt], 2.0 ** -20)
    assert not torch.equal(head.w, start)


@pytest.mark.parametrize("n,V", [(10, 200), (100, 60), (100, 200), (300, 3000), (500, 1000)])
def test_fp32_words_of_minus_infinity(D, n, V):
    """Words masked by -infinity in one value (h is positive there), in every layout of fp32 operands: no row reaches them, and
    the loss is that of the other words.  Where it is one of theirs that is the label, the loss is infinite; a word of +infinity
    and a NaN make it NaN."""
    C = 72
    g = gen(n)
    h, w = normal(g, n, C), normal(g, V, C, scale=0.3)
    h[:, 5] = h[:, 5].abs() + 0.1
    gone = torch.arange(7, V, 13, device="cuda")
    keep = torch.ones(V, dtype=torch.bool, device="cuda")
    keep[gone] = False
    labels = keep.nonzero()[torch.randint(0, int(keep.sum()), (n,), generator=g, device="cuda"), 0]
    w[gone, 5] = -math.inf
    loss, lse = D.densenet_softmax_loss(h, w, labels)
    logits = h.double() @ w[keep].double().T
    want = torch.logsumexp(logits, 1)
    at = (h.double() * w[labels].double()).sum(1)
    err = 6 * sum_err(C) * (h.double().abs() @ w[keep].double().abs().T).amax(1)
    tol = 2 * err + 2.0 ** -21 * (want.abs() + 16)
    within(lse, want, tol, "lse")
    within(loss, want - at, 2 * tol, "loss")
    if n > 64 and V > 64:  # (as they lie, dh holds 0 times -infinity; in two parts g is 0 and so is the word's gradient)
        _, dw = D.densenet_softmax_loss_backward(h, w, labels, lse)
        assert n < 400 or not bool(dw[gone].any())
    one = labels.clone()
    one[3] = int(gone[0])
    loss, lse2 = D.densenet_softmax_loss(h, w, one)
    assert float(loss[3]) == math.inf and bool(loss.isfinite().sum() == n - 1) and torch.equal(lse, lse2)
    w[gone[0], 5] = math.inf
    loss, _ = D.densenet_softmax_loss(h, w, labels)
    assert not bool(loss.isfinite().any())
    w[gone[0], 5] = math.nan
    loss, _ = D.densenet_softmax_loss(h, w, labels)
    assert bool(loss.isnan().all())
    w[gone, 5] = 0
    h[4, 9] = math.inf
    loss, _ = D.densenet_softmax_loss(h, w, labels)
    assert not bool(loss[4].isfinite()) and int(loss.isfinite().sum()) == n - 1


@pytest.mark.parametrize("n,C,V,dt,per_row", [(20000, 40, 30000, "bf16", False), (17000, 72, 20011, "f16", True), (20000, 24, 15013, "f32", True),
                                              (64, 24, 2100000, "f32", False), (100, 16, 2700000, "f32", True), (40, 16, 7000003, "bf16", True)])
def test_gradient_in_pieces_of_the_vocabulary(D, n, C, V, dt, per_row):
    """More words than one piece of g holds (2^28 values in 16 bits; fp32 of few rows 2^27), in each layout: labels, factors and
    sums go on from piece to piece."""
    torch.cuda.empty_cache()
    assert n * V > 1 << (27 if dt == "f32" and n <= 64 else 28)
    base.test_loss_gradient(D, n, C, V, dt, 0, 0, per_row)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [100, 450])
def test_fp32_gradient_holds_fp32(D, n):
    """dh and dw of fp32 to 2^-21 of their terms, which takes all six products of the bf16 parts (of each of the three smaller
    ones some terms hold over 2^-20).  Row i's softmax is all on word i (logits 256 and 0), its label is word i + 1, so g is
    +-dloss in two places; words and rows meet in columns of their own.  What is left out is below 2^-24; the sums of a result's two
    terms, and its factor, round six times to 2^-24."""
    K = 64
    g = gen(n)
    h, w = torch.zeros(n, n + 2 * K, device="cuda"), torch.zeros(n, n + 2 * K, device="cuda")
    at = torch.arange(n, device="cuda")
    h[at, at] = w[at, at] = 16
    w[:, n:n + K], h[:, n + K:] = normal(g, n, K), normal(g, n, K)
    labels, dloss = (at + 1) % n, normal(g, n)
    dh, dw = D.densenet_softmax_loss_backward(h, w, labels, torch.full((n,), 256.0, device="cuda"), dloss=dloss)
    c, W, H = dloss.double()[:, None], w.double(), h.double()
    want, terms = c * (W - W[labels]), c.abs() * (W.abs() + W[labels].abs())
    within(dh, want, 2.0 ** -21 * terms, "dh")
    want, terms = c * H, (c * H).abs()
    back = (at - 1) % n  # the row whose label the word is
    within(dw, want - want[back], 2.0 ** -21 * (terms + terms[back]), "dw")


def test_infinite_gradient_spoils_its_own_value_only(D):
    """8-bit states share a scale: an infinite (and a NaN) gradient must not reach its block's other values, in the step itself or
    in those that follow from the states."""
    n = 700
    g = gen(3)
    p, grads = normal(g, n), [normal(g, n, scale=0.01) for _ in range(3)]
    grads[0][[5, 300, 699]] = 0
    runs = []
    for values in ((0.0, 0.0, 0.0), (math.inf, math.nan, -math.inf)):
        plan = D.AdamWPlan([p.clone()], [grads[0].clone()], state_bits=8)
        for i, x in zip((5, 300, 699), values):
            plan.grads[0][i] = x
        for step in (1, 2, 3):
            if step > 1:
                plan.grads[0].copy_(grads[step - 1])
                plan.grads[0][[5, 300, 699]] = 0
            D.densenet_adamw(plan, lr=1e-2, step=step, seed=step)
        runs.append((plan.params[0], plan.m.view(torch.uint8)[:n], plan.v.view(torch.uint8)[:n], plan.m_scale, plan.v_scale))
    kept = torch.ones(n, dtype=torch.bool, device="cuda")
    kept[[5, 300, 699]] = False
    for a, b in zip(*runs):
        kept_of = kept if len(a) == n else slice(None)
        assert torch.equal(a[kept_of], b[kept_of])
    assert bool(runs[1][0][~kept].isnan().all()) and bool(runs[0][0].isfinite().all())
