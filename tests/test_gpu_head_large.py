"""The head's operators on batches of more rows than one launch has threads for: HIP counts a launch's threads in 32 bits,
and runs fewer workgroups than asked past that.  Values repeat with a period that divides nothing, so every row's result is
that of a small batch at its place in the period, to the bit."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PERIOD = 1009


@pytest.fixture(scope="module")
def D():
    from paper_1404_1869_amd import densenet
    assert torch.cuda.is_available()
    densenet.lib()
    return densenet


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def cycle(base, n):
    """Rows of `base` over and over, n in all."""
    out = torch.empty((n, *base.shape[1:]), dtype=base.dtype, device="cuda")
    for i in range(0, n, PERIOD * 1024):
        part = out[i:i + PERIOD * 1024]
        part.copy_(base.repeat(-(-len(part) // PERIOD), *[1] * (base.dim() - 1))[:len(part)])
    return out


def same_cycle(got, base, what):
    for i in range(0, len(got), PERIOD * 1024):
        part = got[i:i + PERIOD * 1024]
        want = base.repeat(-(-len(part) // PERIOD), *[1] * (base.dim() - 1))[:len(part)]
        assert torch.equal(part.view(torch.uint8), want.view(torch.uint8)), f"{what}: rows {i} on"


@pytest.mark.parametrize("n,C,out,block,res", [((1 << 26) + 5, 16, "bf16", 0, True), ((1 << 26) + 5, 8, "f8", 0, False),
                                              ((1 << 26) + 5, 40, "f8", 32, False), ((1 << 32) // 192 + 77, 2049, "f8", 0, False)])
def test_norm_of_many_rows(D, n, C, out, block, res):
    """A wave per row (64 threads), and a workgroup of 192 per row: 2^26 rows of the one and 2^32 / 192 of the other end a launch."""
    base = torch.randn(PERIOD, C, generator=gen(1), device="cuda").bfloat16()
    other = torch.randn(PERIOD, C, generator=gen(2), device="cuda").bfloat16() if res else None
    kind = {"bf16": D.DN_BF16, "f8": D.DN_F8}[out]
    want = D.densenet_rms_norm(base, residual=other, out_dtype=kind, block=block)
    x = cycle(base, n)
    r = cycle(other, n) if res else None
    got = D.densenet_rms_norm(x, residual=r, out_dtype=kind, block=block)
    for g, w, what in zip(got, want, ("y", "sum", "scale")):
        assert (g is None) == (w is None)
        if g is not None:
            same_cycle(g, w, what)


def base_loss(h, w, labels, times):
    """64-bit loss of a period's rows; times: how often each word stands in the vocabulary."""
    logits = h.double() @ w.double().T
    lse = torch.logsumexp(logits + times.double().log(), 1)
    return logits, lse


@pytest.mark.parametrize("n,C,V,dt", [((1 << 24) + 3, 8, 100, "f32"), ((1 << 26) + 5, 8, 10, "bf16"), ((1 << 26) + 5, 8, 10, "f32"),
                                      ((1 << 23) + 1, 8, 300, "f16")])
def test_loss_of_many_rows(D, n, C, V, dt):
    """Rows in two fp16 parts (a workgroup each), looked through for masked infinities and joined by waves, and the forward
    pass in pieces of rows.  Bounds: a logit of 8 products, 2^-20 of their magnitudes; the softmax 2^-20; a result's own unit."""
    kind = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dt]
    unit = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dt]
    h, w = torch.randn(PERIOD, C, generator=gen(1), device="cuda").to(kind), torch.randn(V, C, generator=gen(2), device="cuda").to(kind)
    labels = torch.randint(-1, V, (PERIOD,), generator=gen(3), device="cuda")
    labels[4] = -1  # the last row's, for n of 2^26 + 5 among others
    has = labels >= 0
    logits, lse = base_loss(h, w, labels, torch.ones(V, device="cuda"))
    at = logits.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    err = 2.0 ** -19 * ((h.double().abs() @ w.double().abs().T).amax(1) + 16)
    H, L = cycle(h, n), cycle(labels, n)
    gone = int((L < 0).nonzero()[-1])
    H[gone] = float("nan")
    got, sums = torch.full((n,), -7.0, device="cuda"), torch.full((n,), -7.0, device="cuda")
    D.densenet_softmax_loss(H, w, L, loss=got, lse=sums)
    step = PERIOD * 1024

    def whole(base, k):
        return base.repeat(-(-k // PERIOD), *[1] * (base.dim() - 1))[:k]
    for i in range(0, n, step):
        k = min(step, n - i)
        for t, want in ((got, torch.where(has, lse - at, 0.0)), (sums, torch.where(has, lse, 0.0))):
            assert bool(((t[i:i + k].double() - whole(want, k)).abs() <= whole(err, k)).all()), f"rows {i} on"
    # the gradient of the mean, times a scale that brings a row's share back to about 1
    dh, dw = torch.full((n, C), 7.0, device="cuda", dtype=kind), torch.full((V, C), 7.0, device="cuda", dtype=kind)
    D.densenet_softmax_loss_backward(H, w, L, sums, scale=float(n), dh=dh, dw=dw)
    c = n / int((L >= 0).sum())
    g = torch.exp(logits - lse[:, None])
    g.scatter_add_(1, labels.clamp(min=0)[:, None], -torch.ones_like(g[:, :1]))
    g *= torch.where(has, c, 0.0)[:, None]
    want = g @ w.double()
    bound = unit * want.abs() * 1.01 + (unit + err[:, None] * 4 + 2.0 ** -18) * (g.abs() @ w.double().abs()) + 2.0 ** -24
    for i in range(0, n, step):
        k = min(step, n - i)
        assert bool(((dh[i:i + k].double() - whole(want, k)).abs() <= whole(bound, k)).all()), f"dh of rows {i} on"
    if dt == "f16":  # (times n, past fp16's range)
        _, dw = D.densenet_softmax_loss_backward(H, w, L, sums)
        g /= n
    times = torch.full((PERIOD, 1), float(n // PERIOD), device="cuda", dtype=torch.float64)
    times[:n % PERIOD] += 1
    ref, terms = (g * times).T @ h.double(), (g.abs() * times).T @ h.double().abs()
    # running sums of n rows in 32 bits: roundings of either sign, sqrt(n / 8) 2^-24 of the whole is 2^-13
    assert bool(((dw.double() - ref).abs() <= unit * ref.abs() * 1.01 + (unit + 2.0 ** -10) * terms).all())


def test_loss_over_many_words(D):
    """fp32 words in two fp16 parts, a workgroup each, of 2^24 + 3 words."""
    n, C, V = 100, 8, (1 << 24) + 3
    h, w = torch.randn(n, C, generator=gen(1), device="cuda"), torch.randn(PERIOD, C, generator=gen(2), device="cuda")
    labels = torch.randint(V - 50, V, (n,), generator=gen(3), device="cuda")
    times = torch.full((PERIOD,), float(V // PERIOD), device="cuda", dtype=torch.float64)
    times[:V % PERIOD] += 1
    logits, lse = base_loss(h, w, labels % PERIOD, times)
    at = logits.gather(1, (labels % PERIOD)[:, None])[:, 0]
    err = 2.0 ** -19 * ((h.double().abs() @ w.double().abs().T).amax(1) + 16)
    W = cycle(w, V)
    loss, sums = D.densenet_softmax_loss(h, W, labels)
    assert bool(((loss.double() - (lse - at)).abs() <= err).all()) and bool(((sums.double() - lse).abs() <= err).all())
    dw = torch.full((V, C), 7.0, device="cuda")
    D.densenet_softmax_loss_backward(h, W, labels, sums, scale=2.0 ** 24, dw=dw)
    p = torch.exp(logits - lse[:, None]) * (2.0 ** 24 / n)
    ref, terms = p.T @ h.double(), p.T @ h.double().abs()
    bound = terms * (4 * float(err.max()) + 2.0 ** -18)
    kept = torch.ones(V, dtype=torch.bool, device="cuda")
    kept[labels] = False
    for i in range(0, V, PERIOD * 1024):
        part = dw[i:i + PERIOD * 1024]
        off = (part.double() - ref.repeat(-(-len(part) // PERIOD), 1)[:len(part)]).abs()
        good = off <= bound.repeat(-(-len(part) // PERIOD), 1)[:len(part)]
        assert bool((good.all(1) | ~kept[i:i + len(part)]).all()), f"dw of words {i} on"


def test_adamw_of_a_tensor_past_a_launch(D):
    """2^24 workgroups of 2048 values end a launch: a tensor of 2^35 + 5000 16-bit values, states in 8 bits (194 GB).  All
    values are alike, so all parameters and all codes have to be."""
    n = (1 << 35) + 5000
    if torch.cuda.mem_get_info()[0] < 205 << 30:
        pytest.skip("needs 205 GiB")
    make = lambda k: ([torch.full((k,), 1.0, dtype=torch.bfloat16, device="cuda")], [torch.full((k,), 0.5, dtype=torch.bfloat16, device="cuda")])  # noqa: E731
    small, large = (D.AdamWPlan(*make(k), state_bits=8) for k in (256, n))
    for plan in (small, large):
        D.densenet_adamw(plan, lr=0.125, step=1, seed=3)
    step = 1 << 30
    for what in ("p", "m", "v", "m_scale", "v_scale"):
        got, want = (plan.params[0] if what == "p" else getattr(plan, what) for plan in (large, small))
        got, want = (t.view(torch.uint8) if t.element_size() == 1 else t for t in (got, want))
        value, off = float(want[0]), int((want != want[0]).sum())
        assert off == 0 and value not in (0, 1)
        got = got[:n] if what in "pmv" else got
        for i in range(0, len(got), step):
            off = int((got[i:i + step] != want[0]).sum())  # (not in the assertion, whose report would go through the values)
            assert off == 0, f"{what}: {off} values of {i} on"


def test_binding_refuses_sizes_past_32_bits(D):
    """C and V are 32-bit arguments: sizes of 2^32 and some must not pass as the some."""
    words = torch.empty((1 << 32) + 5, 1, dtype=torch.bfloat16, device="cuda")
    h, labels = torch.zeros(3, 1, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    lse = torch.zeros(3, device="cuda")
    row = words[:(1 << 32) + 3].view(1, -1)
    for call in (lambda: D.densenet_softmax_loss(h, words, labels), lambda: D.densenet_softmax_loss_backward(h, words, labels, lse, dw=words),
                 lambda: D.densenet_rms_norm(row, out=row), lambda: D.densenet_rms_norm_backward(row, row, dx=row),
                 lambda: D.densenet_softmax_loss(row, row, labels[:1])):
        with pytest.raises(D.DenseNetError) as e:
            call()
        assert e.value.status == D.DN_E_TOO_LARGE
