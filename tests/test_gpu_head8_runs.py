"""The operators of a head in 8 bits together and away from the usual call: a training step against its definition in 64 bits, steps
captured in graphs and replayed, on streams of their own, two at once, the head that trains and answers with them, and places past
2^31 elements."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def D():
    from paper_1404_1869_amd import densenet
    assert torch.cuda.is_available()
    densenet.lib()
    return densenet


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def same(a, b):
    if a is None or b is None:
        return a is b
    if a.dtype == F8:
        a, b = a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)
    return torch.equal(a, b)


def wide(codes, scale, rows):
    n, C = codes.shape
    k = scale.double().repeat_interleave(128, 1)[:, :C]
    return codes.double() * (k if rows == 1 else k.repeat_interleave(128, 0)[:n])


def step(D, x, gamma, w, tokens, dlogp, dH, muon=None, top=3):
    """Norm, logits, scores, their gradient, and the gradients of the rows and of w, all products from 8-bit operands."""
    y, _, _ = D.densenet_rms_norm(x, gamma, out_dtype=D.DN_F32)
    q = D.densenet_quantize_blocks(y)
    qt = D.densenet_quantize_blocks(y, rows=128, codes=False, turned=True)
    w8 = D.densenet_quantize_blocks(w, rows=128, turned=True)
    logits = D.densenet_block_product(q[0], q[1], w8[0], w8[1], out_dtype=D.DN_F32)
    s = D.densenet_token_scores(logits, tokens, top=top)
    g = D.densenet_token_scores_backward(logits, tokens, s[2], entropy=s[1], dlogp=dlogp, dentropy=dH)
    g8 = D.densenet_quantize_blocks(g, turned=True)
    dy = D.densenet_block_product(g8[0], g8[1], w8[2], w8[3], out_dtype=D.DN_F32)
    dw = D.densenet_block_product(g8[2], g8[3], qt[2], qt[3], out_dtype=D.DN_F32)
    dx, dgamma = D.densenet_rms_norm_backward(dy, x, gamma)
    if muon is not None:
        muon.grads[0].copy_(dw)
        D.densenet_muon(muon, lr=0.01)
    return dict(y=y, q=q[0], qk=q[1], qt=qt[2], qtk=qt[3], w8=w8[0], wk=w8[1], wt=w8[2], wtk=w8[3], logits=logits, logp=s[0], H=s[1], lse=s[2],
                ids=s[3], best=s[4], g=g, g8=g8[0], gk=g8[1], gt=g8[2], gtk=g8[3], dy=dy, dw=dw, dx=dx, dgamma=dgamma)


def inputs(seed, n=150, C=300, V=700):
    g = gen(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return (r(n, C), 1 + 0.1 * r(C), 0.1 * r(V, C), torch.randint(-1, V, (n,), generator=g, device="cuda"), r(n) / n, 0.1 * r(n) / n)


def test_training_step(D):
    """Each product against its own operands' values (a sum of K products: (K / 8 + 16) 2^-24 of their magnitudes), and the gradients
    against those of the same step without 8-bit operands, whose codes are off by 2^-4 of a value, at random: over K of them a product
    is off by about 2^-4 / sqrt(3) of its operands' root-mean-square product times sqrt(K), for each of two rounded operands; five
    times that is never reached."""
    x, gamma, w, tokens, dlogp, dH = inputs(3)
    o = step(D, x, gamma, w, tokens, dlogp, dH)
    for y, a, ak, b, bk in (("logits", "q", "qk", "w8", "wk"), ("dy", "g8", "gk", "wt", "wtk"), ("dw", "gt", "gtk", "qt", "qtk")):
        p, q = wide(o[a], o[ak], 1), wide(o[b], o[bk], 128)
        K = p.shape[1]
        off, size = (o[y].double() - p @ q.T).abs(), p.abs() @ q.abs().T
        assert bool((off <= (K / 8 + 17) * 2.0 ** -24 * size).all()), y
    xd, gd, wd = (t.double().requires_grad_() for t in (x, gamma, w))
    yd = xd * gd / (xd.square().mean(1, keepdim=True) + 1e-6).sqrt()
    logp = torch.log_softmax(yd @ wd.T, 1)
    has = tokens >= 0
    at = torch.where(has, logp.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    H = -(logp.exp() * logp).sum(1)
    (dlogp.double() @ at + dH.double() @ H).backward()
    noise = 5 * math.sqrt(2) * 2.0 ** -4 / math.sqrt(3)
    rms = lambda t: float(t.square().mean().sqrt())  # noqa: E731
    dlogits = torch.autograd.grad
    logit_off = noise * rms(yd.detach()) * rms(wd.detach()) * math.sqrt(300)
    assert rms(o["logits"].double() - (yd @ wd.T).detach()) <= logit_off
    assert rms(o["logp"].double() - at.detach()) <= 2 * logit_off and rms(o["H"].double() - H.detach()) <= 4 * logit_off
    # gradients of the whole: cosine and size, since the logits' errors go into them too
    for a, b in ((o["dw"], wd.grad), (o["dx"], xd.grad)):
        cos = float((a.double() * b).sum() / (a.double().norm() * b.norm()))
        assert cos > 0.99 and abs(float(a.double().norm() / b.norm()) - 1) < 0.05


def test_step_in_a_graph(D):
    """Captured and replayed, with eager work between the replays: each replay gives what eager calls give, to the bit."""
    x, gamma, w, tokens, dlogp, dH = inputs(4)
    plans = []
    for _ in range(2):
        p = w.clone()
        plans.append(D.MuonPlan([p], [torch.zeros_like(p)]))
    step(D, x, gamma, w, tokens, dlogp, dH, D.MuonPlan([w.clone()], [torch.zeros_like(w)]))  # warm up outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(D, x, gamma, plans[0].params[0], tokens, dlogp, dH, plans[0])
    for k in range(4):
        new = inputs(10 + k)
        for a, b in zip((x, tokens, dlogp, dH), (new[0], new[3], new[4], new[5])):
            a.copy_(b)
        graph.replay()
        want = step(D, x, gamma, plans[1].params[0], tokens, dlogp, dH, plans[1])
        torch.cuda.synchronize()
        for name in want:
            assert same(out[name], want[name]), (k, name)
        assert torch.equal(plans[0].params[0], plans[1].params[0]) and torch.equal(plans[0].momentum[0], plans[1].momentum[0])


def test_muon_in_a_graph(D):
    """Small matrices (a workgroup each) and larger ones, captured and replayed with other work between."""
    g = gen(12)
    shapes = [(96, 256), (300, 400), (5, 9), (700, 130)]
    make = lambda: [torch.randn(s, generator=gen(13), device="cuda") for s in shapes]  # noqa: E731
    grads = [torch.randn(s, generator=g, device="cuda").bfloat16() for s in shapes]
    a, b = D.MuonPlan(make(), grads), D.MuonPlan(make(), grads)
    D.densenet_muon(D.MuonPlan(make(), grads), lr=0.01)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.densenet_muon(a, lr=0.01, weight_decay=0.1)
    for _ in range(4):
        for t in grads:
            t.normal_(generator=g)
        graph.replay()
        D.densenet_muon(b, lr=0.01, weight_decay=0.1)
        torch.cuda.synchronize()
        for x, y in zip(a.params + a.momentum, b.params + b.momentum):
            assert torch.equal(x, y)


def test_two_streams_and_two_graphs(D):
    """Two streams at once, and two graphs replayed at once, give what each gives alone: no memory is shared but the caller's."""
    sets = [inputs(20, 150, 300, 700), inputs(21, 33, 1000, 5000)]
    alone = [step(D, *s) for s in sets]
    torch.cuda.synchronize()
    streams, graphs, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for s, st in zip(sets, streams):
        with torch.cuda.stream(st):
            step(D, *s)
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                got.append(step(D, *s))
        torch.cuda.synchronize()
        for a, b in zip(got, alone):
            assert all(same(a[k], b[k]) for k in b)
    for s in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(step(D, *s))
    for _ in range(3):
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, alone):
            assert all(same(a[k], b[k]) for k in b)


@pytest.mark.parametrize("muon,eight,dt", [(False, True, "bf16"), (True, False, "bf16"), (True, True, "f32"), (True, True, "f16")])
def test_region_head(D, muon, eight, dt):
    """The example runs, its gradients are the definition's, and its answers are those of its own logits."""
    from paper_1404_1869_amd.region_head import RegionHead
    g = gen(5)
    n, C, V = 200, 384, 90
    desc = torch.randn(n, C, generator=g, device="cuda")
    labels = torch.randint(-1, V, (n,), generator=g, device="cuda")
    head = RegionHead(V, C, dtype=D.DTYPES[dt], muon=muon)
    run = head.step_8bit if eight else head.step
    w0, g0 = head.products.double().clone().requires_grad_(), head.gamma.double().clone().requires_grad_()
    loss = run(desc, labels)
    d = desc.double()
    logp = torch.log_softmax(d * g0 / (d.square().mean(1, keepdim=True) + 1e-6).sqrt() @ w0.T, 1)
    has = labels >= 0
    want = torch.where(has, -logp.gather(1, labels.clamp(min=0)[:, None])[:, 0], 0.0)
    (want.sum() / has.sum()).backward()
    # logits of size sum |y w| 2^-4 / sqrt(C) (as above) in 8 bits, 2^-9 of them in 16
    assert float((loss.double() - want.detach()).abs().max()) < (0.1 if eight else 0.01)
    for a, b in ((head.dw.double() / head.scale, w0.grad), (head.dgamma.double() / head.scale, g0.grad)):
        cos = float((a * b).sum() / (a.norm() * b.norm()))
        assert cos > (0.98 if eight else 0.9999) and abs(float(a.norm() / b.norm()) - 1) < (0.05 if eight else 0.005)
    for _ in range(3):
        run(desc, labels)
    if dt != "f32":
        assert torch.equal(head.products, head.w.to(head.products.dtype))
    ids, best, H = head.answer(desc, top=7)
    assert ids.shape == best.shape == (n, 7) and bool((best[:, :-1] >= best[:, 1:]).all()) and bool((H >= 0).all())
    assert bool(((ids >= 0) & (ids < V)).all()) and bool((best.exp().sum(1) <= 1 + 1e-5).all())
    assert head.answer(desc, top=7)[0].equal(ids)


def test_region_head_command(D):
    from paper_1404_1869_amd import region_head
    region_head.main(["--words", "40", "--boxes", "80", "--steps", "2", "--muon", "--eight"])


def test_rows_past_32_bits(D):
    """Logits, codes and rows of more than 2^31 values: what lies at the end is computed like what lies at the start."""
    g = gen(6)
    n, C, V = 70001, 32, 32000
    a, w = torch.randn(n, C, generator=g, device="cuda").bfloat16(), torch.randn(V, C, generator=g, device="cuda").bfloat16()
    assert n * V > 2 ** 31
    a[-300:] = a[:300]
    q, k, _, _ = D.densenet_quantize_blocks(a)
    w8, wk, _, _ = D.densenet_quantize_blocks(w, rows=128)
    y = D.densenet_block_product(q, k, w8, wk)
    assert torch.equal(y[-300:], y[:300]) and torch.equal(y[:300], D.densenet_block_product(q[:300], k[:300], w8, wk))
    token = torch.randint(0, V, (n,), generator=g, device="cuda")
    token[-300:] = token[:300]
    logp, H, lse, ids, best = D.densenet_token_scores(y, token, top=3)
    for t in (logp, H, lse, ids, best):
        assert torch.equal(t[-300:], t[:300])
    few = D.densenet_token_scores(y[:300].contiguous(), token[:300], top=3)
    assert torch.equal(few[3], ids[:300])  # (few rows are split over workgroups: sums in another order)
    one = torch.ones(n, device="cuda")
    want = D.densenet_token_scores_backward(y[-300:].contiguous(), token[-300:], lse[-300:], entropy=H[-300:], dlogp=one[:300], dentropy=one[:300])
    D.densenet_token_scores_backward(y, token, lse, entropy=H, dlogp=one, dentropy=one, out=y)
    assert torch.equal(y[-300:], want) and torch.equal(y[:300], want)
    # the gradient's codes, as it lies and turned: [V][n] past 2^31 too
    c, ck, t, tk = D.densenet_quantize_blocks(y, turned=True)
    last = n // 128 * 128
    part = D.densenet_quantize_blocks(y[last:].contiguous(), turned=True)
    assert same(c[last:], part[0]) and torch.equal(ck[last:], part[1]) and same(t[:, last:], part[2]) and torch.equal(tk[:, -1:], part[3])


def test_long_products_past_32_bits(D):
    """Operands of more than 2^31 codes each way: of a, and of w."""
    g = gen(7)
    C, V, n = 9216, 40, 240001
    assert n * C > 2 ** 31
    few = torch.randint(0, 120, (97, C), generator=g, device="cuda", dtype=torch.uint8)
    big = torch.empty(n, C, dtype=torch.uint8, device="cuda")
    for i in range(0, n, 9700):
        big[i:i + 9700] = few.repeat(100, 1)[:len(big[i:i + 9700])]
    scale = torch.rand(97, 72, generator=g, device="cuda").repeat(-(-n // 97), 1)[:n].contiguous()
    w = torch.randint(0, 120, (V, C), generator=g, device="cuda", dtype=torch.uint8).view(F8)
    wk = torch.rand(1, 72, generator=g, device="cuda")
    y = D.densenet_block_product(big.view(F8), scale, w, wk, out_dtype=0)
    x = few.view(F8).double() * scale[:97].double().repeat_interleave(128, 1)
    z = w.double() * wk.double().repeat_interleave(128, 1)
    bound = (C / 8 + 17) * 2.0 ** -24 * (x.abs() @ z.abs().T)
    for first in (0, 97 * 2000, n // 97 * 97 - 97):
        assert bool(((y[first:first + 97].double() - x @ z.T).abs() <= bound).all())
    rows, wk = 12, torch.rand(-(-n // 128), 72, generator=g, device="cuda")
    y = D.densenet_block_product(few[:rows].view(F8), scale[:rows], big.view(F8), wk, out_dtype=0)
    x = x[:rows]
    for first in (0, n - 130):
        part = slice(first, first + 130)
        z = big[part].view(F8).double() * wk.double().repeat_interleave(128, 1).repeat_interleave(128, 0)[part]
        assert bool(((y[:, part].double() - x @ z.T).abs() <= (C / 8 + 17) * 2.0 ** -24 * (x.abs() @ z.abs().T)).all())


def test_scores_of_many_rows(D):
    """More rows than a launch has waves for (2^26 of them): results repeat with the rows."""
    n, V, period = (1 << 26) + 5, 9, 1009
    base = torch.randn(period, V, generator=gen(8), device="cuda").half()
    x = base.repeat(-(-n // period), 1)[:n]
    token = torch.randint(0, V, (period,), generator=gen(9), device="cuda")
    want = D.densenet_token_scores(base, token, top=1)
    got = D.densenet_token_scores(x, token.repeat(-(-n // period))[:n], top=1)
    for a, b in zip(got, want):
        for first in (0, (1 << 26) // period * period - period):
            assert torch.equal(a[first:first + period], b)
        assert torch.equal(a[-5:], b[torch.arange(n - 5, n, device="cuda") % period])


def test_answers_follow_the_weights(D):
    """Words that a caller keeps give the same answers; without them an answer is of the weights as they are now."""
    from paper_1404_1869_amd.region_head import RegionHead
    head = RegionHead(256, 500, seed=3)  # two squares of rows, which change places when the rows are turned about
    desc = torch.randn(40, 500, generator=gen(51), device="cuda")
    kept = head.words_8bit()
    ids, logp, H = head.answer(desc, top=3)
    again = head.answer(desc, top=3, words=kept)
    assert torch.equal(ids, again[0]) and torch.equal(logp, again[1]) and torch.equal(H, again[2])
    head.products.copy_(head.products.flip(0))
    alone = logp[:, 0] > logp[:, 1]  # (of equal logits, which bf16 has many of, the lower index comes first before and after)
    assert int(alone.sum()) > 10
    assert torch.equal(head.answer(desc, top=1)[0][alone], 255 - ids[alone, :1])
    assert torch.equal(head.answer(desc, top=3, words=kept)[0], ids)
