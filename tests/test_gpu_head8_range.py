"""What the 8-bit head's operators hold of their sums and states, at the ends of the ranges that they take.

Products: of codes far apart in size.  Muon: singular values of X up to 4, where A and P reach 16 and more, against the 64-bit form,
with the bound that its roundings grow to (half a unit of 11 or 22 bits for each value held)."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_head8 import DT, E24, UNIT, gen, within  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    from paper_1404_1869_amd import densenet
    assert torch.cuda.is_available()
    densenet.lib()
    return densenet


def codes(D, x):
    """Values that e4m3 holds, as codes in rows that start on 16 bytes."""
    q = D._codes(x.shape, x.device)
    q.copy_(x.to(torch.float8_e4m3fn))
    assert torch.equal(q.float(), x)
    return q


@pytest.mark.parametrize("n", [1, 40, 300, 3000])
@pytest.mark.parametrize("yt", ["f32", "f16", "bf16"])
def test_products_of_codes_that_cancel(D, n, yt):
    """448 448 - 448 448 + 1: in 32 bits 1; of three of one eight, results in 16 bits may be off by 7 times 2^-13 of 448 448; of three
    different eights, or where no product is below 2^-12 of the largest, they are exact."""
    V, C, dev = 3001 if n == 3000 else 130, 300, "cuda"
    g = gen(n)
    one = lambda m: torch.ones(m, -(-C // 128), device=dev)  # noqa: E731
    wk = one(-(-V // 128))
    run = lambda a, w: D.densenet_block_product(codes(D, a), one(n), codes(D, w), wk, out_dtype=D.DTYPES[yt])  # noqa: E731
    a, w = torch.zeros(n, C, device=dev), torch.zeros(V, C, device=dev)
    a[:, 136:139] = torch.tensor([448.0, 448.0, 1.0])
    w[:, 136:139] = torch.tensor([448.0, -448.0, 1.0])
    y = run(a, w).float()
    assert float((y - 1).abs().max()) <= (0 if yt == "f32" else 7 * 2.0 ** -13 * 448 * 448)
    # each row's three in eights of its own: w has 448 in even ones, -448 in odd ones of the first 64 codes, 1 in the eights of the next
    a, w = torch.zeros(n, C, device=dev), torch.zeros(V, C, device=dev)
    w[:, :64] = torch.where(torch.arange(64, device=dev) // 8 % 2 == 0, 448.0, -448.0)
    w[:, 64:128] = 1.0
    r = torch.arange(n, device=dev)
    for first in (0, 8):
        a[r, torch.randint(0, 4, (n,), generator=g, device=dev) * 16 + first + torch.randint(0, 8, (n,), generator=g, device=dev)] = 448.0
    a[r, 64 + torch.randint(0, 64, (n,), generator=g, device=dev)] = 1.0
    assert bool((run(a, w) == 1).all())
    # products of 1, 2^-6 and 2^-12: sums of 300 of them are whole numbers of 2^-12 below 2^9, and rounded once
    pick = lambda m: torch.where(torch.rand(m, C, generator=g, device=dev) < 0.5, 1.0, 2.0 ** -6) * (torch.randint(0, 3, (m, C), generator=g, device=dev) - 1)  # noqa: E731,E501
    a, w = pick(n), pick(V)
    assert torch.equal(run(a, w), (a.double() @ w.double().T).to(DT[yt]))


def plain(u, coefs, unit):
    """X after the steps in 64 bits, and a bound of its error in the Frobenius norm where every value held is rounded to `unit`."""
    norm = lambda t: float(torch.linalg.vector_norm(t))  # noqa: E731
    spec = lambda t: float(torch.linalg.matrix_norm(t, 2)) if bool(t.any()) else 0.0  # noqa: E731
    X = (u.T if u.shape[0] > u.shape[1] else u).double()
    X = X / (norm(X) + 1e-7)
    err = 2 * unit * norm(X)
    for a, b, c in coefs:
        A = X @ X.T
        P = b * A + c * A @ A
        s = spec(X) + err
        # from X's error on either side and from rounding A; of P likewise; of the new X from all, and rounding it
        dA = 2 * s * err + 2 * unit * norm(A)
        dP = abs(b) * dA + abs(c) * (2 * s * s * dA + 2 * unit * norm(A) * norm(A)) + 2 * unit * norm(P)
        new = a * X + P @ X
        err = abs(a) * err + spec(P) * err + dP * s + 2 * unit * norm(new) + 2 * unit * norm(P) * norm(X)
        X = new
    return X.T if u.shape[0] > u.shape[1] else X, err


# From a singular value of 1: 3.1 and 0.39 (A is 9.6 in the second step), 3.9 and -0.96 (A 15.2, P -0.75), 3.95, 3.95 and 3.39 (A 15.6
# twice), 2.9, 0.11 and -2.2 (A 8.4), and 3.9 in the last step alone.
HIGH = [
    [(4.0, -1.0, 0.1), (0.5, -1.0, 0.1)],
    [(3.9, 0.0, 0.0), (0.5, -0.3, 0.0165)],
    [(3.95, 0.0, 0.0), (1.0, 0.0, 0.0), (0.02, -0.5, 0.0355)],
    [(2.9, 0.0, 0.0), (0.0, -0.5, 0.06), (-20.0, 0.0, 0.0)],
    [(1.0, 0.0, 0.0), (3.9, 0.0, 0.0)],
]
# One workgroup's matrices and larger ones, wide and tall, of one row and of many.
SHAPES = [(1, 9), (1, 5000), (5, 7), (100, 300), (300, 100), (200, 1500), (700, 130), (300, 300)]


@pytest.mark.parametrize("pt", ["f32", "bf16"])
@pytest.mark.parametrize("coefs", HIGH)
def test_muon_of_singular_values_up_to_4(D, coefs, pt):
    g = gen(len(coefs))
    ups = []
    for a, b in SHAPES:  # one direction that has nearly all of the norm, and a little of others
        u, v = (torch.nn.functional.normalize(torch.randn(s, generator=g, device="cuda"), dim=0) for s in (a, b))
        noise = torch.randn(a, b, generator=g, device="cuda") * (0.01 / (a * b) ** 0.5)
        ups.append(u[:, None] * v + noise)
    p = [torch.zeros(s, dtype=DT[pt], device="cuda") for s in SHAPES]
    plan = D.MuonPlan(p, ups, rates=[1.0] * len(p))
    D.densenet_muon(plan, lr=1.0, momentum=0.0, steps=len(coefs), coefficients=coefs)
    unit = 2.0 ** -11 if pt == "bf16" else 2.0 ** -20
    for q, u in zip(p, ups):
        want, err = plain(u, coefs, unit)
        want = -want
        assert float(torch.linalg.matrix_norm(want, 2)) < 4
        within(q, want, err + (UNIT[pt] + 4 * E24) * (want.abs() + err), f"{tuple(q.shape)}")


def test_scores_of_the_longest_row(D):
    """2^31 - 257 logits, the most that a row may have: six above the rest, at the end and past 2^30 too, equal ones by place."""
    V = (1 << 31) - 257
    at = {5: 3.0, V - 1: 4.0, V - 2: 4.0, 1 << 30: 2.0, (1 << 30) + 1: 2.0, V - 300: 1.0}
    x = torch.full((1, V), -20.0, dtype=torch.bfloat16, device="cuda")
    for place, value in at.items():
        x[0, place] = value
    token = torch.tensor([V - 1], device="cuda")
    logp, H, lse, ids, best = D.densenet_token_scores(x, token, top=8)
    assert ids.tolist() == [[V - 2, V - 1, 5, 1 << 30, (1 << 30) + 1, V - 300, 0, 1]]
    z = (V - 6) * math.exp(-20) + sum(math.exp(v) for v in at.values())
    want = math.log(z)
    # equal logits count in whole numbers, below 2^24 in a lane; the exponents (at most 24) of 24 joins are off by 3 roundings each
    # where they have weight: d1, the mean distance to the maximum
    d1 = ((V - 6) * math.exp(-20) * 24 + sum(math.exp(v) * (4 - v) for v in at.values())) / z
    off = E24 * (4 * d1 + 64)
    assert abs(float(lse) - want) <= off + 4 * E24 * want and abs(float(logp) - (4 - want)) <= off + 4 * E24 * want
    for got, place in zip(best[0].tolist(), ids[0].tolist()):
        assert abs(got - (at.get(place, -20.0) - want)) <= off + 4 * E24 * 26
    dx = D.densenet_token_scores_backward(x, token, lse, dlogp=torch.ones(1, device="cuda"), out=x)  # in the logits' own memory
    for place, value in [*at.items(), (0, -20.0), (V - 301, -20.0), (V // 2 + 99, -20.0)]:
        p = math.exp(value - want)
        g = (place == V - 1) - p
        # p is off by what lse is, and by two roundings of an exponent of at most 26 and of the exponential; bf16 rounds once
        assert abs(float(dx[0, place]) - g) <= UNIT["bf16"] * abs(g) * 1.01 + p * (off + E24 * (4 * 26 + 4)), place
    del x, dx
    torch.cuda.empty_cache()


@pytest.mark.parametrize("tall", [True, False])
def test_muon_past_32_bits(D, tall):
    """A matrix of 65537 x 32768 (2^31 values and more, the smaller side the largest that there may be) whose update is 0 but for 6 x 5
    places spread to its ends: there the step is that of the 6 x 5 matrix, and elsewhere weights stay 0."""
    r, c = torch.tensor([0, 300, 32768, 50001, 65535, 65536], device="cuda"), torch.tensor([0, 1, 20000, 32766, 32767], device="cuda")
    u = torch.randn(6, 5, generator=gen(31), device="cuda").bfloat16()
    shape = (65537, 32768)
    if not tall:
        r, c, u, shape = c, r, u.T, shape[::-1]
    g = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    g[r[:, None], c] = u
    p = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    D.densenet_muon(D.MuonPlan([p], [g], rates=[1.0]), lr=-1.0, momentum=0.0, steps=3)
    want, err = plain(u, [(3.4445, -4.775, 2.0315)] * 3, 2.0 ** -11)
    within(p[r[:, None], c], want, err + UNIT["bf16"] * (want.abs() + err), "p")
    p[r[:, None], c] = 0
    assert not any(bool(t.any()) for t in p.split(4096))
    del g, p
    torch.cuda.empty_cache()


def test_quantize_more_rows_than_a_launch_holds(D):
    """2^28 rows of one value and a few (a launch has 2^24 workgroups of 16 rows): codes and scales repeat with the rows."""
    n, period = (1 << 28) + 77, 1009
    base = torch.randn(period, 1, generator=gen(32), device="cuda").bfloat16()
    x = base.repeat(-(-n // period), 1)[:n]
    out = torch.empty(n, 1, dtype=torch.float8_e4m3fn, device="cuda")
    q, k, _, _ = D.densenet_quantize_blocks(x, out=out)
    want, wk, _, _ = D.densenet_quantize_blocks(base)
    last = (1 << 28) // period * period  # the last period, cut short, has row 2^28 among its first
    for first in (0, last - period, last - 5 * period):
        part = slice(first, first + period)
        assert torch.equal(q[part].view(torch.uint8), want.contiguous().view(torch.uint8)) and torch.equal(k[part], wk)
    rest = n - last
    assert rest > 77 and torch.equal(q[last:].view(torch.uint8), want[:rest].contiguous().view(torch.uint8)) and torch.equal(k[last:], wk[:rest])
    del x, out, q, k
    torch.cuda.empty_cache()
