"""The kernels that large calls of an 8-bit head's operators run, against 64-bit forms, element by element: products in tiles of 256 x
256, whole and in parts along k, and Muon's products in tiles of 256 x 256 and 128 x 128, whole and in parts, wide and tall, in
one and two fp16 parts, with more matrices than a launch holds."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_head8 import DT, E24, TINY, UNIT, cut_off, gen, operands, plain_product, within  # noqa: E402

pytestmark = pytest.mark.gpu
NS = (3.4445, -4.7750, 2.0315)


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


# ---------------------------------------------------------------------------------------------------------------------
# Products.  Of 129 tiles of 256 x 256 and more, results in 16 bits have a workgroup for each; beyond 256 of them, the last ones are
# split along k where a row is long.  Blocks of 128 k: an even and an odd number, a few, past 64; rows that end within 16 codes.
# ---------------------------------------------------------------------------------------------------------------------
PRODUCT = [  # n, C, V, y type, layout, whether some tiles are split
    (3000, 129, 3001, "bf16", "rows", False), (3001, 257, 3000, "f16", "rows", False), (3000, 641, 3001, "bf16", "odd", False),
    (3001, 1000, 2999, "f16", "rows", False), (3000, 1037, 3001, "bf16", "rows", False), (2817, 1003, 3073, "f16", "tight", False),
    (2999, 2050, 3003, "bf16", "rows", False), (3000, 8292, 3001, "bf16", "rows", False), (2000, 9211, 10007, "bf16", "rows", True),
    (2001, 4099, 10005, "f16", "odd", True),
]


@pytest.mark.parametrize("n,C,V,yt,how,split", PRODUCT)
def test_product_in_tiles_of_256(D, n, C, V, yt, how, split):
    g = gen(n + C + V)
    a, ak, w, wk = operands(D, g, n, C, V, how)
    need = D._work_bytes("densenet_block_product", 4096, 1 << 16, None, 4096, 1 << 16, None, n, C, V, None, 0, D.DTYPES[yt])
    if split:  # sums of tiles of 256 x 256 in fp32 beside codes that lie well
        assert need > D.DN_NO_WORKSPACE and (need - D.DN_NO_WORKSPACE) % (256 * 256 * 4) == 0
    else:
        assert need == D.DN_NO_WORKSPACE
    held = torch.full((n + 1, V + 9), 5.0, dtype=DT[yt], device="cuda")
    y = held[:n, 4:V + 4]
    D.densenet_block_product(a, ak, w, wk, out_dtype=D.DTYPES[yt], out=y)
    want, size = plain_product(a, ak, w, wk)
    lost = cut_off(a, ak, w, wk)
    within(y, want, UNIT[yt] * (want.abs() + lost) + lost + (C / 8 + 16) * E24 * size + TINY[yt], "y")
    assert bool((held[n:] == 5).all()) and bool((held[:, :4] == 5).all()) and bool((held[:, V + 4:] == 5).all())
    assert torch.equal(D.densenet_block_product(a, ak, w, wk, out_dtype=D.DTYPES[yt]), y)  # the same bits every time


# ---------------------------------------------------------------------------------------------------------------------
# Muon
# ---------------------------------------------------------------------------------------------------------------------
def bounded_muon(u, steps, parts):
    """X after `steps` steps in 64 bits, and what each of its elements may be off by: the roundings of the values held (unit), and of
    sums in 32 bits, carried through each product by magnitudes.  Two parts: 22 bits, and of the products of parts the smallest is
    left out, so three units of 2^-22 at most for a product of two values; 2^-20 for each has it all.  Held values have powers of
    two of at least 2^11 and fp16's smallest step, of which half is 2^-25."""
    a, b, c = NS
    unit = 2.0 ** -11 if parts == 1 else 2.0 ** -20
    tall = u.shape[0] > u.shape[1]
    X = (u.T if tall else u).double().contiguous()
    X = X / (torch.linalg.vector_norm(X) + 1e-7)
    r, k = X.shape
    E = X.abs() * (unit + 100 * E24) + 2.0 ** -38  # the sum of squares: 64 values and 20 joins one after the other in 32 bits
    t = lambda m: m.T.contiguous()  # noqa: E731
    for _ in range(steps):
        M = X.abs()
        A = X @ t(X)
        EA = M @ t(E)
        EA = EA + t(EA) + E @ t(E) + unit * A.abs() + (3 * k / 8 + 32) * E24 * (M @ t(M)) + 2.0 ** -38
        S, N = A @ A, A.abs()
        ES = N @ EA
        ES = ES + t(ES) + EA @ EA + (3 * r / 8 + 32) * E24 * (N @ N)
        P = b * A + c * S
        EP = abs(b) * EA + abs(c) * ES + (unit + 4 * E24) * (abs(b) * N + abs(c) * S.abs()) + 2.0 ** -36
        new = a * X + P @ X
        E = abs(a) * E + (P.abs() + EP) @ E + EP @ M + (3 * r / 8 + 32) * E24 * (P.abs() @ M)
        E = E + (unit + 8 * E24) * (new.abs() + abs(a) * M + E) + 2.0 ** -38
        X = new
    return (t(X), t(E)) if tall else (X, E)


def turned(i, r, c):
    return (c, r) if i % 2 else (r, c)


MUON = [  # shapes, parts, steps, weights' type
    # X X' and A^2 in whole tiles of 256 x 256, and the update too
    ([turned(i, 897 + 2 * i, 930 - i) for i in range(16)], 1, 2, "bf16"), ([turned(i, 897 + 2 * i, 930 - i) for i in range(16)], 2, 2, "f32"),
    # both in parts along k, of tiles of 256 x 256 (and X X' alone, of one fp16 part)
    ([(1297, 1301), (1305, 1296), (1300, 1300), (1290, 1311)], 2, 2, "f16"), ([turned(i, 899 + i, 3605 - 3 * i) for i in range(8)], 1, 1, "bf16"),
    # both in parts of tiles of 128 x 128: updates of 64 x 128, and of 256 x 256 of one wide or tall matrix
    ([(509, 515), (515, 510), (512, 512), (511, 520)], 2, 2, "f32"), ([(1001, 9213)], 2, 2, "f32"), ([(9213, 1001)], 2, 2, "f16"),
    ([(2001, 1999)], 2, 2, "f32"), ([(257, 1028)], 1, 2, "bf16"), ([(2047, 8189), (8189, 2047)], 1, 2, "bf16"),
    # in one call with matrices of fewer k than there are parts
    ([(1001, 9213), (129, 130), (200, 131), (300, 5), (100, 100), (3, 6000)], 2, 2, "f32"),
]


@pytest.mark.parametrize("shapes,parts,steps,pt", MUON)
def test_muon_of_large_matrices(D, shapes, parts, steps, pt):
    g = gen(sum(r * 3 + c for r, c in shapes) + parts)
    new = lambda s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    # a few strong directions over noise, as gradients have them
    grads = [new((r, c)) + new((r, 4)) @ new((4, c)) for r, c in shapes]
    p = [torch.zeros(s, dtype=DT[pt], device="cuda") for s in shapes]
    copies = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes] if pt == "f32" else None
    plan = D.MuonPlan(p, grads, copies=copies, rates=[1.0] * len(p), parts=parts)
    D.densenet_muon(plan, lr=-1.0, momentum=0.0, steps=steps)
    for i, u in enumerate(grads):
        want, off = bounded_muon(u, steps, parts)
        assert float(off.mean() / want.abs().mean()) < (0.5 if parts == 1 else 0.1)  # (no bound that another matrix would meet)
        within(p[i], want, off + UNIT[pt] * (want.abs() + off) + TINY[pt], f"{tuple(u.shape)}")
        if copies:
            within(copies[i], want, off + (UNIT[pt] + UNIT["bf16"] + E24) * (want.abs() + off), "copy")


def test_muon_of_more_large_matrices_than_a_launch_holds(D):
    """35 that need the general path and 60 that a workgroup holds, among each other: each as alone, to sums in another order."""
    g = gen(99)
    shapes = []
    for i in range(35):
        shapes.append(turned(i, 257 + i % 3, 514 + i % 5) if i < 33 else turned(i, 140, 1400 + i))
        if i < 30:
            shapes += [(20 + i, 30), (60, 50 + i)]
    new = lambda s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    grads = [new((r, c)) + new((r, 4)) @ new((4, c)) for r, c in shapes]
    p = [torch.zeros(s, device="cuda") for s in shapes]
    plan = D.MuonPlan(p, grads, rates=[1.0] * len(p))
    D.densenet_muon(plan, lr=-1.0, momentum=0.0, steps=2)
    # the workspace is that of the larger of the two groups (32 matrices and 3), with two parts of X twice, A and P for each of its
    assert plan.work_bytes[0] >= 32 * 2 * 2 * (2 * 257 * 514 + 2 * 257 * 257)
    assert plan.work_bytes[0] < 35 * 2 * 2 * (2 * 260 * 520 + 2 * 260 * 264) + (1 << 20)
    for q, u in zip(p, grads):
        want, off = bounded_muon(u, 2, 2)
        within(q, want, off + UNIT["f32"] * (want.abs() + off), f"{tuple(u.shape)}")
