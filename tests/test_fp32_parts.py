"""Three bf16 parts of fp32 values, emulated: the six products keep fp32, and without any of the three smaller ones most terms
are off by more than the GPU test of fp32 gradients allows (2^-21 of them)."""
import pytest

torch = pytest.importorskip("torch")

PRODUCTS = [(2, 0), (1, 1), (0, 2), (1, 0), (0, 1), (0, 0)]


def parts(x):
    out = []
    for _ in range(3):
        p = x.bfloat16().float()
        out.append(p.double())
        x = x - p
    return out


def test_six_products_keep_fp32_and_five_do_not():
    g = torch.Generator().manual_seed(1)
    x, y = torch.randn(20000, generator=g), torch.randn(20000, generator=g)
    a, b, exact = parts(x), parts(y), x.double() * y.double()
    whole = sum(a[i] * b[j] for i, j in PRODUCTS)
    assert float(((whole - exact) / exact).abs().max()) < 2.0 ** -24
    for i, j in PRODUCTS[:3]:
        off = ((whole - a[i] * b[j] - exact) / exact).abs()
        assert float((off > 2.0 ** -20).double().mean()) > 0.5
