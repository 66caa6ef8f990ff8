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
