"""Copies of the parameters that AdamW steps: a parameter may be its own, copies in 32 bits are refused when the plan is made."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    from paper_1404_1869_amd import densenet
    assert torch.cuda.is_available()
    densenet.lib()
    return densenet


def tensors(dtype, n=3):
    g = torch.Generator(device="cuda").manual_seed(4)
    return [[torch.randn(300 + 7 * i, generator=g, device="cuda").to(t) for i in range(n)] for t in (dtype, torch.bfloat16)]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_a_parameter_may_be_its_own_copy(D, dtype, bits):
    """The same weights as without copies, to the bit, and beside it copies of other parameters."""
    runs = []
    for own in (False, True):
        p, g = tensors(dtype)
        low = torch.bfloat16 if dtype == torch.float32 else dtype
        other = torch.empty_like(p[1], dtype=low)
        copies = [p[0].to(dtype), other, p[2]] if own else [None, other, None]
        assert not own or copies[0] is p[0]
        plan = D.AdamWPlan(p, g, copies=copies, state_bits=bits)
        assert plan.copies[0] is None and plan.copies[2] is None
        for k in range(3):
            D.densenet_adamw(plan, lr=0.1, step=k + 1, weight_decay=0.1, seed=k)
        assert torch.equal(other, p[1].to(low))
        runs.append(p)
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_copies_in_32_bits_are_refused_when_the_plan_is_made(D):
    p, g = tensors(torch.bfloat16)
    with pytest.raises(D.DenseNetError) as e:
        D.AdamWPlan(p, g, copies=[t.float() for t in p])
    assert e.value.status == D.DN_E_UNSUPPORTED
    p, g = tensors(torch.float32)
    with pytest.raises(D.DenseNetError) as e:
        D.AdamWPlan(p, g, copies=[t.clone() for t in p])
    assert e.value.status == D.DN_E_UNSUPPORTED
