"""The norm of gradients to its last bit: the sum of squares is taken in 64 bits."""
import pytest
import torch

from fp8_oracle import TYPES
from paper_2609_26077_b200 import gradients

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [4, 8, 16, 100, 4096])
def test_norm_is_rounded_once(n, dtype):
    """Against the sum of squares in 64 bits: half a step of fp32, and what 64-bit sums in another order may differ by."""
    g = torch.Generator("cuda").manual_seed(n)
    many = torch.randn(200, n, device="cuda", generator=g).to(dtype)
    got = torch.stack([gradients.norm([t]) for t in many.clone().unbind()]).double()
    want = many.double().square().sum(1).sqrt()
    assert ((got - want).abs() <= want * (2.0 ** -24 + n * 2.0 ** -53)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_many_and_unaligned_tensors_is_rounded_once(dtype):
    flat = torch.randn(1 << 20, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
    for seed in range(20):
        g = torch.Generator().manual_seed(seed)
        ts = [flat[a:a + n] for a, n in zip(torch.randint(0, 1 << 19, (50,), generator=g).tolist(), torch.randint(1, 20000, (50,), generator=g).tolist())]
        want = torch.stack([t.double().square().sum() for t in ts]).sum().sqrt()
        assert (gradients.norm(ts).double() - want).abs() <= want * (2.0 ** -24 + 2.0 ** -33)
