"""Lists of as many tensors as a launch's arguments hold, and one more, tensors without a number among them."""
import pytest
import torch

from paper_2609_26077_b200 import gradients

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count", [c + d for c in (32, 64, 128, 256, 512, 1000, 2000) for d in (0, 1)])
def test_every_tensor_of_a_list_takes_part(count):
    """Whole numbers, whose squares and sums are exact, and a factor that is a power of two."""
    g = torch.Generator().manual_seed(count)
    sizes = torch.randint(0, 400, (count,), generator=g).tolist()
    flat = torch.randint(-3, 4, (sum(sizes),), generator=g).float().cuda()
    ts = list(flat.split(sizes))
    total = flat.double().square().sum()
    norm = total.sqrt().float()
    assert torch.equal(gradients.norm(ts), norm)
    out = torch.full_like(flat, -7.0)
    assert torch.equal(gradients.clip(ts, total.sqrt().item() / 4, out=list(out.split(sizes))), norm)
    assert torch.equal(out, flat / 4)
    assert torch.equal(gradients.clip(ts, total.sqrt().item() / 2), norm)
    assert torch.equal(flat, 2 * out)
