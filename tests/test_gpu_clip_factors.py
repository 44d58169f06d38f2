"""Factors of clipping that are no normal fp32 numbers, in place and not."""
import pytest
import torch

from paper_2609_26077_b200 import gradients

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("values,max_norm", [
    ([2.0 ** 64, 2.0 ** 50], 1.0),                           # norm 2^64 (1 + 2^-29): a factor of less than 2^-64 that rounds to it
    ([1.0, 2.0 ** -14], 2.0 ** -64),
    ([1.0, 2.0 ** -15], 2.0 ** -64),
    ([2.0 ** 64], 1.0),                                      # 2^-64 itself
    ([2.0 ** 64, 2.0 ** 60], 1.0),
    ([3.0 * 2.0 ** 70, 5.0], 2.0 ** -10),
    ([1.0, 2.0 ** -14], 1.0),                                # a factor that rounds to 1
])
def test_in_place_is_as_not_in_place(values, max_norm, dtype):
    ts = [torch.tensor(values, device="cuda").to(dtype)] + [torch.zeros(300, device="cuda", dtype=dtype)]
    out = [torch.full_like(t, -7.0) for t in ts]
    mine = [t.clone() for t in ts]
    a, b = gradients.clip(ts, max_norm, out=out), gradients.clip(mine, max_norm)
    assert torch.equal(a, b) and all(torch.equal(x, y) for x, y in zip(mine, out))
    norm = torch.cat(ts).double().square().sum().sqrt()
    want = ts[0].double() * min(1.0, max_norm / norm.item())
    # the factor, each part of the product, the type: half a step each
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]
    assert ((mine[0].double() - want).abs() <= want.abs() * (4 * 2.0 ** -24 + half) + 2.0 ** -133).all()
