"""Offsets that are not as they should be - beyond the tokens, below their predecessors - mean the same to every call of a layer of experts."""
import pytest
import torch

import fp8_oracle as O
from paper_2609_26077_b200 import fmm, fp8

pytestmark = pytest.mark.gpu


def gradient(M, N, K, offsets, tokens, dtype=torch.float32, out=None, accumulate=False, stream=None):
    """grouped_grad_weight of forms whose unused rows hold NaN, and what it should be."""
    E, off = len(offsets) - 1, torch.tensor(offsets, dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(M)
    dy, x = torch.randn(M, N, device="cuda", generator=g), torch.randn(M, K, device="cuda", generator=g)
    forms = []
    for t in (dy, x):
        rows = fp8.column_rows(M, off)
        codes = torch.full((rows, -(-t.shape[1] // 16) * 16), 0x7F, dtype=torch.uint8, device="cuda").view(fp8.CODES)[:, :t.shape[1]]
        scales = torch.full((rows // 128, t.shape[1]), float("nan"), device="cuda")
        forms += fp8.quantize_columns(t, off, out=(codes, scales))
    got = fp8.grouped_grad_weight(*forms, off, dtype=dtype, out=out, accumulate=accumulate, tokens=tokens, stream=stream)
    (dc, ds, _), (xc, xs, _) = O.columns(dy, offsets), O.columns(x, offsets)
    want, bound, at = [], [], 0
    for lo, hi in zip(O.bounds(offsets, M), O.bounds(offsets, M)[1:]):
        n = -(-(hi - lo) // 128) * 128
        a, b = O.column_values(dc[at:at + n], ds[at // 128:(at + n) // 128]).t(), O.column_values(xc[at:at + n], xs[at // 128:(at + n) // 128])
        at += n
        want.append(a @ b)
        bound.append(O.product_bound(a.abs() @ b.abs(), n, a @ b, dtype))
    return got, torch.stack(want), torch.stack(bound)


BAD = [([0, 100, 400, 7], 300), ([-5, 20, 2 ** 31 - 1], 257), ([0, 100, 50, 400, 7], 300), ([0, 1000], 130), ([500, 600, 700], 300), ([0, 0, 5000, 5000, 6000], 129), ([0, 150, 300], 300)]


@pytest.mark.parametrize("N,K", [(64, 130), (300, 640)])
@pytest.mark.parametrize("offsets,M", BAD)
def test_weight_gradients_of_offsets_beyond_the_tokens(offsets, M, N, K):
    got, want, bound = gradient(M, N, K, offsets, M)
    O.close(got, want, bound)
    other = torch.cuda.Stream()
    again, _, _ = gradient(M, N, K, offsets, M, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(again, got)
    held = torch.ones_like(got)
    added, _, _ = gradient(M, N, K, offsets, M, out=held, accumulate=True)
    O.close(added, want + 1, bound + 2.0 ** -23 * (want.abs() + 1))


def test_no_tokens_at_all():
    off = torch.tensor([0, 5, 900], dtype=torch.int32, device="cuda")
    x = torch.empty(0, 130, device="cuda")
    c = fp8.quantize_columns(x, off)
    assert (fp8.grouped_grad_weight(*c, *c, off, tokens=0) == 0).all()
    held = torch.ones(2, 130, 130, device="cuda")
    assert (fp8.grouped_grad_weight(*c, *c, off, tokens=0, out=held, accumulate=True) == 1).all()


def test_refusals():
    off = torch.tensor([0, 5, 40], dtype=torch.int32, device="cuda")
    c = fp8.quantize_columns(torch.randn(40, 64, device="cuda"), off)
    for bad in (-1, c[0].shape[0] + 1, 1 << 40):
        with pytest.raises(ValueError):
            fp8.grouped_grad_weight(*c, *c, off, tokens=bad)
    with pytest.raises(TypeError):
        fp8.grouped_grad_weight(*c, *c, off, tokens="40")
    assert torch.equal(fp8.grouped_grad_weight(*c, *c, off, tokens=40), fp8.grouped_grad_weight(*c, *c, off))
