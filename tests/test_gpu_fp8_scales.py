"""Scales of the 8-bit floating-point layer on their way into its products: a different one for every block of every row and column, so that a scale that
is late, early or another block's shows in the result, bit for bit."""
import pytest
import torch

from paper_2609_26077_b200 import fp8

pytestmark = pytest.mark.gpu

SHAPES = [(0, 1), (64, 1), (128, 1), (256, 1), (64, 2), (128, 2), (128, 3), (64, 4), (128, 4)]


@pytest.fixture
def forced():
    yield fp8.force_tile
    fp8.force_tile(0)


def exact(M, N, K, seed=0):
    """Codes from -2 to 2 and scales from 1 to 8: a block's sum is a whole number of at most 512, times its scales at most 2^15, and sums of up to 512 blocks
    are whole numbers below 2^24, so that fp32 holds every one of them."""
    g = torch.Generator("cuda").manual_seed(seed)
    whole = lambda *s: torch.randint(-2, 3, s, device="cuda", generator=g)
    powers = lambda *s: torch.exp2(torch.randint(0, 4, s, device="cuda", generator=g).float())

    def held(values):
        rows, cols = values.shape
        return torch.nn.functional.pad(values.float(), (0, -cols % 16)).to(fp8.CODES)[:, :cols]

    def apart(scales):
        return torch.nn.functional.pad(scales, (0, -scales.shape[1] % 4))[:, :scales.shape[1]]
    blocks = lambda n: -(-n // 128)
    return held, apart, whole, powers, blocks


def operands(which, M, N, K, seed=0):
    """The call's operands, and its result in 64 bits."""
    held, apart, whole, powers, blocks = exact(M, N, K, seed)
    wide = lambda s, rows, cols: s.double().repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    if which == "grad_weight":
        rows = blocks(M) * 128
        dy, x, dys, xs = whole(rows, N), whole(rows, K), powers(rows // 128, N), powers(rows // 128, K)
        want = (dy.double() * dys.double().repeat_interleave(128, 0)).t() @ (x.double() * xs.double().repeat_interleave(128, 0))
        return [held(dy), apart(dys), held(x), apart(xs)], want
    depth = K if which == "matmul" else N
    a, s, w, ws = whole(M, depth), powers(blocks(depth), M), whole(N, K), powers(blocks(N), blocks(K))
    av, wv = a.double() * s.double().t().repeat_interleave(128, 1)[:, :depth], w.double() * wide(ws, N, K)
    return [held(a), apart(s), held(w), ws], av @ (wv.t() if which == "matmul" else wv)


@pytest.mark.parametrize("which", ["matmul", "grad_input", "grad_weight"])
@pytest.mark.parametrize("M,N,K", [(300, 520, 650), (1500, 1300, 4000), (130, 4100, 8200), (5000, 700, 260)])
def test_every_block_takes_its_own_scales(which, M, N, K, forced):
    call, (args, want) = getattr(fp8, which), operands(which, M, N, K, M)
    for tile, shares in SHAPES:
        if which != "matmul" and tile == 64:
            continue
        forced(tile, shares)
        for _ in range(5):
            assert torch.equal(call(*args, dtype=torch.float32).double(), want), (tile, shares)
    assert fp8.status() == (0, 0)


@pytest.mark.parametrize("which", ["matmul", "grad_input", "grad_weight"])
def test_many_blocks_again_and_again(which):
    """A contraction of 300 blocks, in which every ring comes round many times, beside another stream's work."""
    sizes = {"matmul": (700, 600, 38400), "grad_input": (700, 38400, 600), "grad_weight": (38400, 600, 700)}[which]
    call, (args, want) = getattr(fp8, which), operands(which, *sizes)
    other = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        with torch.cuda.stream(other):
            busy.mul_(1.0)
        got.append(call(*args, dtype=torch.float32))
    for g in got:
        assert torch.equal(g.double(), want)
    assert fp8.status() == (0, 0)
