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


# ------------------------------------------------------------------------------------------------ scales as any fp32 numbers
def relaid(scales, how):
    """The same scales: contiguous, at a distance that is no multiple of four, or starting off a 16-byte boundary; NaN around them."""
    rows, cols = scales.shape
    if how == "contiguous":
        return scales.clone(memory_format=torch.contiguous_format)
    ld, skip = {"apart": (cols + 1 | 1, 0), "skipped": (-(-cols // 4) * 4 + 8, 1), "both": (cols + 5 | 1, 3)}[how]
    store = torch.full((rows * ld + skip,), float("nan"), device="cuda")
    view = store[skip:].view(rows, ld)[:, :cols]
    view.copy_(scales)
    return view


LAYOUTS = ["contiguous", "apart", "skipped", "both"]


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("which", ["matmul", "grad_input", "grad_weight"])
@pytest.mark.parametrize("M,N,K", [(1, 257, 300), (13, 130, 1000), (777, 513, 2047), (1001, 2048, 2047), (389, 1301, 4100)])
def test_scales_of_any_alignment(which, M, N, K, how, forced):
    call, (args, want) = getattr(fp8, which), operands(which, M, N, K, M)
    loose = [args[0], relaid(args[1], how), args[2], relaid(args[3], how) if which == "grad_weight" else args[3]]
    for tile, shares in SHAPES + [(8, 1)]:
        if which != "matmul" and tile in (8, 64):
            continue
        forced(tile, shares)
        assert torch.equal(call(*loose, dtype=torch.float32).double(), want), (tile, shares)
    if which == "grad_weight":                               # one side alone
        forced(0)
        assert torch.equal(call(*args[:3], loose[3], dtype=torch.float32).double(), want)
        assert torch.equal(call(*loose[:2], *args[2:], dtype=torch.float32).double(), want)
    assert fp8.status() == (0, 0)


@pytest.mark.parametrize("which", ["matmul", "grad_input", "grad_weight"])
def test_many_blocks_of_loose_scales(which):
    sizes = {"matmul": (701, 600, 38400), "grad_input": (701, 38400, 600), "grad_weight": (38400, 601, 703)}[which]
    call, (args, want) = getattr(fp8, which), operands(which, *sizes)
    args[1] = relaid(args[1], "both")
    if which == "grad_weight":
        args[3] = relaid(args[3], "contiguous")
    for g in [call(*args, dtype=torch.float32) for _ in range(10)]:
        assert torch.equal(g.double(), want)
    assert fp8.status() == (0, 0)


@pytest.mark.parametrize("offsets,M", [([0, 300], 300), ([0, 130, 130, 131, 600, 1000], 1000), ([7, 9, 200, 480], 501), ([0, 2, 701, 1500, 1501, 1501, 2299], 2299), (list(range(0, 65)), 64)])
def test_groups_with_loose_scales(offsets, M):
    E, N, K = len(offsets) - 1, 262, 515
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(M)
    w = fp8.quantize_weight(torch.randn(E, N, K, device="cuda", generator=g))
    x, dy = torch.randn(M, K, device="cuda", generator=g), torch.randn(M, N, device="cuda", generator=g)
    q, d = fp8.quantize_both(x, off), fp8.quantize_both(dy, off)
    for t in (q, d):                                         # (what belongs to no group is not written)
        t.scales.nan_to_num_(nan=1.0, posinf=1.0, neginf=1.0)
        t.column_scales.nan_to_num_(nan=1.0, posinf=1.0, neginf=1.0)

    def step(lay):
        zeros = lambda *s: torch.zeros(*s, device="cuda")
        return (fp8.grouped_matmul(q.codes, lay(q.scales), *w, off, out=zeros(M, N)), fp8.grouped_grad_input(d.codes, lay(d.scales), *w, off, out=zeros(M, K)),
                fp8.grouped_grad_weight(d.column_codes, lay(d.column_scales), q.column_codes, lay(q.column_scales), off))
    want = step(lambda s: s)
    for how in LAYOUTS:
        assert all(torch.equal(a, b) for a, b in zip(step(lambda s: relaid(s, how)), want))


@pytest.mark.parametrize("M,N,K", [(300, 256, 1000), (1001, 512, 256)])
def test_some_of_a_batch(M, N, K):
    """Tokens from the fifth on: their scales start off a 16-byte boundary."""
    (a, s, *w), want = operands("matmul", M, N, K, 3)
    for some in (slice(5, None), slice(5, 200), slice(7, 8), slice(6, 19)):
        assert torch.equal(fp8.matmul(a[some], s[:, some], *w, dtype=torch.float32).double(), want[some])


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("M,K", [(1, 130), (129, 127), (301, 1001)])
def test_quantized_into_scales_of_any_alignment(M, K, how):
    """Outputs that are given; what lies around them stays."""
    x = torch.randn(M, K, device="cuda")
    q = fp8.quantize_both(x)
    to = fp8.Forms(q.codes, relaid(torch.full_like(q.scales, -7.0), how), q.column_codes, relaid(torch.full_like(q.column_scales, -7.0), how))
    out = fp8.quantize_both(x, out=to)
    assert torch.equal(out.scales, q.scales) and torch.equal(out.column_scales, q.column_scales)
    to[1].fill_(-7.0), to[3].fill_(-7.0)
    fp8.quantize(x, out=to[:2])
    fp8.quantize_columns(x, out=to[2:])
    assert torch.equal(to[1], q.scales) and torch.equal(to[3], q.column_scales)
    for t in (to[1], to[3]):
        if how != "contiguous":
            store = torch.as_strided(t, (t.untyped_storage().nbytes() // 4,), (1,), 0).clone()
            inside = torch.as_strided(store, t.shape, t.stride(), t.storage_offset())
            inside.fill_(float("nan"))
            assert torch.isnan(store).all()


def test_captured_with_loose_scales():
    call, (args, want) = fp8.grad_weight, operands("grad_weight", 1001, 515, 2047)
    args[1], args[3] = relaid(args[1], "contiguous"), relaid(args[3], "skipped")
    call(*args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(*args)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got.double(), want)


def test_refusals_of_scales():
    a, s, w, ws = operands("matmul", 20, 130, 300)[0]
    for bad in (s.t(), s[:, :19], s[:2], s.flip(0)[:, ::2]):
        with pytest.raises(ValueError):
            fp8.matmul(a, bad, w, ws)
    for bad in (s.double(), s.cpu(), None):
        with pytest.raises(TypeError):
            fp8.matmul(a, bad, w, ws)
    with pytest.raises(ValueError):
        fp8.matmul(a, s[:1].expand(3, 20), w, ws)
