"""Every kernel form of the 8-bit product and its gradients, taken by name: ragged tiles on each side, the longest contraction and the largest
sums, scales far apart, outputs with gaps, several tiles to a CTA pair, and sums that leave the accumulator in time."""
import numpy as np
import pytest
import torch

import int8_oracle as O
from paper_2609_26077_b200 import fmm, int8
from test_gpu_int8_product import check_matmul, codes_of, padded, scales_of

pytestmark = pytest.mark.gpu

FEW, PAIRS = (int8.KERNEL_FEW_TOKENS, 8, 1), (int8.KERNEL_PAIRS, 256, 1)
CLUSTERS = [(int8.KERNEL_CLUSTER, columns, shares) for columns in (16, 32, 64, 128) for shares in (1, 2, 3, 5, 8)]
PRODUCT_FORMS = [FEW, PAIRS] + CLUSTERS
GRAD_FORMS = [PAIRS] + [f for f in CLUSTERS if f[1] >= 64]


@pytest.fixture(autouse=True)
def chosen_again():
    yield
    int8.force_product_shape()
    assert int8.status() == (0, 0)


def force(form):
    int8.force_product_shape(*form)
    assert tuple(int8.product_shape(int8.MATMUL, 5, 5, 5)) == form


def tokens_of(form):
    """Rows of a that leave the last of several tiles ragged."""
    return {FEW: 7, PAIRS: 300}.get(form, 2 * form[1] + 5)


@pytest.mark.parametrize("form", PRODUCT_FORMS)
def test_product(form):
    force(form)
    M = tokens_of(form)
    # ragged tiles of channels and of the contraction, a stage a share and fewer codes than a stage
    for N, K in ((300, 1100), (129, 1024), (1, 1025), (517, 8 * 128 + 16)):
        check_matmul(M, N, K, bias=N > 200, seed=N)
    if form[2] == 1:
        check_matmul(M, 77, 3, torch.bfloat16, seed=5)
    out = O.strided(torch.zeros(M, 333, device="cuda"), 5, 1)
    check_matmul(M, 333, 1300, out=out, extra=48)
    assert torch.isnan(torch.as_strided(out, (M - 1, 5), (338, 1), 1 + 333)).all()


@pytest.mark.parametrize("form", PRODUCT_FORMS)
def test_largest_sums(form):
    """Sums up to 2^31: every code at its limit, the longest K."""
    force(form)
    K, M = 131071, min(tokens_of(form), 70)
    for va, vb in ((-128, -128), (127, -128), (127, 127)):
        a = torch.full((M, 131072), va, dtype=torch.int8, device="cuda")[:, :K]
        b = torch.full((70, 131072), vb, dtype=torch.int8, device="cuda")[:, :K]
        c = int8.matmul(a, torch.ones(M, device="cuda"), b, torch.ones(70, device="cuda"), dtype=torch.float32)
        assert (c == float(np.float32(va * vb * K))).all()


@pytest.mark.parametrize("form", PRODUCT_FORMS)
def test_scales_far_apart(form):
    force(form)
    M, N, K = tokens_of(form), 140, 1030
    a, b = codes_of(M, K, 1), codes_of(N, K, 2)
    sa, sb = np.ones(M, np.float32), np.ones(N, np.float32)
    sa[:5], sb[:6] = [1e-30, 1e30, 1.0, np.nan, 2.0], [1e30, 1e-30, 1.0, 1e30, 1e-30, np.nan]
    sb[N - 1], sa[M - 1] = 1e-30, 1e30
    c = int8.matmul(padded(a), torch.from_numpy(sa).cuda(), padded(b), torch.from_numpy(sb).cuda(), dtype=torch.float32)
    acc = torch.from_numpy(a).cuda().double() @ torch.from_numpy(b).cuda().double().t()
    want = acc * torch.from_numpy(sa).cuda().double()[:, None] * torch.from_numpy(sb).cuda().double()
    assert torch.equal(torch.isnan(c), torch.isnan(want)) and torch.isnan(c[3]).all() and torch.isnan(c[:, 5]).all()
    off, size = (c.double() - want).abs(), want.abs()
    # three roundings; below 1e-30 in fp32's subnormal numbers, above 3e38 infinite
    good = (size < 3e38) & (size > 1e-30)
    assert (off[good] <= 4 * O.U32 * size[good]).all() and good.sum() > (M - 4) * (N - 5)
    assert torch.isinf(c[size > 3.5e38]).all()


def test_all_product_forms_agree_to_the_bit():
    """The sums are exact, so that the form leaves no trace."""
    for M, N, K in ((8, 300, 1100), (200, 700, 2048)):
        a, b = padded(codes_of(M, K, 1)), padded(codes_of(N, K, 2))
        sa, sb = [torch.from_numpy(scales_of(n, n)).cuda() for n in (M, N)]
        int8.force_product_shape()
        want = int8.matmul(a, sa, b, sb, dtype=torch.float32)
        for form in PRODUCT_FORMS:
            if form == FEW and M > 8:
                continue
            force(form)
            assert torch.equal(int8.matmul(a, sa, b, sb, dtype=torch.float32), want), form


@pytest.mark.parametrize("M,N,K", [(4100, 4100, 130), (257, 20000, 260), (20000, 300, 129)])
def test_pairs_walk_many_tiles(M, N, K):
    """Three and more tiles of 256 x 256 to each of 74 pairs, or one and two: both accumulators, each tile's own scales."""
    force(PAIRS)
    check_matmul(M, N, K, bias=True, seed=7)


# ------------------------------------------------------------------------------------------------ gradients
def check_gradient(which, M, N, K, dtype, out_type, pow2, seed=0, accumulate=False):
    """Against 64 bits: a unit of 2^-23 for each addition of up to three parts; an fp16 value's parts are 2^-21 off at
    most, two of bf16 2^-15; the output."""
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()
    rows = M if which == int8.GRAD_WEIGHT else N
    codes, scales = codes_of(rows, K, seed), scales_of(rows, seed, pow2)
    v, d = torch.from_numpy(O.values64(codes, scales)).cuda(), dy.double()
    d = d.t() if which == int8.GRAD_WEIGHT else d
    want, size = d @ v, d.abs() @ v.abs()
    run = int8.grad_weight if which == int8.GRAD_WEIGHT else int8.grad_input
    old = torch.randn(want.shape, generator=torch.Generator().manual_seed(1)).to(out_type).cuda() if accumulate else None
    out = O.strided(old if accumulate else torch.zeros(want.shape, dtype=out_type, device="cuda"), 3, 1)
    run(dy, padded(codes), torch.from_numpy(scales).cuda(), out=out, accumulate=accumulate)
    bound = ((3 * rows + 2) * 2 * O.U32 + (2.0 ** -15 if out_type is torch.bfloat16 else 2.0 ** -21 if dtype is torch.float16 else 0.0)) * size
    if accumulate:
        want = want + old.double()
        bound = bound + 2 * O.U32 * (size + old.double().abs())
    if which == int8.GRAD_INPUT and dtype is out_type is torch.bfloat16:
        bound = bound + 2.0 ** -11 * size + 2.0 ** -39 * (dy.double() * torch.from_numpy(scales).cuda().double()).abs().max(1).values[:, None] * 127 * N
    bound = bound + 1.01 * O.U[out_type] * want.abs() + O.TINY[out_type]
    O.close(O.host(out), want.cpu().numpy(), bound.cpu().numpy())
    gap = torch.as_strided(out, (want.shape[0] - 1, 3), (K + 3, 1), 1 + K)
    assert torch.isnan(gap.float()).all()


@pytest.mark.parametrize("which", [int8.GRAD_WEIGHT, int8.GRAD_INPUT])
@pytest.mark.parametrize("form", GRAD_FORMS)
def test_gradient(form, which):
    force(form)
    across, contraction = tokens_of(form), 64 * 8 + 13
    for dtype, out_type in ((torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16)):
        for pow2 in (False, True):
            M, N = (contraction, across) if which == int8.GRAD_WEIGHT else (across, contraction)
            check_gradient(which, M, N, 300, dtype, out_type, pow2, seed=1, accumulate=not pow2)
    M, N = (512, across) if which == int8.GRAD_WEIGHT else (across, 512)
    check_gradient(which, M, N, 129, torch.bfloat16, torch.float32, True, seed=2)
    if form[2] == 1:
        check_gradient(which, 3, 2, 5, torch.bfloat16, torch.float32, False, seed=3)


@pytest.mark.parametrize("which", [int8.GRAD_WEIGHT, int8.GRAD_INPUT])
@pytest.mark.parametrize("pow2", [True, False])
def test_gradient_of_many_tiles_a_pair(which, pow2):
    """13 x 12 tiles among 74 pairs, several chunks of the contraction each."""
    force(PAIRS)
    M, N = (2200, 3000) if which == int8.GRAD_WEIGHT else (3000, 2200)
    check_gradient(which, M, N, 3300, torch.bfloat16, torch.float32, pow2, seed=4)


@pytest.mark.parametrize("contraction", [8192, 16384])
@pytest.mark.parametrize("form", [PAIRS, (int8.KERNEL_CLUSTER, 64, 1), (int8.KERNEL_CLUSTER, 128, 3)])
@pytest.mark.parametrize("which,pow2", [(int8.GRAD_WEIGHT, True), (int8.GRAD_INPUT, True), (int8.GRAD_WEIGHT, False), (int8.GRAD_INPUT, False)])
def test_sums_leave_the_accumulator_in_time(which, pow2, form, contraction):
    """Positive terms, whose running sum only grows.  The tensor cores cut off what is below a unit of it, 2^-23 of its size at most, at each
    of a chunk's 32 additions of 16 terms, the running sum being half of the chunk's in the mean: below 32 * 2^-24 = 1.9e-6 of the sum.  The
    parts behind the first are 2^-7 of it and come before it.  A sum that stayed in the accumulator would be 512 or 1024 such additions long:
    3e-5 or 6e-5 at most, a quarter to half of that in the mean."""
    force(form)
    N, K = (3000, 3300) if form == PAIRS and contraction == 8192 else (300, 290)
    g = torch.Generator().manual_seed(contraction)
    dy = (torch.rand(*((contraction, N) if which == int8.GRAD_WEIGHT else (N, contraction)), generator=g) + 0.5).bfloat16().cuda()
    codes = torch.from_numpy(np.abs(codes_of(contraction, K, 3)).astype(np.int8)).cuda()
    codes = torch.cat([codes, codes.new_zeros(contraction, -K % 16)], 1)[:, :K]
    scales = torch.from_numpy(scales_of(contraction, 5, pow2)).cuda()
    run = int8.grad_weight if which == int8.GRAD_WEIGHT else int8.grad_input
    got = run(dy, codes, scales, dtype=torch.float32)
    d, v = dy.double(), codes.double() * scales.double()[:, None]
    want = (d.t() if which == int8.GRAD_WEIGHT else d) @ v
    off = (got.double() - want) / want
    assert abs(off.mean().item()) <= 1.95e-6, off.mean().item()


@pytest.mark.parametrize("form", [None, PAIRS, (int8.KERNEL_CLUSTER, 64, 1)])
def test_sums_of_a_16_bit_output_too(form):
    """A million tokens: 65536 additions of 16 positive terms each, which an accumulator that cuts off would lose up to 3.9e-3 of; of
    8192 terms at a time 512 * 2^-24 = 3.1e-5.  fp16's rounding, 2.1e-4 in the mean and independent from column to column of dY (their factors
    differ), leaves 2.6e-5 in the mean of 64 of them, of which four times are allowed."""
    if form:
        force(form)
    M, N, K = (1 << 20) + 100, 64, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    factor = torch.exp(torch.randn(N, device="cuda", generator=g)) * 2.0 ** -13
    dy = ((torch.rand(M, N, device="cuda", generator=g) + 0.5) * factor).half()
    codes = torch.randint(1, 128, (M, K), device="cuda", generator=g, dtype=torch.int8)
    scales = torch.full((M,), 2.0 ** -6, device="cuda")
    got = int8.grad_weight(dy, codes, scales, dtype=torch.float16)
    want = dy.double().t() @ (codes.double() * 2.0 ** -6)
    off = (got.double() - want) / want
    assert abs(off.mean().item()) <= 3.1e-5 + 4 * 2.6e-5, off.mean().item()


# ------------------------------------------------------------------------------------------------ choice and refusals
def test_choice():
    shape = lambda *a, **k: tuple(int8.product_shape(*a, **k))
    assert shape(int8.MATMUL, 8, 4096, 4096) == FEW
    assert shape(int8.MATMUL, 9, 4096, 4096)[0] == int8.KERNEL_CLUSTER
    assert shape(int8.MATMUL, 16384, 8192, 8192, torch.bfloat16) == PAIRS
    assert shape(int8.GRAD_WEIGHT, 8192, 8192, 8192) == shape(int8.GRAD_INPUT, 8192, 8192, 8192, torch.bfloat16) == PAIRS
    assert shape(int8.GRAD_WEIGHT, 64, 64, 64)[0] == shape(int8.GRAD_INPUT, 64, 64, 64)[0] == int8.KERNEL_CLUSTER


def test_refusals():
    for form in ((0, 256, 1), (4, 64, 1), (1, 128, 1), (1, 256, 2), (2, 256, 1), (2, 48, 1), (2, 64, 0), (2, 64, 9), (3, 16, 1), (3, 8, 2)):
        with pytest.raises(fmm.FmmError) as e:
            int8.force_product_shape(*form)
        assert e.value.status == 1
    b, s = padded(codes_of(20, 200, 0)), torch.ones(20, device="cuda")
    dy = torch.zeros(20, 40, dtype=torch.bfloat16, device="cuda")
    for form, call in ((FEW, lambda: int8.matmul(b, s, b, s)), ((2, 64, 3), lambda: int8.matmul(b, s, b, s)), (FEW, lambda: int8.grad_weight(dy, b, s)),
                       ((2, 32, 1), lambda: int8.grad_weight(dy, b, s)), ((2, 64, 2), lambda: int8.grad_weight(dy, b, s))):
        int8.force_product_shape(*form)
        with pytest.raises(fmm.FmmError) as e:
            call()
        assert e.value.status == 2


def test_forced_for_the_calling_thread_alone():
    import threading
    seen = []
    force(PAIRS)
    t = threading.Thread(target=lambda: seen.append(tuple(int8.product_shape(int8.MATMUL, 4, 64, 64))))
    t.start()
    t.join()
    assert seen == [FEW] and tuple(int8.product_shape(int8.MATMUL, 4, 64, 64)) == PAIRS
