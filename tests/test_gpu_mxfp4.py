"""GPU parity of include/class_mxfp4.h against plain implementations in 64 bits: codes, exponents and values bit for bit; logits bit for bit
where every sum is a 32-bit number whatever its order, else within the roundings of their sums."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U32, TYPES = 2.0 ** -24, {torch.float32: 0.0, torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2}
INF = float("inf")
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def ks():
    import paper_2102_06025_amd as ks
    ks.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return ks


@pytest.fixture(autouse=True)
def name_the_case(request):
    print(f"[mxfp4] {request.node.name}", flush=True)


def rng_of(*seed):
    return np.random.default_rng([2102, 4, *seed])


# ---------------------------------------------------------------------------------------------------- plain forms
def plain_codes(V):
    """Codes [n, D] (bit 3: the sign, none for 0) and exponent bytes [n, ceil(D / 32)]."""
    V = np.asarray(V, dtype=np.float64)
    n, D = V.shape
    nb = (D + 31) // 32
    v = np.zeros((n, nb * 32))
    v[:, :D] = V
    v = v.reshape(n, nb, 32)
    top = np.abs(v).max(2)
    broken = ~np.isfinite(v).all(2)
    e = np.where((top > 0) & ~broken, np.maximum(np.frexp(np.where(broken, 1.0, top))[1] - 3, -127), -127)
    a = np.abs(np.where(broken[:, :, None], 0.0, v)) / np.exp2(e)[:, :, None]
    gap = np.abs(a[..., None] - GRID)
    gap[..., 1::2] += 1e-12  # of two equally near ones the even code: other gaps differ by 2^-24 at least
    code = gap.argmin(3)
    code += 8 * ((v < 0) & (code > 0))
    return code.reshape(n, -1)[:, :D], np.where(broken, 255, e + 127)


def plain_values(code, e):
    n, D = code.shape
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    unit = np.where(e == 255, np.nan, np.exp2(e.astype(np.float64) - 127))
    return v * np.repeat(unit, 32, 1)[:, :D]


def rows_of(codes, n, D, classes):
    """The documented order of codes and exponents, undone; what lies beyond the rows has to be 0.  A negative 0 counts as 0."""
    P, Q = (D + 63) // 64, (D + 255) // 256
    c = codes.cpu().numpy().reshape(-1, P * 1024 + Q * 256)
    q = c[:, :P * 1024].reshape(-1, P, 2, 32, 16)
    q = np.stack([q & 15, q >> 4], 5).transpose(0, 3, 1, 2, 4, 5).reshape(-1, 32, P * 64)  # group, row, element
    e = c[:, P * 1024:].reshape(-1, Q, 2, 32, 4).transpose(0, 3, 1, 4, 2).reshape(-1, 32, Q * 8)

    def order(t):
        return (t.reshape(-1, 2, 32, t.shape[2]).transpose(0, 2, 1, 3) if classes else t).reshape(-1, t.shape[2])
    q, e = order(q).astype(np.int64), order(e).astype(np.int64)
    q[q == 8] = 0
    assert not q[n:].any() and not q[:, D:].any() and not e[n:].any() and not e[:, (D + 31) // 32:].any()
    return q[:n, :D], e[:n, :(D + 31) // 32]


def check_codes(codes, V, classes):
    n, D = V.shape
    q, e = rows_of(codes, n, D, classes)
    want_q, want_e = plain_codes(V.double().cpu().numpy())
    assert np.array_equal(e, want_e)
    assert np.array_equal(q, want_q)


# ---------------------------------------------------------------------------------------------------- codes
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("classes", [False, True])
@pytest.mark.parametrize("n,D", [(1, 1), (5, 31), (33, 128), (65, 257), (129, 333), (300, 512), (40, 1_100), (3, 4_097)])
def test_codes_and_back(ks, n, D, classes, dtype):
    r = rng_of(n, D, classes)
    V = torch.from_numpy((r.standard_normal((n, D)) * np.exp(r.uniform(-8, 8, (n, 1)))).astype(np.float32)).cuda().to(dtype)
    codes = ks.class_quantize_mxfp4(V, classes=classes)
    check_codes(codes, V, classes)
    want = plain_values(*plain_codes(V.double().cpu().numpy()))
    for t in (torch.float32, torch.bfloat16):
        back = ks.class_dequantize_mxfp4(codes, n, D, classes=classes, dtype=t)
        assert back.dtype == t and np.array_equal(back.double().cpu().numpy(), want)
    # values that the codes hold keep their codes
    again = ks.class_quantize_mxfp4(back, classes=classes)
    assert torch.equal(rows_values(ks, again, n, D, classes), back)


def rows_values(ks, codes, n, D, classes):
    return ks.class_dequantize_mxfp4(codes, n, D, classes=classes)


def test_borders_and_ends_of_the_range(ks):
    """Every middle of two values and its neighbours, for block exponents from the least to the largest; rows below the least one."""
    middle = (GRID[1:] + GRID[:-1]) / 2
    rows = []
    for e in (-126, -125, -60, 0, 30, 100, 125):
        at = np.concatenate([GRID, middle]).astype(np.float32)
        for f in (at, np.nextafter(at, np.float32(INF)), np.nextafter(at, np.float32(-INF))):
            for sign in (1, -1):
                rows.append(np.pad(np.concatenate([[4.0], f]) * sign, (0, 32 - 1 - len(at))).astype(np.float64) * 2.0 ** e)
    rows.append(np.full(32, 3.4028234e38))
    rows.append(np.linspace(-7.99, 7.99, 32))
    for tiny in (1e-45, 1e-40, 2.0 ** -127, 2.0 ** -126, 1.5 * 2.0 ** -125, 2.0 ** -124):
        rows.append(np.linspace(-1, 1, 32) * tiny)
    rows.append(np.zeros(32))
    rows.append(-np.zeros(32))
    V = torch.from_numpy(np.stack(rows).astype(np.float32)).cuda()
    codes = ks.class_quantize_mxfp4(V)
    check_codes(codes, V, False)
    want = plain_values(*plain_codes(V.double().cpu().numpy()))
    for t in (torch.float32, torch.bfloat16):
        assert np.array_equal(ks.class_dequantize_mxfp4(codes, len(rows), 32, dtype=t).double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,D,ld,shift", [(70, 100, 100, 0), (33, 512, 520, 0), (50, 333, 341, 3), (65, 64, 71, 1)])
def test_strides(ks, n, D, ld, shift, dtype):
    r = rng_of(n, D, ld)
    store = torch.from_numpy(r.standard_normal(n * ld + shift).astype(np.float32)).cuda().to(dtype)
    V = store[shift:].view(n, ld)[:, :D]
    for classes in (False, True):
        codes = ks.class_quantize_mxfp4(V, classes=classes)
        check_codes(codes, V, classes)
        to = torch.full((n * ld + shift,), 7.0, device="cuda", dtype=dtype)
        out = to[shift:].view(n, ld)[:, :D]
        assert ks.class_dequantize_mxfp4(codes, n, D, classes=classes, out=out) is out
        assert np.array_equal(out.double().cpu().numpy(), plain_values(*plain_codes(V.double().cpu().numpy())))
        rest = to.clone()
        rest[shift:].view(n, ld)[:, :D] = 7.0
        assert (rest == 7.0).all()


def test_infinities_and_nan_stay_in_their_block_and_reach_the_row(ks):
    r = rng_of(1)
    V = torch.from_numpy(r.standard_normal((70, 200)).astype(np.float32)).cuda()
    V[3, 40], V[5, 199], V[69, 0] = INF, float("nan"), -INF
    for classes in (False, True):
        codes = ks.class_quantize_mxfp4(V, classes=classes)
        check_codes(codes, V, classes)
        back = ks.class_dequantize_mxfp4(codes, 70, 200, classes=classes)
        assert [tuple(x) for x in back.isnan().nonzero()[:, 0].unique(return_counts=True)[0][:, None].tolist()] == [(3,), (5,), (69,)]
        assert back.isnan().sum().item() == 32 + 8 + 32
    x = torch.from_numpy(r.standard_normal((40, 200)).astype(np.float32)).cuda()
    z = ks.class_logits_mxfp4(ks.class_quantize_mxfp4(x), codes, 40, 70, 200, 1.0)
    bad = torch.zeros(70, dtype=torch.bool, device="cuda")
    bad[[3, 5, 69]] = True
    assert torch.equal(z.isnan(), bad.expand(40, 70))
    z = ks.class_logits_mxfp4(ks.class_quantize_mxfp4(V), ks.class_quantize_mxfp4(x, classes=True), 70, 40, 200, 1.0, dtype=torch.bfloat16)
    assert torch.equal(z.isnan(), bad[:, None].expand(70, 40))


# ---------------------------------------------------------------------------------------------------- logits
def few_bits(gen, n, D):
    """Rows of 4-bit values whose blocks' exponents are 0, 1 or 2: products are multiples of 1/4 below 36 * 16, so that all sums of up to
    4,096 of them are 32-bit numbers."""
    v = torch.tensor(GRID, dtype=torch.float32, device="cuda")[torch.randint(0, 8, (n, D), generator=gen, device="cuda")]
    v *= 1 - 2 * torch.randint(0, 2, (n, D), generator=gen, device="cuda")
    v[:, ::32] = 4.0  # keeps the block's exponent
    e = torch.randint(0, 3, (n, (D + 31) // 32), generator=gen, device="cuda").repeat_interleave(32, 1)[:, :D]
    return torch.ldexp(v, e)


def product(x, w):
    return torch.cat([x.double() @ part.double().t().contiguous() for part in w.split(1 << 15)], 1)


def same_logits(ks, B, C, D, dtype, bias, pad=None, shift=0, w=None, w_codes=None):
    gen = torch.Generator("cuda").manual_seed(B * 7 + C * 3 + D)
    x = few_bits(gen, B, D)
    if w is None:
        w = few_bits(gen, C, D)
        w_codes = ks.class_quantize_mxfp4(w, classes=True)
    b = torch.randint(-1000, 1000, (C,), generator=gen, device="cuda").float() if bias else None
    ld = (C + 63) // 64 * 64 if pad is None else C + pad
    store = torch.full((B * ld + shift + 64,), 7.0, device="cuda", dtype=dtype)
    out = torch.as_strided(store, (B, C), (ld, 1), shift)
    # scale 1/4: the scaled sum is exact, the bias is added with one rounding, which is none here either
    ks.class_logits_mxfp4(ks.class_quantize_mxfp4(x), w_codes, B, C, D, 0.25, bias=b, out=out)
    want = product(x, w) * 0.25 + (0.0 if b is None else b.double())
    assert (want == want.float().double()).all()
    assert torch.equal(out, want.to(dtype)), (out.double() - want).abs().max().item()
    out.fill_(7.0)
    assert (store == 7.0).all(), "written outside the logits"


SIZES = [(1, 1, 1), (1, 64, 64), (2, 63, 65), (31, 65, 32), (32, 130, 200), (33, 1_000, 96), (64, 500, 256), (65, 127, 300), (1, 10_000, 128), (7, 3_001, 1_024),
         (5, 700, 2_049), (40, 640, 1_500), (77, 5_021, 333), (128, 4_096, 512), (200, 2_051, 1_024), (300, 1_500, 1_100), (129, 9_000, 64), (257, 777, 4_096),
         (1_030, 330, 160), (513, 20_000, 130), (96, 40_000, 512), (320, 33_001, 512), (1_024, 16_390, 512), (260, 30_011, 800), (520, 20_001, 2_050)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,D", SIZES)
def test_logits_without_roundings(ks, B, C, D, dtype):
    same_logits(ks, B, C, D, dtype, bias=(B + C) % 2 == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,D,pad,shift", [(3, 101, 96, 0, 0), (3, 101, 96, 1, 1), (70, 1_001, 512, 0, 1), (70, 1_001, 512, 1, 0), (300, 9_001, 512, 5, 0), (300, 9_001, 512, 0, 0),
                                             (150, 6_000, 1_300, 2, 0), (150, 6_001, 1_300, 4, 1), (40, 63, 64, 1, 0), (1_030, 40, 320, 0, 0), (300, 9_002, 512, 0, 0)])
def test_rows_that_lie_apart_or_beside_the_lines(ks, B, C, D, pad, shift, dtype):
    same_logits(ks, B, C, D, dtype, bias=True, pad=pad, shift=shift)


@pytest.mark.parametrize("B,C,D", [(3, 500, 40), (70, 3_000, 512), (300, 9_001, 700), (130, 5_000, 4_096)])
def test_logits_of_ordinary_rows(ks, B, C, D):
    """A sum of D products in 32 bits is off by D roundings or cuttings (2^-23) of the sum of their magnitudes at most, in any order."""
    gen = torch.Generator("cuda").manual_seed(D)
    x, w = torch.randn((B, D), generator=gen, device="cuda"), torch.randn((C, D), generator=gen, device="cuda").to(torch.bfloat16)
    x *= torch.exp(4 * torch.randn((B, D), generator=gen, device="cuda"))
    bias = torch.randn(C, generator=gen, device="cuda")
    xc, wc = ks.class_quantize_mxfp4(x), ks.class_quantize_mxfp4(w, classes=True)
    xv, wv = ks.class_dequantize_mxfp4(xc, B, D, dtype=torch.float32), ks.class_dequantize_mxfp4(wc, C, D, classes=True, dtype=torch.float32)
    want, size = product(xv, wv) * 30.0 + bias.double(), product(xv.abs(), wv.abs()) * 30.0
    for dtype in (torch.float32, torch.bfloat16):
        z = ks.class_logits_mxfp4(xc, wc, B, C, D, 30.0, bias=bias, dtype=dtype)
        off = (z.double() - want).abs() - 1.01 * (2 * U32 * D * size + U32 * want.abs() + TYPES[dtype] * want.abs())
        assert off.max().item() <= 0


def test_many_samples_of_few_classes(ks):
    same_logits(ks, 40_001, 10, 96, torch.float32, bias=True, pad=2)
    same_logits(ks, 9_000, 600, 512, torch.bfloat16, bias=False)


def test_streams_and_graphs(ks):
    gen = torch.Generator("cuda").manual_seed(11)
    B, C, D = 70, 3_000, 512
    x, w = few_bits(gen, B, D), few_bits(gen, C, D)
    wc = ks.class_quantize_mxfp4(w, classes=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    xc = ks.class_quantize_mxfp4(x, stream=side)
    z = ks.class_logits_mxfp4(xc, wc, B, C, D, 1.0, stream=side)
    side.synchronize()
    assert torch.equal(z.double(), product(x, w))
    # a captured run of quantisation, product and the way back, replayed on new features with eager work in between
    x_in, out, back = x.clone(), torch.empty((B, C), device="cuda"), torch.empty((B, D), device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ks.class_quantize_mxfp4(x_in, codes=xc)
        ks.class_logits_mxfp4(xc, wc, B, C, D, 1.0, out=out)
        ks.class_dequantize_mxfp4(xc, B, D, out=back)
    for _ in range(3):
        x_in.copy_(few_bits(gen, B, D))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.double(), product(x_in, w)) and torch.equal(back, x_in)
        eager = ks.class_logits_mxfp4(ks.class_quantize_mxfp4(x_in), wc, B, C, D, 1.0)
        assert torch.equal(out, eager)


def test_refusals_of_tensors(ks):
    c = ks.class_quantize_mxfp4(torch.ones((3, 64), device="cuda"))
    w = ks.class_quantize_mxfp4(torch.ones((5, 64), device="cuda"), classes=True)
    with pytest.raises(ValueError):
        ks.class_logits_mxfp4(c, w, 33, 5, 64, 1.0)
    with pytest.raises(ValueError):
        ks.class_logits_mxfp4(c, w, 3, 65, 64, 1.0)
    with pytest.raises(ValueError):
        ks.class_logits_mxfp4(c, w, 3, 5, 64, 1.0, out=torch.empty((3, 6), device="cuda"))
    with pytest.raises(TypeError):
        ks.class_logits_mxfp4(c, w, 3, 5, 64, 1.0, out=torch.empty((3, 5), device="cuda", dtype=torch.float16))
    with pytest.raises(TypeError):
        ks.class_quantize_mxfp4(torch.ones((3, 64), device="cuda").t())
    with pytest.raises(ValueError):
        ks.class_quantize_mxfp4(torch.ones((3, 64), device="cuda"), codes=torch.empty(7, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        ks.class_dequantize_mxfp4(c, 33, 64)


def test_every_middle_at_every_exponent(ks):
    """The middles of two values, their neighbours in 32 bits and the values themselves, for every exponent that a block can have."""
    at = np.concatenate([GRID, (GRID[1:] + GRID[:-1]) / 2]).astype(np.float32)
    rows = []
    for e in range(-130, 126):
        for f in (at, np.nextafter(at, np.float32(INF)), np.nextafter(at, np.float32(-INF))):
            for sign in (1, -1):
                rows.append(np.pad(np.concatenate([[4.0], f]) * sign, (0, 32 - 1 - len(at))).astype(np.float64) * 2.0 ** e)
    V = torch.from_numpy(np.stack(rows).astype(np.float32)).cuda()  # below 2^-126 the neighbours fall on the middles or on multiples of 2^-149
    for classes in (False, True):
        codes = ks.class_quantize_mxfp4(V, classes=classes)
        check_codes(codes, V, classes)
    assert sorted(set(plain_codes(V.double().cpu().numpy())[1][:, 0].tolist())) == list(range(0, 253))
    want = plain_values(*plain_codes(V.double().cpu().numpy()))
    for t in (torch.float32, torch.bfloat16):
        assert np.array_equal(ks.class_dequantize_mxfp4(codes, len(rows), 32, classes=True, dtype=t).double().cpu().numpy(), want)


# The ways of the product: wavefronts of their own; samples in LDS, for up to 256 and up to 512 elements, where there are many groups of 64 classes and
# products; chunks of depth through LDS for more.  The sizes lie well inside each, or on both sides of where one begins.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,D", [
    # samples in LDS, 257 to 512 elements: whole ones and ragged ones, even and odd numbers of classes, more than eight tiles of samples
    (1_024, 16_389, 512), (1_024, 16_391, 333), (1_040, 24_000, 448), (2_049, 20_001, 257), (4_200, 10_500, 512), (8_300, 10_303, 400),
    # up to 256 elements, 1 to 4 pieces
    (1_024, 20_001, 200), (1_030, 20_002, 150), (1_024, 51_300, 100), (1_024, 51_301, 64), (2_050, 60_000, 33), (9_000, 11_003, 256),
    # on both sides of 160 groups of classes, 3,800 and 1,280 wavefronts
    (4_096, 10_240, 512), (4_096, 10_241, 512), (1_024, 15_168, 512), (1_024, 15_233, 512), (640, 8_192, 576), (640, 8_193, 576),
    # chunks of depth: more than 32 tiles of samples, few tiles of classes, ragged depths
    (4_200, 5_000, 640), (20_000, 500, 576), (20_001, 513, 1_000), (9_000, 1_001, 520), (1_024, 16_391, 1_025)])
def test_every_way_of_the_product(ks, B, C, D, dtype):
    same_logits(ks, B, C, D, dtype, bias=(B + C + D) % 2 == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,D,pad,shift", [(300, 30_011, 800, 0, 0), (300, 30_010, 800, 1, 1), (300, 30_010, 800, 2, 1), (1_024, 20_001, 200, 1, 0), (1_024, 20_000, 200, 6, 2),
                                             (1_024, 20_002, 512, 0, 1), (1_030, 20_003, 512, 3, 0)])
def test_rows_beside_the_lines_on_every_way(ks, B, C, D, pad, shift, dtype):
    same_logits(ks, B, C, D, dtype, bias=True, pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_lie_far_apart(ks, dtype):
    """64 MB from row to row and more, offsets beyond 32 bits: stored element by element."""
    ld = (1 << 26) // dtype.itemsize + 2
    same_logits(ks, 70, 101, 96, dtype, bias=True, pad=ld - 101)


def test_a_matrix_of_more_than_2_31_elements(ks):
    gen = torch.Generator("cuda").manual_seed(12)
    B, C, D = 5_600, 390_625, 64
    x, w = few_bits(gen, B, D), few_bits(gen, C, D)
    z = ks.class_logits_mxfp4(ks.class_quantize_mxfp4(x), ks.class_quantize_mxfp4(w, classes=True), B, C, D, 0.25, dtype=torch.bfloat16)
    assert B * z.stride(0) > 1 << 31
    for first in range(0, B, 700):
        assert torch.equal(z[first:first + 700], (product(x[first:first + 700], w) * 0.25).to(torch.bfloat16)), first
