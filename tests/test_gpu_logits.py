"""GPU parity of include/class_logits.h against plain implementations in 64 bits: codes bit for bit, logits and adjusted logits within the
roundings that their formulas count (2^-24 for each fp32 operation, half a step of the type for the stored value)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U32, TYPES = 2.0 ** -24, {torch.float32: 0.0, torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2}
INF = float("inf")


@pytest.fixture(scope="module")
def ks():
    import paper_2102_06025_amd as ks
    ks.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return ks


@pytest.fixture(autouse=True)
def name_the_case(request):
    print(f"[logits] {request.node.name}", flush=True)


def rng_of(*seed):
    return np.random.default_rng([2102, *seed])


# ---------------------------------------------------------------------------------------------------- plain forms
def plain_codes(V, normalize=False):
    """Codes and 64-bit scales.  127 v is exact in 64 bits and a quotient of two 32-bit numbers is no nearer to a half than 2^-32
    without being one, so rint() of the rounded quotient is the code."""
    V = np.asarray(V, dtype=np.float64)
    q, s = np.zeros(V.shape, dtype=np.int64), np.zeros(len(V))
    for i, v in enumerate(V):
        a = np.abs(v).max()
        if not np.isfinite(v).all():
            s[i] = np.nan
        elif a > 0:
            q[i] = np.rint(v * 127.0 / a)
            s[i] = a / 127.0 / (np.sqrt((v * v).sum()) if normalize else 1.0)
    return q, s


def rows_of(codes, n, D, classes):
    """The documented order of the codes, undone; what lies beyond the rows has to be 0."""
    kb = (D + 31) // 32
    c = codes.cpu().numpy().reshape(-1, kb, 2, 32, 16).transpose(0, 3, 1, 2, 4).reshape(-1, 32, kb * 32)  # block, row, element
    if classes:
        c = c.reshape(-1, 2, 32, kb * 32).transpose(0, 2, 1, 3)
    c = c.reshape(-1, kb * 32)
    assert not c[n:].any() and not c[:, D:].any()
    return c[:n, :D]


def plain_logits(q, s, w, t, scale, bias):
    """-> logits, and the sum of the magnitudes that roundings are relative to: four on the product, one on the sum."""
    z = (q.astype(np.int64) @ w.astype(np.int64).T).astype(np.float64) * (scale * s[:, None]) * t[None, :]
    out = z + (0.0 if bias is None else bias[None, :].astype(np.float64))
    return out, 4 * np.abs(z) + np.abs(out)


def near(got, want, size, dtype, tag=""):
    g, finite = got.double().cpu().numpy(), np.isfinite(want)
    assert np.array_equal(np.isnan(g), np.isnan(want)), tag
    assert np.array_equal(g[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)]), tag
    # 1.01: products of roundings; fp32 values below the normal range are stored in steps of 2^-149
    g, want, size = g[finite], want[finite], size[finite]
    off = np.abs(g - want) - 1.01 * (U32 * size + TYPES[dtype] * np.abs(want)) - 2.0 ** -149
    assert off.size == 0 or off.max() <= 0, (tag, off.max())


# ---------------------------------------------------------------------------------------------------- codes
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("classes,normalize", [(False, False), (True, True), (True, False)])
@pytest.mark.parametrize("n,D", [(1, 1), (5, 31), (33, 128), (129, 333), (300, 512), (40, 1_100), (3, 4_097)])
def test_codes(ks, n, D, classes, normalize, dtype):
    r = rng_of(n, D, classes)
    V = torch.from_numpy((r.standard_normal((n, D)) * np.exp(r.uniform(-8, 8, (n, 1)))).astype(np.float32)).cuda().to(dtype)
    codes, scale = ks.class_quantize_rows(V, classes=classes, normalize=normalize)
    q, s = plain_codes(V.float().cpu().numpy(), normalize)
    assert np.array_equal(rows_of(codes, n, D, classes), q)
    # the 64-bit scale is off by less than 1e-12 of itself and rounded once
    assert (np.abs(scale.cpu().numpy() - s) <= 1.0001 * U32 * s).all()


def rows_of_gpu(codes, n, D, classes):
    c = codes.view(-1, (D + 31) // 32, 2, 32, 16).permute(0, 3, 1, 2, 4).reshape(-1, 32, (D + 31) // 32 * 32)
    c = (c.view(-1, 2, 32, c.shape[2]).transpose(1, 2) if classes else c).reshape(-1, c.shape[2])
    assert not c[n:].any() and not c[:, D:].any()
    return c[:n, :D]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("classes,normalize", [(False, False), (True, True), (False, True)])
@pytest.mark.parametrize("n,D", [(16_353, 33), (16_384, 256), (20_001, 300), (17_000, 512), (33_333, 700), (16_400, 1_024), (16_500, 1_500)])
def test_codes_of_many_rows(ks, n, D, classes, normalize, dtype):
    gen = torch.Generator("cuda").manual_seed(n + D)
    V = torch.randn((n, D), generator=gen, device="cuda") * torch.exp(16 * torch.rand((n, 1), generator=gen, device="cuda") - 8)
    V[n // 2], V[n - 1, D // 2], V[3, 0] = 0.0, float("nan"), INF
    V = V.to(dtype)
    codes, scale = ks.class_quantize_rows(V, classes=classes, normalize=normalize)
    v = V.double()
    top = v.abs().amax(1)
    broken, a = ~torch.isfinite(top), torch.where(torch.isfinite(top) & (top > 0), top, 1.0)
    assert broken.nonzero().flatten().tolist() == [3, n - 1]
    q = torch.where((broken | (top == 0))[:, None], 0.0, torch.round(v * 127.0 / a[:, None]))
    assert torch.equal(rows_of_gpu(codes, n, D, classes).double(), q)
    s = top / 127.0 / (torch.where(top > 0, (v * v).sum(1).sqrt(), 1.0) if normalize else 1.0)
    assert torch.equal(scale.isnan(), broken)
    assert ((scale.double() - s).abs() <= 1.0001 * U32 * s)[~broken].all()


@pytest.mark.parametrize("classes", [False, True])
@pytest.mark.parametrize("n,D,ld,shift", [(16_400, 64, 64, 0), (17_001, 500, 503, 1), (16_390, 1_000, 1_024, 4), (16_384, 1_100, 1_100, 0)])
def test_bytes_of_many_rows(ks, n, D, ld, shift, classes):
    gen = torch.Generator("cuda").manual_seed(n + D)
    V = torch.randint(-128, 128, (n * ld + shift,), generator=gen, device="cuda", dtype=torch.int8)[shift:].view(n, ld)[:, :D]
    codes, scale = ks.class_quantize_rows(V, classes=classes)
    assert scale is None and torch.equal(rows_of_gpu(codes, n, D, classes), V)


def test_codes_at_the_borders(ks):
    """Halves go to the even code, and values next to a half to their own side: rows whose largest value is 127 * 2^e, and rows of
    any largest value with the fp32 numbers around each border."""
    rows = []
    half = (np.arange(-127, 127) + 0.5)
    for e in (-130, -20, 0, 60, 120):
        rows.append(np.concatenate([[127.0], half, [0.0, -0.0]]) * 2.0 ** e)
    for a in (1.0, 3.0, 0.7, 1e-39, 3e38):
        a = np.float32(a)
        at = (half * (np.float64(a) / 127.0)).astype(np.float32)
        for step in (-INF, INF):
            rows.append(np.concatenate([[a], np.nextafter(at, np.float32(step)), at[:2]]))
        rows.append(np.concatenate([[a], at, at[:2]]))
    V = np.stack(rows).astype(np.float32)
    codes, scale = ks.class_quantize_rows(torch.from_numpy(V).cuda())
    q, s = plain_codes(V)
    assert np.array_equal(rows_of(codes, *V.shape, False), q)
    assert (np.abs(scale.cpu().numpy() - s) <= 1.0001 * U32 * s + 2.0 ** -150).all()


@pytest.mark.parametrize("n", [1, 16_400])
def test_codes_of_every_bf16_value(ks, n):
    """All bf16 values of the eleven binades up to the largest of the row, both signs: ties among them in every row."""
    for top in (0x7F7F, 0x7F00, 0x7E81, 0x3F80, 0x3FD5, 0x3F83, 0x2001, 0x0D81, 0x0D7F, 0x0600, 0x0087):
        bits = np.arange(max(1, top - 11 * 128), top + 1, dtype=np.int64)
        bits = np.concatenate([bits, bits | 0x8000])
        row = torch.from_numpy((bits << 16).astype(np.uint32).view(np.float32)).cuda()
        V = row.to(torch.bfloat16)[None].expand(n, -1).contiguous()
        codes, scale = ks.class_quantize_rows(V)
        q, s = plain_codes(row.cpu().numpy()[None])
        assert torch.equal(rows_of_gpu(codes, n, len(bits), False), torch.from_numpy(q.astype(np.int8)).cuda().expand(n, -1)), hex(top)
        assert (np.abs(scale.cpu().numpy() - s) <= 1.0001 * U32 * s + 2.0 ** -150).all()


def test_codes_of_empty_and_broken_rows(ks):
    V = rng_of(3).standard_normal((9, 70)).astype(np.float32)
    V[1], V[2], V[3, 5], V[4, 69], V[5, 0] = 0.0, -0.0, np.inf, np.nan, -np.inf
    for classes in (False, True):
        codes, scale = ks.class_quantize_rows(torch.from_numpy(V).cuda(), classes=classes, normalize=classes)
        q, s = plain_codes(V, classes)
        assert np.array_equal(rows_of(codes, 9, 70, classes), q)
        got = scale.cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(s)) and got[1] == 0 and got[2] == 0
    # a NaN scale reaches every logit of its row or class, a zero row gives the bias
    x, xs = ks.class_quantize_rows(torch.from_numpy(V).cuda())
    w, ws = ks.class_quantize_rows(torch.from_numpy(V).cuda(), classes=True)
    z = ks.class_logits_int8(x, xs, w, ws, 2.0, bias=torch.full((9,), 7.0, device="cuda")).cpu()
    assert z[3:6].isnan().all() and z[:, 3:6].isnan().all() and (z[1, :3] == 7).all() and not z[6:, 6:].isnan().any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.int8])
@pytest.mark.parametrize("D,ld,shift", [(64, 64, 0), (64, 71, 0), (64, 68, 1), (63, 80, 3), (1_030, 1_032, 2)])
def test_rows_that_lie_apart(ks, dtype, D, ld, shift):
    n, r = 45, rng_of(D, ld, shift)
    raw = r.integers(-128, 128, (n * ld + shift)) if dtype == torch.int8 else r.standard_normal(n * ld + shift)
    V = torch.from_numpy(raw.astype(np.float32)).cuda().to(dtype)[shift:].view(n, ld)[:, :D]
    codes, scale = ks.class_quantize_rows(V, classes=True)
    if dtype == torch.int8:
        assert scale is None and np.array_equal(rows_of(codes, n, D, True), V.cpu().numpy())
    else:
        assert np.array_equal(rows_of(codes, n, D, True), plain_codes(V.float().cpu().numpy())[0])


def test_all_bytes_of_given_buffers_are_written(ks):
    V = torch.ones((3, 40), device="cuda")
    for classes in (False, True):
        need = ks.class_codes_bytes(3, 40, classes)
        whole = torch.full((need + 4096,), 85, dtype=torch.int8, device="cuda")
        ks.class_quantize_rows(V, classes=classes, codes=whole[:need], row_scale=torch.empty(3, device="cuda"))
        rows_of(whole[:need], 3, 40, classes)
        assert (whole[need:] == 85).all()


# ---------------------------------------------------------------------------------------------------- product
def product_case(ks, B, C, D, seed, largest=False):
    r = rng_of(B, C, D, seed)
    q = (np.full((B, D), -128) if largest else r.integers(-127, 128, (B, D))).astype(np.int8)
    w = (np.full((C, D), -128) if largest else r.integers(-127, 128, (C, D))).astype(np.int8)
    s, t = r.uniform(0.001, 0.1, B).astype(np.float32), r.uniform(0.001, 0.1, C).astype(np.float32)
    x = ks.class_quantize_rows(torch.from_numpy(q).cuda())[0]
    y = ks.class_quantize_rows(torch.from_numpy(w).cuda(), classes=True)[0]
    return q, s, w, t, x, torch.from_numpy(s).cuda(), y, torch.from_numpy(t).cuda(), r.standard_normal(C).astype(np.float32) * 9


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,D", [(1, 1, 1), (1, 1_000, 64), (2, 129, 33), (31, 127, 96), (32, 4_096, 512), (33, 515, 128), (64, 640, 1_000),
                                   (65, 10_007, 31), (127, 1_025, 544), (128, 128, 32), (129, 5_000, 256), (300, 999, 513), (513, 2_049, 160),
                                   (1_024, 1_537, 64), (256, 512, 4_096), (7, 300, 9_000), (200, 260, 1_056)])
def test_product(ks, B, C, D, dtype):
    q, s, w, t, x, xs, y, ys, bias = product_case(ks, B, C, D, 0)
    for b in (None, bias):
        z = ks.class_logits_int8(x, xs, y, ys, 30.0, bias=None if b is None else torch.from_numpy(b).cuda(), dtype=dtype)
        assert z.dtype == dtype and z.shape == (B, C)
        near(z, *plain_logits(q, s, w, t, 30.0, b), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,D", [(3, 300, 64), (70, 1_000, 160), (300, 777, 96)])
@pytest.mark.parametrize("ld,shift", [(1_001, 0), (1_004, 0), (1_008, 2), (1_024, 1), (1_032, 4)])
def test_logits_rows_that_lie_apart(ks, B, C, D, dtype, ld, shift):
    """A node's columns of a larger matrix: what lies around them stays as it is."""
    q, s, w, t, x, xs, y, ys, bias = product_case(ks, B, C, D, 1)
    whole = torch.full((B * ld + shift,), 77.0, dtype=dtype, device="cuda")
    mat = whole[shift:].view(B, ld)
    z = ks.class_logits_int8(x, xs, y, ys, -2.5, bias=torch.from_numpy(bias).cuda(), out=mat[:, :C])
    near(z, *plain_logits(q, s, w, t, -2.5, bias), dtype)
    assert (whole[:shift] == 77).all() and (mat[:, C:] == 77).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("B,C,D", [
    (300, 40_001, 64), (1_024, 30_000, 33), (257, 65_537, 128), (1_100, 32_700, 128), (1_024, 32_701, 352), (1_000, 32_001, 512), (900, 65_000, 400),
    (2_050, 16_130, 290), (1_024, 20_001, 512), (257, 30_011, 256), (129, 90_001, 160), (1_300, 9_999, 192), (700, 30_007, 768), (300, 40_000, 1_152),
    (600, 20_001, 1_184), (300, 33_000, 4_096), (129, 50_001, 2_500), (2_500, 5_001, 1_300), (64, 70_003, 512), (33, 90_001, 1_024), (20, 200_001, 96),
    (32, 20_000, 800), (50, 16_000, 1_100), (400, 65_500, 320), (500, 65_535, 512), (257, 262_200, 256)])
def test_products_of_many_classes(ks, B, C, D, dtype, apart):
    """Batches, layers and depths on both sides of the sizes at which the work is divided in another way; rows next to each other, and
    rows of an odd distance, with what lies between them."""
    gen = torch.Generator("cuda").manual_seed(B + C + D)
    rand = lambda *n: torch.rand(n, generator=gen, device="cuda")  # noqa: E731
    q, w = (torch.randint(-127, 128, (n, D), generator=gen, device="cuda", dtype=torch.int8) for n in (B, C))
    xs, ws, bias = 0.001 + 0.1 * rand(B), 0.001 + 0.1 * rand(C), 9 * rand(C) - 4.5
    x, y = ks.class_quantize_rows(q)[0], ks.class_quantize_rows(w, classes=True)[0]
    ld, shift = (C + 5 + C % 2, 3) if apart else (C, 0)
    whole = torch.full((B * ld + shift,), 77.0, dtype=dtype, device="cuda")
    mat = whole[shift:].view(B, ld)
    z = ks.class_logits_int8(x, xs, y, ws, 30.0, bias=bias, out=mat[:, :C])
    assert (whole[:shift] == 77).all() and (mat[:, C:] == 77).all()
    for lo in range(0, C, 1 << 14):
        hi = min(C, lo + (1 << 14))
        plain = torch.mm(q.double(), w[lo:hi].double().t().contiguous()) * (30.0 * xs.double())[:, None] * ws[None, lo:hi].double()
        want = plain + bias[None, lo:hi].double()
        off = (z[:, lo:hi].double() - want).abs() - 1.01 * (U32 * (4 * plain.abs() + want.abs()) + TYPES[dtype] * want.abs())
        assert off.max() <= 0, (lo, float(off.max()))


@pytest.mark.parametrize("C,B,D", [(64, 81_920, 512), (1_000, 5_120, 512), (64, 131_072, 128), (500, 10_240, 1_024)])
def test_large_batches_of_few_classes_fill_the_chip(ks, C, B, D):
    """Twice the batch, on the other side of the batch sizes that go to other kernels where there are many classes: about twice the time
    (with the chip left nearly empty it was ten to eighty times)."""
    def least(n):
        x, xs = torch.zeros(ks.class_codes_bytes(n, D), dtype=torch.int8, device="cuda"), torch.ones(n, device="cuda")
        w, ws = torch.zeros(ks.class_codes_bytes(C, D, True), dtype=torch.int8, device="cuda"), torch.ones(C, device="cuda")
        z, times = torch.empty((n, (C + 63) // 64 * 64), device="cuda")[:, :C], []
        for _ in range(4):
            ends = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            torch.cuda.synchronize()
            ends[0].record()
            for _ in range(10):
                ks.class_logits_int8(x, xs, w, ws, 1.0, out=z)
            ends[1].record()
            torch.cuda.synchronize()
            times.append(ends[0].elapsed_time(ends[1]))
        return min(times)
    assert least(2 * B) < 5 * least(B)


@pytest.mark.parametrize("C,ld", [(3, 3), (10, 10), (9, 10)])
def test_product_of_the_largest_batch(ks, C, ld):
    B, D = 4_194_240, 20
    gen = torch.Generator("cuda").manual_seed(C)
    q, w = (torch.randint(-127, 128, (n, D), generator=gen, device="cuda", dtype=torch.int8) for n in (B, C))
    xs, ws = (0.001 + 0.1 * torch.rand(n, generator=gen, device="cuda") for n in (B, C))
    mat = torch.full((B + 70, ld), 77.0, device="cuda")
    z = ks.class_logits_int8(ks.class_quantize_rows(q)[0], xs, ks.class_quantize_rows(w, classes=True)[0], ws, 2.0, out=mat[:B, :C])
    assert (mat[B:] == 77).all() and (mat[:, C:] == 77).all()
    want = torch.mm(q.double(), w.double().t().contiguous()) * (2.0 * xs.double())[:, None] * ws[None].double()
    assert ((z.double() - want).abs() <= 4.1 * U32 * want.abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,D", [(4_500, 8_191, 64), (1_500, 8_257, 320), (1_700, 6_143, 320), (2_000, 6_145, 320), (1_000, 6_144, 1_152), (3_000, 2_048, 1_184), (3_000, 2_049, 1_200), (7_000, 1_999, 31)])
def test_products_on_both_sides_of_few_classes(ks, B, C, D, dtype):
    gen = torch.Generator("cuda").manual_seed(B + C + D)
    rand = lambda *n: torch.rand(n, generator=gen, device="cuda")  # noqa: E731
    q, w = (torch.randint(-127, 128, (n, D), generator=gen, device="cuda", dtype=torch.int8) for n in (B, C))
    xs, ws, bias = 0.001 + 0.1 * rand(B), 0.001 + 0.1 * rand(C), 9 * rand(C) - 4.5
    x, y = ks.class_quantize_rows(q)[0], ks.class_quantize_rows(w, classes=True)[0]
    plain = torch.mm(q.double(), w.double().t().contiguous()) * (30.0 * xs.double())[:, None] * ws[None].double()
    want = plain + bias[None].double()
    for ld in (C, C + 1):
        mat = torch.full((B + 9, ld), 77.0, dtype=dtype, device="cuda")
        z = ks.class_logits_int8(x, xs, y, ws, 30.0, bias=bias, out=mat[:B, :C])
        assert (mat[B:] == 77).all() and (mat[:, C:] == 77).all()
        off = (z.double() - want).abs() - 1.01 * (U32 * (4 * plain.abs() + want.abs()) + TYPES[dtype] * want.abs())
        assert off.max() <= 0, (ld, float(off.max()))


@pytest.mark.parametrize("B", [1, 40, 200])
def test_the_largest_sum(ks, B):
    """-128 everywhere at the largest depth: 2^14 * 2^16 = 2^30."""
    q, s, w, t, x, xs, y, ys, _ = product_case(ks, B, 3, 65_536, 2, largest=True)
    near(ks.class_logits_int8(x, xs, y, ys, 1.0), *plain_logits(q, s, w, t, 1.0, None), torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B", [1, 3, 31, 33, 65])
@pytest.mark.parametrize("D", [33, 200, 800])
def test_few_classes_in_tight_rows(ks, B, D, dtype):
    """Rows of fewer than 64 classes next to each other: the rows behind the last sample are not the call's."""
    for C in (1, 2, 9, 10, 31, 32, 40, 61, 62, 63, 64, 65, 70):
        q, s, w, t, x, xs, y, ys, bias = product_case(ks, B, C, D, 3)
        for ld in (C, C + 1, C + 2):
            mat = torch.full((B + 70, ld), 77.0, dtype=dtype, device="cuda")
            z = ks.class_logits_int8(x, xs, y, ys, 30.0, bias=torch.from_numpy(bias).cuda(), out=mat[:B, :C])
            assert (mat[B:] == 77).all() and (mat[:, C:] == 77).all(), (C, ld)
            near(z, *plain_logits(q, s, w, t, 30.0, bias), dtype, (C, ld))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,D,ld", [(131_100, 10, 64, 10), (131_075, 41, 33, 42), (82_000, 40, 512, 40), (81_985, 63, 300, 64), (82_010, 62, 1_200, 62),
                                      (82_017, 9, 1_184, 10), (82_017, 9, 1_184, 9)])
def test_few_classes_of_a_large_batch_in_tight_rows(ks, B, C, D, ld, dtype):
    """The same for the kernels that large batches take."""
    gen = torch.Generator("cuda").manual_seed(B + C + D)
    rand = lambda *n: torch.rand(n, generator=gen, device="cuda")  # noqa: E731
    q, w = (torch.randint(-127, 128, (n, D), generator=gen, device="cuda", dtype=torch.int8) for n in (B, C))
    xs, ws, bias = 0.001 + 0.1 * rand(B), 0.001 + 0.1 * rand(C), 9 * rand(C) - 4.5
    x, y = ks.class_quantize_rows(q)[0], ks.class_quantize_rows(w, classes=True)[0]
    mat = torch.full((B + 300, ld), 77.0, dtype=dtype, device="cuda")
    z = ks.class_logits_int8(x, xs, y, ws, 30.0, bias=bias, out=mat[:B, :C])
    assert (mat[B:] == 77).all() and (mat[:, C:] == 77).all()
    plain = torch.mm(q.double(), w.double().t().contiguous()) * (30.0 * xs.double())[:, None] * ws[None].double()
    want = plain + bias[None].double()
    off = (z.double() - want).abs() - 1.01 * (U32 * (4 * plain.abs() + want.abs()) + TYPES[dtype] * want.abs())
    assert off.max() <= 0, float(off.max())


def test_codes_and_logits_beyond_32_bits(ks):
    """Weights of more than 4 GB of codes, and rows of logits more than 2^31 elements apart."""
    D, C, B, ld = 4_352, 1_000_064, 3, 1_200_000_000
    r = rng_of(9)
    q, w = r.integers(-127, 128, (B, D)).astype(np.int8), r.integers(-127, 128, (128, D)).astype(np.int8)
    codes = torch.zeros(ks.class_codes_bytes(C, D, True), dtype=torch.int8, device="cuda")
    last = ks.class_quantize_rows(torch.from_numpy(w).cuda(), classes=True)[0]
    codes[-last.numel():] = last
    x = ks.class_quantize_rows(torch.from_numpy(q).cuda())[0]
    out = torch.empty((B, ld), dtype=torch.bfloat16, device="cuda")[:, :C]
    z = ks.class_logits_int8(x, torch.ones(B, device="cuda"), codes, torch.ones(C, device="cuda"), 0.01, out=out)
    want, size = plain_logits(q, np.ones(B), w, np.ones(128), float(np.float32(0.01)), None)
    near(z[:, -128:], want, size, torch.bfloat16)
    assert not z[:, :-128].any()
    allowed = torch.full((1, (C + 31) // 32), -1, dtype=torch.int32, device="cuda")
    allowed[0, -1] = 0x7FFFFFFF  # all but the last class
    ids = torch.tensor([C - 1, C - 2, 0], dtype=torch.int32, device="cuda")
    ks.class_logits_adjust(z, bias=(ids, torch.full((3,), 4.0, device="cuda"), torch.tensor([0, 0, 0, 3], device="cuda")),
                           allowed=allowed, mask_row=torch.tensor([-1, -1, 0], dtype=torch.int32, device="cuda"))
    assert z[2, -1] == -INF and z[2, 0] == 4
    near(z[2:, -2:-1], want[2:, -2:-1] + 4.0, size[2:, -2:-1] + 100, torch.bfloat16)


# ---------------------------------------------------------------------------------------------------- penalties, biases, masks
def plain_adjust(z, a, c0, C):
    """-> adjusted logits, the magnitudes of the roundings, and which logits are computed anew."""
    z = z.astype(np.float64)
    size, new = np.zeros(z.shape), np.zeros(z.shape, dtype=bool)
    for b in range(len(z)):
        seen, said, bias = set(), {}, {}
        if a.get("seen"):
            ids, off = a["seen"]
            prompt = a["n_prompt"][b] if a.get("n_prompt") is not None else 0
            for e, c in enumerate(ids[off[b]:off[b + 1]]):
                if c >= 0 and 0 <= c - c0 < C:
                    seen.add(c - c0)
                    if e >= prompt:
                        said[c - c0] = said.get(c - c0, 0) + 1
        if a.get("bias"):
            ids, val, off = a["bias"]
            for c, v in zip(ids[off[b]:off[b + 1]], val[off[b]:off[b + 1]]):
                if c >= 0 and 0 <= c - c0 < C:
                    bias[c - c0] = float(v)
        for c in seen | set(bias):
            v, s, new[b, c] = z[b, c], 0.0, True
            if c in seen:
                r = float(a["repetition"][b]) if a.get("repetition") is not None else 1.0
                v = v / r if v > 0 else v * r
                v = v if abs(v) < 2.0 ** 128 else np.sign(v) * INF  # fp32 ends there
                s += abs(v)
                if said.get(c):
                    f = float(a["frequency"][b]) * said[c] if a.get("frequency") is not None else 0.0
                    p = float(a["presence"][b]) if a.get("presence") is not None else 0.0
                    v -= f + p
                    s += abs(f) + abs(f + p) + abs(v)
            if c in bias:
                v += bias[c]
                s += abs(v)
            z[b, c], size[b, c] = v, s
        m = -1
        if a.get("allowed") is not None:
            m = a["mask_row"][b] if a.get("mask_row") is not None else b
        if m >= 0:
            bits = np.unpackbits(a["allowed"][m].view(np.uint8), bitorder="little")[:C].astype(bool)
            z[b, ~bits], new[b, ~bits], size[b, ~bits] = -INF, True, 0.0
    return z, size, new


def lists(r, B, most, Cg, repeat=True):
    n = r.integers(0, most + 1, B)
    n[0] = most
    if B > 2:
        n[2] = 0
    off = np.zeros(B + 1, dtype=np.int64)
    off[1:] = n.cumsum()
    ids = (r.random(off[-1]) ** (4 if repeat else 1) * Cg).astype(np.int32) * 7 % Cg
    ids[r.random(off[-1]) < 0.05] = -1
    return ids.astype(np.int32), off


def adjust_case(r, B, C, Cg, seen, biases, masks):
    a = {}
    if seen:
        a["seen"] = lists(r, B, seen, Cg)
        a["n_prompt"] = r.integers(-1, seen + 2, B).astype(np.int32)
        a["repetition"] = r.uniform(0.5, 2.0, B).astype(np.float32)
        a["presence"] = r.uniform(-1, 1, B).astype(np.float32)
        a["frequency"] = r.uniform(-1, 1, B).astype(np.float32)
    if biases:
        ids, off = lists(r, B, biases, Cg)
        a["bias"] = (ids, (5 * r.standard_normal(len(ids))).astype(np.float32), off)
    if masks:
        words = (C + 31) // 32 + 2
        bits = r.random((max(1, B // 2), words * 32)) < r.choice([0.02, 0.5, 0.95], (max(1, B // 2), 1))
        bits[:, :200] = r.random(1) < 0.5
        bits[0] &= B == 1  # a mask that allows nothing
        a["allowed"] = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
        a["mask_row"] = r.integers(-1, len(bits), B).astype(np.int32)
        if B > 1:
            a["mask_row"][-1] = 0
    return a


def to_gpu(a):
    put = lambda v: tuple(put(x) for x in v) if isinstance(v, tuple) else torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    return {k: put(v) for k, v in a.items()}


def check_adjust(ks, r, B, C, c0, Cg, a, dtype, in_place, ld, shift=0, extreme=True, **known):
    whole = torch.from_numpy((4 * r.standard_normal(B * ld + shift)).astype(np.float32)).cuda().to(dtype)
    z = whole[shift:].view(B, ld)[:, :C]
    if extreme and C > 50:
        z[:, 3], z[:, 11], z[:, 13], z[0, 40] = INF, -INF, float("nan"), torch.finfo(dtype).min
    want, size, new = plain_adjust(z.float().cpu().numpy(), a, c0, C)
    before = whole.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = dict(c0=c0, Cg=Cg, dev_status=status, **to_gpu(a), **known)
    if in_place:
        got = ks.class_logits_adjust(z, **args)
        assert got is z
        rest = torch.ones_like(whole, dtype=torch.bool)
        rest[shift:].view(B, ld)[:, :C] = False
        assert torch.equal(whole[rest], before[rest])
    else:
        other = torch.full((B, ld + 8), 77.0, dtype=dtype, device="cuda")
        got = ks.class_logits_adjust(z, out=other[:, :C], **args)
        assert (other[:, C:] == 77).all()
        ints = torch.int32 if dtype == torch.float32 else torch.int16
        assert torch.equal(whole.view(ints), before.view(ints))
    assert int(status) == 0
    near(got, want, size, dtype)
    old = torch.from_numpy(~new).cuda()
    ints = torch.int32 if dtype == torch.float32 else torch.int16
    assert torch.equal(got.contiguous().view(ints)[old], before[shift:].view(B, ld)[:, :C].contiguous().view(ints)[old])
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("B,C,nodes,seen,biases,masks,ld", [
    (1, 1, 1, 1, 1, True, 1), (1, 10_000, 1, 300, 20, True, 10_000), (5, 1_000, 1, 40, 0, False, 1_000), (4, 999, 3, 0, 30, True, 1_003),
    (3, 8_193, 2, 500, 3, False, 8_200), (7, 4_133, 1, 0, 0, True, 4_136), (9, 20_001, 4, 3_000, 700, True, 20_001), (2, 100, 1, 9_000, 0, True, 104),
    (3, 40_000, 1, 20_000, 100, True, 40_064), (33, 555, 1, 60, 60, True, 560), (70, 250_001, 1, 100, 20, True, 250_008),
    (2, 70_000, 1, 50_000, 5_000, True, 70_001), (17, 9_001, 1, 5_000, 0, True, 9_008), (20, 12_000, 2, 7_000, 1_100, False, 12_001),
    (16, 3_001, 1, 4_000, 97, True, 3_002), (300, 60_000, 1, 5, 2, True, 60_000), (256, 24_576, 1, 900, 100, True, 24_576),
    (3, 24_577, 1, 900, 100, True, 24_584), (257, 1_000, 2, 2_000, 10, True, 1_000), (2, 6_143, 1, 3_000, 90, False, 6_143), (4, 49_152, 1, 1_000, 24, True, 49_160)])
def test_adjust(ks, B, C, nodes, seen, biases, masks, ld, in_place, dtype):
    r = rng_of(B, C, seen, biases)
    Cg, c0 = C * nodes, C * (nodes // 2)
    check_adjust(ks, r, B, C, c0, Cg, adjust_case(r, B, C, Cg, seen, biases, masks), dtype, in_place, ld)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ld,shift", [(1_001, 0), (1_008, 1), (1_016, 3), (1_002, 8)])
def test_adjust_of_rows_that_lie_apart(ks, dtype, ld, shift):
    r = rng_of(ld, shift)
    for in_place in (True, False):
        check_adjust(ks, r, 6, 1_000, 1_000, 3_000, adjust_case(r, 6, 1_000, 3_000, 50, 9, True), dtype, in_place, ld, shift)


@pytest.mark.parametrize("seen,biases", [(40, 10), (1_500, 200), (9_000, 900)])
def test_adjust_one_kind_at_a_time(ks, seen, biases):
    """Each penalty alone, lists without a prompt, and the lists' lengths given as they are."""
    r = rng_of(seen, biases)
    full = adjust_case(r, 4, 30_000, 30_000, seen, biases, True)
    for keep in (["seen", "repetition"], ["seen", "presence"], ["seen", "frequency", "n_prompt"], ["seen"], ["bias"], ["seen", "repetition", "bias"]):
        a = {k: full[k] for k in keep}
        check_adjust(ks, r, 4, 30_000, 0, 30_000, a, torch.float32, True, 30_000, seen_max=seen, bias_max=biases)


def test_adjust_lists_far_shorter_than_the_array(ks):
    """Many requests without word of their longest list: what the array holds is all that is known."""
    r = rng_of(5)
    for B, most in ((60, 400), (300, 90), (7, 6_000)):
        check_adjust(ks, r, B, 5_001, 0, 5_001, adjust_case(r, B, 5_001, 5_001, most, 9, True), torch.float32, True, 5_001)


def test_adjust_the_largest_batch(ks):
    """2^31 - 1 rows of one class: the row behind the last launch's rows is no 32-bit number."""
    B = 2 ** 31 - 1
    z, row = torch.zeros((B, 1), dtype=torch.bfloat16, device="cuda"), torch.full((B,), -1, dtype=torch.int32, device="cuda")
    at = [0, 1, 2 ** 21 - 1, 2 ** 21, B - 2 ** 21, B - 2, B - 1]
    row[at] = 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ks.class_logits_adjust(z, allowed=torch.zeros((1, 1), dtype=torch.int32, device="cuda"), mask_row=row, dev_status=status)
    assert int(status) == 0 and z.flatten()[at].isneginf().all()
    z.view(-1)[at] = 0
    assert not z.any()


def test_adjust_one_row_in_place_by_another_view(ks):
    z = torch.randn((1, 64), generator=torch.Generator().manual_seed(2)).cuda()
    want = z.clone()
    want[0, 5] = -INF
    allowed = torch.tensor([[~(1 << 5), -1]], dtype=torch.int32, device="cuda")
    ks.class_logits_adjust(z, out=z.as_strided((1, 64), (100, 1)), allowed=allowed)
    assert torch.equal(z, want)


def test_adjust_the_same_class_again_and_again(ks):
    """One class all along a list, once in the prompt and then behind it; of a class named twice among the biases the last one counts."""
    for n in (5, 3_000, 20_000):
        ids = np.full(n, 17, dtype=np.int32)
        a = {"seen": (ids, np.array([0, n], dtype=np.int64)), "n_prompt": np.array([2], dtype=np.int32), "frequency": np.array([0.25], dtype=np.float32),
             "repetition": np.array([1.5], dtype=np.float32),
             "bias": (ids, np.arange(n, dtype=np.float32), np.array([0, n], dtype=np.int64))}
        check_adjust(ks, rng_of(n), 1, 100, 0, 100, a, torch.float32, True, 100, extreme=False)


def test_adjust_ids_that_share_their_low_bits(ks):
    """Ids a power of two apart, as many as the lists may hold in one way of counting them."""
    C = 1 << 20
    for step in (1, 256, 4_096, 65_536):
        n = min(4_000, C // step)
        ids = (np.arange(n, dtype=np.int64) * step).astype(np.int32)
        a = {"seen": (ids, np.array([0, n], dtype=np.int64)), "presence": np.array([2.0], dtype=np.float32)}
        check_adjust(ks, rng_of(step), 1, C, 0, C, a, torch.float32, True, C)


@pytest.mark.parametrize("B,n,twice", [(1, 9_000, False), (40, 5_000, True)])
def test_adjust_classes_that_fall_into_one_part(ks, B, n, twice):
    """Lists of which all classes are neighbours once their keys are spread (by the odd factor that divides long lists among
    workgroups): one workgroup gets them all, several times what its table takes."""
    C = 1 << 20
    keys = (np.arange(1, C + 1, dtype=np.uint64) * 0x9E3779B1 % 2 ** 32).argsort()[:n].astype(np.int32)
    ids = np.concatenate([keys, keys[::-1]]) if twice else keys
    off = np.zeros(B + 1, dtype=np.int64)
    off[1:] = len(ids)  # the first request's list; the others have none
    a = {"seen": (ids, off), "presence": np.full(B, 2.0, dtype=np.float32), "frequency": np.full(B, 0.5, dtype=np.float32),
         "repetition": np.full(B, 1.5, dtype=np.float32)}
    check_adjust(ks, rng_of(B, n), B, C, 0, C, a, torch.bfloat16, True, C)


def test_adjust_reports_what_it_cannot_use(ks):
    z0 = torch.randn((3, 64), generator=torch.Generator().manual_seed(1)).cuda()
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    o = lambda *v: torch.tensor(v, dtype=torch.int64, device="cuda")  # noqa: E731
    f = lambda *v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    full, two = torch.full((2, 2), -1, dtype=torch.int32, device="cuda"), f(2.0, 2.0, 2.0)
    for args, bit in ((dict(seen=(i(3, 64, 5), o(0, 1, 2, 3)), presence=two), ks.KS_DEV_BAD_LABEL),
                      (dict(bias=(i(3, 70, 5), two, o(0, 1, 2, 3))), ks.KS_DEV_BAD_INDEX),
                      (dict(seen=(i(3, 4, 5), o(0, 1, 2, 4)), presence=two), ks.KS_DEV_BAD_COUNT),
                      (dict(seen=(i(3, 4, 5), o(0, 2, 1, 3)), presence=two), ks.KS_DEV_BAD_COUNT),
                      (dict(seen=(i(3, 4, 5), o(-1, 1, 2, 3)), presence=two), ks.KS_DEV_BAD_COUNT),
                      (dict(seen=(i(3, 4, 5), o(0, 0, 0, 3)), presence=two, seen_max=2), ks.KS_DEV_BAD_COUNT),
                      (dict(bias=(i(3, 4, 5), two, o(0, 1 << 40, 2, 3))), ks.KS_DEV_BAD_COUNT),
                      (dict(allowed=full, mask_row=i(0, 2, -7)), ks.KS_DEV_BAD_INDEX)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        for out in (z0.clone(), None):
            z = z0.clone()
            ks.class_logits_adjust(z, out=out, dev_status=status, **args)
            torch.cuda.synchronize()
            assert int(status) == bit, (args, int(status))


@pytest.mark.parametrize("B,C,dtype", [(3, 64, torch.float32), (3, 6_000_000, torch.bfloat16), (3, 100_001, torch.float32), (300, 1_000, torch.bfloat16)])
def test_adjust_reports_lists_where_none_may_hold_anything(ks, B, C, dtype):
    z0 = torch.randn((B, C), generator=torch.Generator("cuda").manual_seed(4), device="cuda").to(dtype)
    off = torch.zeros(B + 1, dtype=torch.int64, device="cuda")
    full = off.clone()
    full[2:] = 5  # the second request's list
    ids, words = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.full((1, (C + 31) // 32), -2, dtype=torch.int32, device="cuda")
    none, masked = ids[:0], z0.clone()
    masked[:, ::32] = -INF
    masks = dict(allowed=words, mask_row=torch.zeros(B, dtype=torch.int32, device="cuda"))
    for lists in (lambda o: dict(seen=(none, o)), lambda o: dict(bias=(none, none.float(), o)), lambda o: dict(seen=(ids, o), seen_max=0),
                  lambda o: dict(bias=(ids, ids.float(), o), bias_max=0), lambda o: dict(seen=(none, off), bias=(none, none.float(), o))):
        for args, want in (({}, z0), (masks, masked)):
            for offsets, bit in ((off, 0), (full, ks.KS_DEV_BAD_COUNT)):
                for out in (None, torch.empty_like(z0)):
                    z, status = z0.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
                    got = ks.class_logits_adjust(z, out=out, dev_status=status, **lists(offsets), **args)
                    assert torch.equal(got, want) and int(status) == bit
                    assert torch.equal(ks.class_logits_adjust(z0.clone(), **lists(offsets), **args), want)


def test_binding_refuses(ks):
    V = torch.ones((4, 8), device="cuda")
    with pytest.raises(TypeError):
        ks.class_quantize_rows(V.half())
    with pytest.raises(TypeError):
        ks.class_quantize_rows(V.t())
    with pytest.raises(ValueError):
        ks.class_quantize_rows(V, codes=torch.empty(8, dtype=torch.int8, device="cuda"))
    with pytest.raises(ValueError):
        ks.class_quantize_rows(V.to(torch.int8), normalize=True)
    x, xs = ks.class_quantize_rows(V)
    w, ws = ks.class_quantize_rows(V, classes=True)
    for bad in (dict(w_codes=x), dict(bias=torch.ones(5, device="cuda")), dict(out=torch.empty((4, 5), device="cuda")),
                dict(x_codes=x[:512]), dict(x_codes=x[:1000]), dict(x_scale=torch.ones(33, device="cuda")), dict(x_codes=x[:0]),
                dict(x_codes=x[:512], w_codes=w[:1024]), dict(w_codes=ks.class_quantize_rows(torch.ones((4, 40), device="cuda"), classes=True)[0])):
        with pytest.raises(ValueError):
            ks.class_logits_int8(**{**dict(x_codes=x, x_scale=xs, w_codes=w, w_scale=ws, scale=1.0), **bad})
    with pytest.raises(TypeError):
        ks.class_logits_int8(x, xs, w, ws, 1.0, dtype=torch.float16)
    z = torch.zeros((4, 40), device="cuda")
    m = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    for bad in (dict(out=torch.zeros((4, 41), device="cuda")), dict(repetition=torch.ones(3, device="cuda")), dict(allowed=m[:3]), dict(allowed=m[:, :1]),
                dict(mask_row=torch.zeros(4, dtype=torch.int32, device="cuda")),
                dict(bias=(torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(5, dtype=torch.int64, device="cuda")))):
        with pytest.raises(ValueError):
            ks.class_logits_adjust(z, **bad)
    with pytest.raises(ks.KsError):
        ks.class_logits_adjust(z, c0=1, Cg=40, allowed=m)


def test_binding_refuses_sizes_beyond_a_c_int(ks):
    """What is passed for a C int is taken by its low 32 bits: such sizes are refused before.  Nothing here is ever read."""
    new = lambda *n, dtype=torch.int8: torch.empty(n, dtype=dtype, device="cuda")  # noqa: E731
    for D in (65_537, 2 ** 32 + 8):
        with pytest.raises(ks.KsError) as e:
            ks.class_quantize_rows(new(1, D))
        assert e.value.code == ks.KS_UNSUPPORTED
    B = 4_194_241
    with pytest.raises(ks.KsError) as e:
        ks.class_logits_int8(new((B + 31) // 32 * 1024), new(B, dtype=torch.float32), new(64 * 32), new(1, dtype=torch.float32), 1.0)
    assert e.value.code == ks.KS_UNSUPPORTED
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        ks.class_logits_adjust(new(2 ** 32 + 1, 1, dtype=torch.bfloat16), allowed=new(1, 1, dtype=torch.int32), dev_status=status)
    z, none = torch.ones((2, 40), device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    few, many = torch.zeros(9, dtype=torch.int32, device="cuda"), new(2 ** 32 + 5, dtype=torch.int32)
    for bad in (dict(seen=(few, none), seen_max=5 - 2 ** 32), dict(seen=(many, none)), dict(seen=(many, none), seen_max=2 ** 32 + 2),
                dict(bias=(few, few.float(), none), bias_max=5 - 2 ** 32), dict(seen=(few, none), c0=2 ** 64), dict(seen=(few, none), Cg=2 ** 64 + 40),
                dict(seen=(few, none), c0=-2 ** 64)):
        with pytest.raises(ks.KsError) as e:
            ks.class_logits_adjust(z, presence=torch.ones(2, device="cuda"), dev_status=status, **bad)
        assert e.value.code == ks.KS_INVALID_ARG
    ks.class_logits_adjust(z, seen=(many, none), seen_max=5, presence=torch.ones(2, device="cuda"), dev_status=status)  # short lists of a large array
    assert int(status) == 0 and (z == 1).all()


# ---------------------------------------------------------------------------------------------------- together
def answer(ks, X, W8, ws, bias, adjust, stream=None, **args):
    x, xs = ks.class_quantize_rows(X, stream=stream)
    z = ks.class_logits_int8(x, xs, W8, ws, 30.0, bias=bias, stream=stream, **args)
    return ks.class_logits_adjust(z, stream=stream, **adjust)


@pytest.mark.parametrize("B,C,D,dtype", [(1, 5_000, 128, torch.float32), (40, 3_001, 96, torch.float32), (150, 2_000, 320, torch.bfloat16)])
def test_answer_after_training(ks, B, C, D, dtype):
    """Weights that a layer keeps un-normalised in fp32, features in bf16, requests: the whole of a serving step."""
    r = rng_of(B, C, D)
    W = torch.from_numpy((r.standard_normal((C, D)) * np.exp(r.uniform(-1, 1, (C, 1)))).astype(np.float32)).cuda()
    X = torch.from_numpy(r.standard_normal((B, D)).astype(np.float32)).cuda().to(torch.bfloat16)
    W8, ws = ks.class_quantize_rows(W, classes=True, normalize=True)
    bias = r.standard_normal(C).astype(np.float32)
    a = adjust_case(r, B, C, C, 60, 12, True)
    raw = answer(ks, X, W8, ws, torch.from_numpy(bias).cuda(), {}, dtype=dtype)
    got = answer(ks, X, W8, ws, torch.from_numpy(bias).cuda(), to_gpu(a), dtype=dtype)
    q, s = plain_codes(X.float().cpu().numpy())
    w, t = plain_codes(W.cpu().numpy(), True)
    z, size = plain_logits(q, s, w, t, 30.0, bias)
    near(raw, z, size + 2 * np.abs(z - bias[None, :]), dtype)  # the two scales are rounded to fp32 as well
    want, size, _ = plain_adjust(raw.float().cpu().numpy(), a, 0, C)
    near(got, want, size, dtype)
    # how far codes are from the weights themselves: half a code of each side, and |x| <= 127 codes
    cos = X.double().cpu().numpy() @ (W.double() / W.double().norm(dim=1, keepdim=True)).cpu().numpy().T
    x_abs = np.abs(X.double().cpu().numpy()).sum(1)
    w_abs = (W.double().abs().sum(1) / W.double().norm(dim=1)).cpu().numpy()
    off = 0.5 * s[:, None] * w_abs[None, :] + 0.5 * t[None, :] * x_abs[:, None] + 0.25 * D * s[:, None] * t[None, :]
    assert (np.abs(z - bias[None, :] - 30.0 * cos) <= 30.0 * off * (1 + 1e-9) + 1e-9).all()


def test_answer_on_another_stream(ks):
    r = rng_of(77)
    W = torch.from_numpy(r.standard_normal((3_000, 128)).astype(np.float32)).cuda()
    X = torch.from_numpy(r.standard_normal((20, 128)).astype(np.float32)).cuda()
    a = to_gpu(adjust_case(r, 20, 3_000, 3_000, 60, 12, True))
    W8, ws = ks.class_quantize_rows(W, classes=True)
    want = answer(ks, X, W8, ws, None, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = answer(ks, X, W8, ws, None, a, stream=side)
    with torch.cuda.stream(side):
        also = answer(ks, X, W8, ws, None, a)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(also, want)


def test_answer_captured_and_replayed(ks):
    r = rng_of(78)
    B, C, D = 24, 6_000, 96
    W8, ws = ks.class_quantize_rows(torch.from_numpy(r.standard_normal((C, D)).astype(np.float32)).cuda(), classes=True)
    batches = [torch.from_numpy(r.standard_normal((B, D)).astype(np.float32)).cuda() for _ in range(4)]
    a = to_gpu(adjust_case(r, B, C, C, 60, 12, True))
    a["dev_status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = [answer(ks, X, W8, ws, None, a).clone() for X in batches]
    X, copy = batches[0].clone(), torch.empty((B, C), device="cuda")
    answer(ks, X, W8, ws, None, a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x, xs = ks.class_quantize_rows(X)
        z = ks.class_logits_int8(x, xs, W8, ws, 30.0)
        ks.class_logits_adjust(z, out=copy, **a)
        got = ks.class_logits_adjust(z, **a)
    for k in (1, 2, 0, 3, 3):
        X.copy_(batches[k])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want[k]) and torch.equal(copy, want[k])
        assert torch.equal(answer(ks, batches[k], W8, ws, None, a), want[k])


def test_two_calls_at_once(ks):
    """No memory is shared between calls: two streams at the same time."""
    r = rng_of(79)
    W8, ws = ks.class_quantize_rows(torch.from_numpy(r.standard_normal((9_000, 256)).astype(np.float32)).cuda(), classes=True)
    jobs = []
    for k in range(2):
        X = torch.from_numpy(r.standard_normal((90, 256)).astype(np.float32)).cuda()
        jobs.append((X, to_gpu(adjust_case(r, 90, 9_000, 9_000, 200, 40, True)), torch.cuda.Stream()))
    want = [answer(ks, X, W8, ws, None, a) for X, a, _ in jobs]
    torch.cuda.synchronize()
    got = [[answer(ks, X, W8, ws, None, a, stream=st) for X, a, st in jobs] for _ in range(3)]
    torch.cuda.synchronize()
    for pair in got:
        assert all(torch.equal(g, w) for g, w in zip(pair, want))


@pytest.mark.parametrize("B,C,D,seen,dtype", [(300, 66_000, 128, 5_000, torch.bfloat16), (300, 33_000, 1_200, 9_000, torch.float32),
                                              (256, 20_000, 512, 700, torch.bfloat16)])
def test_large_answers_captured_and_replayed(ks, B, C, D, seen, dtype):
    """The kernels of large batches and long lists, with the weights' codes made inside the graph; eager calls between the replays."""
    gen = torch.Generator("cuda").manual_seed(B + C + D)
    weights = [torch.randn((C, D), generator=gen, device="cuda") for _ in range(2)]
    batches = [torch.randn((B, D), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    a = to_gpu(adjust_case(rng_of(B, C), B, C, C, seen, 30, True))
    a.update(seen_max=seen, bias_max=30, dev_status=torch.zeros(1, dtype=torch.int32, device="cuda"))

    def whole(W, X, out, copy):
        W8, ws = ks.class_quantize_rows(W, classes=True, normalize=True)
        x, xs = ks.class_quantize_rows(X)
        z = ks.class_logits_int8(x, xs, W8, ws, 30.0, out=out)
        ks.class_logits_adjust(z, out=copy, **a)
        return ks.class_logits_adjust(z, **a)

    new = lambda: torch.empty((B, (C + 63) // 64 * 64), dtype=dtype, device="cuda")[:, :C]  # noqa: E731
    W, X, out, copy = weights[0].clone(), batches[0].clone(), new(), new()
    want = [whole(weights[k], batches[k], new(), new()).clone() for k in range(2)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        whole(W, X, out, copy)
    for k in (1, 0, 1):
        W.copy_(weights[k])
        X.copy_(batches[k])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[k]) and torch.equal(copy, want[k]) and int(a["dev_status"]) == 0
        assert torch.equal(whole(weights[k], batches[k], new(), new()), want[k])
