"""GPU parity of include/class_sample.h against a plain implementation in 64 bits and whole numbers, written from the definition there."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U32, INF, NAN = 2.0 ** -24, float("inf"), float("nan")
LAST = 1.0 - 2.0 ** -24  # the largest u below 1


@pytest.fixture(scope="module")
def ks():
    import paper_2102_06025_amd as ks
    ks.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return ks


@pytest.fixture(autouse=True)
def name_the_case(request):
    print(f"[sample] {request.node.name}", flush=True)


# ---------------------------------------------------------------------------------------------------- plain form
def draw(z, u, T=1.0, k=0, p=1.0, m=0.0):
    """One row, float64 -> id, log-probability, classes that are kept.  Weights as whole numbers; sums below 2^63."""
    C = len(z)
    bits = min(48, 62 - math.ceil(math.log2(C)))
    live = np.flatnonzero(z > -INF)
    if len(live) == 0:
        return -1, -INF, live
    order = live[np.argsort(-z[live], kind="stable")]
    if not T > 0:
        return int(order[0]), 0.0, order[:1]
    if 0 < k < C:
        order = order[:k]
    v, top = z[order], z[order[0]]
    with np.errstate(invalid="ignore", over="ignore"):
        log_w = np.where(v == top, 0.0, (v - top) / T)
    w = np.rint(np.exp(log_w) * 2.0 ** bits).astype(np.uint64)
    if p < 1.0:
        run = np.cumsum(w)
        n = 1 + int(np.searchsorted(run, np.uint64(max(math.ceil(max(p, 0.0) * float(run[-1])), 1)), side="left"))
        order, w, log_w = order[:n], w[:n], log_w[:n]
    if m > 0:
        keep = w >= min(m, 1.0) * 2.0 ** bits
        order, w, log_w = order[keep], w[keep], log_w[keep]
    by_id = np.argsort(order)
    order, w, log_w = order[by_id], w[by_id], log_w[by_id]
    run = np.cumsum(w)
    total = int(run[-1])
    target = min(int(min(max(u, 0.0), 2.0) * float(total)) if u == u else 0, total - 1)
    at = int(np.searchsorted(run, np.uint64(target), side="right"))
    return int(order[at]), float(log_w[at] - math.log(total) + bits * math.log(2.0)), order


def f32(x):
    return np.float64(np.float32(x))


def check(ks, logits, u, T=None, k=None, p=None, m=None, **more):
    B = logits.shape[0]

    def column(v, dtype=torch.float32):
        return None if v is None else torch.tensor(list(v) if np.ndim(v) else [v] * B, dtype=dtype, device="cuda")
    u_, T_, k_, p_, m_ = column(u), column(T), column(k, torch.int32), column(p), column(m)
    ids, lp = ks.class_sample(logits, u_, temperature=T_, top_k=k_, top_p=p_, min_p=m_, **more)
    z = logits.double().cpu().numpy()

    def at(c, b, none):
        return none if c is None else float(c[b])
    u_, T_, k_, p_, m_ = [None if c is None else c.cpu() for c in (u_, T_, k_, p_, m_)]
    for b in range(B):
        want, want_lp, _ = draw(np.where(np.isnan(z[b]), -INF, z[b]), at(u_, b, None), at(T_, b, 1.0), int(at(k_, b, 0)), at(p_, b, 1.0), at(m_, b, 0.0))
        assert int(ids[b]) == want, (b, int(ids[b]), want)
        got = float(lp[b])
        # the 64-bit value, off by less than 1e-11, rounded once
        assert got == want_lp or abs(got - want_lp) <= 1.01 * U32 * abs(want_lp) + 1e-11, (b, got, want_lp)
    return ids, lp


def logits_of(gen, B, C, dtype, spread=1.3, masked=0.0, ld=None):
    store = torch.empty((B, ld or C), dtype=dtype, device="cuda")[:, :C]
    store.copy_(spread * torch.randn((B, C), generator=gen, device="cuda"))
    n = min(40, C)
    at = torch.rand((B, C), generator=gen, device="cuda").argsort(1)[:, :n] if C < 20_000 else torch.randint(0, C, (B, n), generator=gen, device="cuda")
    store.scatter_(1, at, (12 * torch.rand((B, n), generator=gen, device="cuda") ** 2).to(dtype))
    if masked:
        store.masked_fill_(torch.rand((B, C), generator=gen, device="cuda") < masked, -INF)
    return store


RULES = [dict(), dict(T=0.7), dict(k=1), dict(k=40), dict(p=0.9), dict(m=0.05), dict(T=1.3, k=300, p=0.8), dict(T=0.5, p=0.99, m=0.001), dict(k=100, m=0.02),
         dict(T=2.0, k=200, p=0.95, m=0.01), dict(T=0.0), dict(p=0.2), dict(T=3.0, p=0.999), dict(T=1.5, m=1e-6), dict(k=5_000, T=4.0), dict(k=1 << 30)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C", [1, 2, 7, 511, 512, 513, 2_000, 10_000, 32_768, 100_003])
@pytest.mark.parametrize("masked", [0.0, 0.6])
def test_rules(ks, C, dtype, masked):
    gen = torch.Generator("cuda").manual_seed(C)
    for i, rule in enumerate(RULES):
        B = 6
        z = logits_of(gen, B, C, dtype, spread=(0.3, 1.3, 3.0)[i % 3], masked=masked)
        print(rule, flush=True)
        check(ks, z, [0.0, LAST] + torch.rand(B - 2, generator=gen, device="cuda").tolist(), **rule)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_row_its_own_rule(ks, dtype):
    gen = torch.Generator("cuda").manual_seed(5)
    B, C = 64, 30_011
    z = logits_of(gen, B, C, dtype, masked=0.3, ld=30_024)
    r = np.random.default_rng(5)
    T, k = r.choice([0.0, 0.3, 1.0, 2.5], B), r.choice([0, -3, 1, 50, 3_000], B)
    p, m = r.choice([1.0, 0.5, 0.97, 0.0, 1.5], B), r.choice([0.0, 0.1, 1.0, 7.0, -1.0], B)
    u = r.random(B).astype(np.float32)
    ids, lp = check(ks, z, u, T, k, p, m)
    # a row's result does not depend on its neighbours or its place
    for b in (0, 17, 63):
        one, one_lp = ks.class_sample(z[b:b + 1], torch.tensor(u[b:b + 1], device="cuda"), *[torch.tensor(v[b:b + 1], dtype=d, device="cuda") for v, d in (
            (T, torch.float32), (k, torch.int32), (p, torch.float32), (m, torch.float32))])
        assert torch.equal(one, ids[b:b + 1]) and torch.equal(one_lp, lp[b:b + 1])


@pytest.mark.parametrize("C", [600, 9_000, 200_000])
def test_equal_logits_go_by_id(ks, C):
    """A bin of equal logits that LDS does not hold is cut by ids; a cut between equal ones keeps the lowest."""
    for value in (0.0, -3.5, 1e30):
        z = torch.full((5, C), value, device="cuda")
        z[1, ::3] = value - 1.0 if value < 1e20 else 0.0
        z[2, 1::2] = -0.0 if value == 0.0 else value
        z[3, : C // 2] = -INF
        for rule in (dict(), dict(k=C // 3), dict(p=0.37), dict(k=C // 2, p=0.5), dict(m=1.0), dict(k=7), dict(p=1e-9), dict(T=0.0)):
            check(ks, z, [0.0, 0.5, 0.3, LAST, 0.99], **rule)


def test_few_values_with_many_classes_each(ks):
    gen = torch.Generator("cuda").manual_seed(9)
    z = torch.randint(-2, 3, (4, 150_000), generator=gen, device="cuda").to(torch.bfloat16)
    z[1] *= 0.01
    z[2, 77_777] = 30.0
    for rule in (dict(k=70_000), dict(p=0.6), dict(k=40_000, p=0.7), dict(p=0.999), dict(m=0.3), dict(T=0.05, k=100_000)):
        check(ks, z, [0.1, 0.9, 0.6, 0.4], **rule)


def test_infinities_nan_and_rows_without_a_class(ks):
    z = torch.zeros((9, 1_300), device="cuda")
    z[0] = -INF
    z[1] = NAN
    z[2, 5], z[2, 900] = INF, INF
    z[3] = INF
    z[4, 3], z[4, 7] = NAN, 40.0
    z[5] = -INF
    z[5, 1_299] = -2e38
    z[6] = 3e38
    z[6, 4] = -3e38
    z[7, ::2], z[7, 1::2] = NAN, -INF
    z[8] = torch.linspace(-3e38, 3e38, 1_300)
    u = [0.5, 0.5, 0.6, 0.3, 0.2, 0.9, 0.7, 0.1, 0.5]
    for rule in (dict(), dict(k=3), dict(p=0.5), dict(m=0.5), dict(k=10, p=0.9, m=0.1), dict(T=0.0), dict(T=1e-30), dict(T=1e38, p=0.3)):
        ids, lp = check(ks, z, u, **rule)
        assert ids[[0, 1, 7]].tolist() == [-1, -1, -1] and (lp[[0, 1, 7]] == -INF).all()
    # an infinite temperature weighs all classes the same, but for masked ones
    z[:, 100:] = -INF
    check(ks, z[4:7], u[4:7], T=INF)
    check(ks, z[4:7], u[4:7], T=INF, p=0.5)


def test_settings_at_and_beyond_their_ends(ks):
    gen = torch.Generator("cuda").manual_seed(3)
    z = logits_of(gen, 8, 4_000, torch.float32)
    check(ks, z, [0.0, 1.0, 2.0, -1.0, NAN, LAST, 1e-30, INF])
    check(ks, z, 0.999, k=50, p=[0.0, -1.0, 1e-30, 1.0, NAN, 1 - 2 ** -24, INF, -INF])
    check(ks, z, 0.5, m=[0.0, -1.0, 1e-38, 1.0, NAN, 2.0, INF, 1e-44])
    check(ks, z, 0.5, T=[0.0, -1.0, NAN, 1e-38, 1e38, -INF, 1e-3, 300.0])
    check(ks, z, 0.9, T=1e-38, k=3, p=0.5, m=0.5)
    check(ks, z, LAST, k=[0, -5, -2 ** 31, 2 ** 31 - 1, 4_000, 3_999, 4_001, 1])


def test_more_classes_than_short_segments_hold(ks):
    """Segments of 1,024 classes; u at the ends finds the first and the last class that is kept."""
    gen = torch.Generator("cuda").manual_seed(8)
    C = 2_500_000
    z = logits_of(gen, 2, C, torch.bfloat16)
    for rule in (dict(), dict(k=1_000), dict(p=0.9), dict(T=0.6, p=0.5, m=0.01), dict(T=0.0)):
        check(ks, z, [0.31, 0.77], **rule)
    check(ks, z[:, 1:], [0.0, LAST], T=5.0, p=0.999)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides(ks, dtype):
    gen = torch.Generator("cuda").manual_seed(4)
    store = logits_of(gen, 5, 3_010, dtype)
    for shift, C in ((0, 3_010), (1, 3_001), (3, 2_999), (8, 3_000)):
        check(ks, store[:, shift:shift + C], 0.6, k=60, p=0.9)
        check(ks, store[::2, shift:shift + C], 0.6)


def test_offsets_beyond_32_bits(ks):
    C = 3_000
    store = torch.empty((2, (1 << 31) + 64), dtype=torch.bfloat16, device="cuda")
    z = store[:, :C]
    z.copy_(torch.randn((2, C), device="cuda", generator=torch.Generator("cuda").manual_seed(1)))
    check(ks, z, [0.4, 0.8], p=0.9)


def test_shares_of_the_random_numbers(ks):
    """Over evenly spaced u every class is drawn as often as its share says, to within one."""
    N = 4_096
    z = torch.tensor([1.0, -INF, 0.5, 3.0, 2.0, 2.0], device="cuda").expand(N, 6).contiguous()
    u = (torch.arange(N, device="cuda") + 0.5) / N
    ids, lp = ks.class_sample(z, u)
    share = torch.softmax(z[0].double(), 0)
    n = torch.bincount(ids.long(), minlength=6).double()
    assert ((n - share * N).abs() <= 1).all()
    assert torch.allclose(lp.double(), share.log()[ids.long()], atol=1e-6)


def test_streams_graphs_and_shared_workspaces(ks):
    gen = torch.Generator("cuda").manual_seed(6)
    B, C = 12, 20_000
    ws = torch.empty(ks.class_sample_workspace(C, B), dtype=torch.uint8, device="cuda")
    z, u = logits_of(gen, B, C, torch.bfloat16), torch.rand(B, generator=gen, device="cuda")
    k, p = torch.full((B,), 50, dtype=torch.int32, device="cuda"), torch.full((B,), 0.9, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ids, lp = ks.class_sample(z, u, top_k=k, stream=side)
    side.synchronize()
    want = ks.class_sample(z, u, top_k=k)
    assert torch.equal(ids, want[0]) and torch.equal(lp, want[1])
    # two graphs that share a workspace, replayed in turn with eager calls between
    torch.cuda.synchronize()
    graphs, outs = [], []
    for rule in (dict(top_k=k), dict(top_p=p)):
        out = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ks.class_sample(z, u, ids=out[0], logprob=out[1], ws=ws, **rule)
        graphs.append(g)
        outs.append((out, rule))
    for _ in range(3):
        z.copy_(logits_of(gen, B, C, torch.bfloat16))
        u.copy_(torch.rand(B, generator=gen, device="cuda"))
        for g, (out, rule) in zip(graphs, outs):
            g.replay()
            want = ks.class_sample(z, u, **rule)
            torch.cuda.synchronize()
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_a_serving_step(ks):
    """Features in 4 bits, logits of all classes, what the requests change in them, a class for each."""
    gen = torch.Generator("cuda").manual_seed(7)
    B, C, D = 9, 5_003, 200
    W = torch.nn.functional.normalize(torch.randn((C, D), generator=gen, device="cuda"))
    X = torch.nn.functional.normalize(W[torch.randint(0, C, (B,), generator=gen, device="cuda")] + 0.05 * torch.randn((B, D), generator=gen, device="cuda"))
    z = ks.class_logits_mxfp4(ks.class_quantize_mxfp4(X), ks.class_quantize_mxfp4(W, classes=True), B, C, D, 30.0, dtype=torch.bfloat16)
    words = torch.randint(-2 ** 31, 2 ** 31 - 1, (B, (C + 31) // 32), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    words[3] = 0
    ks.class_logits_adjust(z, allowed=words)
    u = torch.rand(B, generator=gen, device="cuda")
    ids, _ = check(ks, z, u.tolist(), T=0.8, k=100, p=0.95)
    assert int(ids[3]) == -1
    for b in range(B):
        if b != 3:
            c = int(ids[b])
            assert int(words[b, c // 32]) >> (c % 32) & 1


def test_refusals_of_tensors(ks):
    z, u = torch.zeros((3, 10), device="cuda"), torch.zeros(3, device="cuda")
    with pytest.raises(ValueError):
        ks.class_sample(z, u[:2])
    with pytest.raises(TypeError):
        ks.class_sample(z, u.double())
    with pytest.raises(TypeError):
        ks.class_sample(z, u, top_k=u)
    with pytest.raises(TypeError):
        ks.class_sample(z.half(), u)
    with pytest.raises(ks.KsError) as e:
        ks.class_sample(z, u, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == ks.KS_WORKSPACE_TOO_SMALL


# ---------------------------------------------------------------------------------------------------- weights at the end of what is counted
def weightless(s, part, C, rest=-5.0):
    """A row whose first `part` classes weigh two fifths of 2^-s each, which is no whole 2^-s, one of the largest logit behind them."""
    z = torch.full((C,), rest, dtype=torch.float64)
    z[:part] = math.log(0.4) - s * math.log(2.0)
    z[part] = 0.0
    return z


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C,part", [(16, 8), (1_000, 16), (30_000, 800), (100_003, 32), (100_003, 32 * 7), (400_000, 1_024), (2_500_000, 3 * 1_024)])
def test_classes_without_a_weight_are_not_drawn(ks, C, part, dtype):
    """Parts of a row whose classes weigh nothing each, but together more than 2^-s: u = 0 and the like draw the first class with a weight."""
    s = min(48, 62 - math.ceil(math.log2(C)))
    z = torch.stack([weightless(s, part, C), weightless(s, part, C), weightless(s, part, C), weightless(s, part - 3, C)]).to(dtype).cuda()
    z[1, 2] = -INF
    z[2, part + 1:] = -200.0  # nothing with a weight behind the largest
    ids, _ = check(ks, z, 0.0)
    assert ids.tolist() == [part, part, part, part - 3]
    check(ks, z, LAST)
    check(ks, z, [1e-30, 2.0 ** -60, 0.5, 0.25])
    check(ks, z[2:3], LAST)  # the running weight ends at the largest


def test_a_part_that_weighs_less_than_the_sum_of_its_classes(ks):
    """One class of a part has the weight 1, seven none: a target between 1 and the part's rounded sum is met behind it."""
    C, s = 64, 48
    z = torch.full((3, C), -INF, dtype=torch.float64)
    z[:, :8] = math.log(0.4) - s * math.log(2.0)
    z[:, 3] = math.log(0.6) - s * math.log(2.0)
    z[:2, 40] = 0.0
    z[2, 20] = 0.0
    z[1, 30] = -0.5
    ids, _ = check(ks, z.float().cuda(), [2.0 ** -48, 2.0 ** -47, 2.0 ** -48])
    assert ids.tolist() == [40, 30, 20]
    assert check(ks, z.float().cuda(), 0.0)[0].tolist() == [3, 3, 3]


def test_the_least_weight_counts_with_and_without_rules(ks):
    """A logit whose weight is just above half of 2^-s, which is the weight 1: u = 0 draws it where it comes first."""
    for T, v in ((0.8333905935287476, -28.30545425415039), (3.8100030422210693, -129.40374755859375), (1.4537763595581055, -49.376365661621094),
                 (3.362499713897705, -114.20465087890625), (1.8140368461608887, -61.612327575683594), (1.421820878982544, -48.29102325439453)):
        for C in (8, 5_000):
            z = torch.full((1, C), -200.0, device="cuda")
            z[0, 1], z[0, 5], z[0, C - 1] = v, 0.0, -1.0
            for rule in (dict(), dict(k=3), dict(m=1e-30), dict(k=3, m=1e-30)):
                ids, _ = check(ks, z, 0.0, T=T, **rule)
                assert ids.item() == 1, (T, C, rule)


@pytest.mark.parametrize("C", [2, 40, 5_000, 40_000])
def test_logits_far_apart_at_large_and_at_small_temperatures(ks, C):
    """Differences beyond the largest 32-bit number weigh something at a large temperature, differences below the least normal one at a small one."""
    rules = (dict(), dict(p=0.99), dict(m=0.1), dict(m=0.2), dict(k=C - 1), dict(k=max(C // 2, 1), p=0.9), dict(p=0.6, m=0.01), dict(p=0.05))
    for T, scale in ((2e38, 2e38), (3e38, 1e38), (1e37, 3e38), (3e38, 3.4e38), (1e-38, 1e-38), (2e-45, 3e-45), (1e-42, 4e-42), (1.3e-37, 3e-37)):
        z = torch.linspace(1.0, -1.0, C, dtype=torch.float64).mul_(scale).float().repeat(6, 1)
        z[1] = z[1].flip(0)
        z[2, :: 3] = -INF
        z[2, 1] = scale
        for rule in rules:
            print(T, scale, rule, flush=True)
            check(ks, z.cuda(), [0.0, 0.3, 0.7, LAST, 0.9, 0.95], T=T, **rule)


# ---------------------------------------------------------------------------------------------------- rows that share what a call has
def test_more_rows_that_keep_much_than_places_for_their_candidates(ks):
    """Places for the classes around a border are there for 256 rows; rows beyond take another way, whichever they are, to the same class."""
    gen = torch.Generator("cuda").manual_seed(31)
    B, C = 320, 40_000
    z = (0.0625 * torch.randint(-160, 161, (B, C), generator=gen, device="cuda")).to(torch.bfloat16)  # 321 values, some 3,700 classes in a bin at T = 85
    z[5], z[77] = 1.5, -INF
    u = torch.rand(B, generator=gen, device="cuda").tolist()
    for rule in (dict(k=C // 2, T=85.0), dict(p=0.6, T=85.0)):
        ids, lp = check(ks, z, u, **rule)
        again = check_again(ks, z, u, **rule)
        assert torch.equal(ids, again[0]) and torch.equal(lp, again[1])
        for b in (0, 5, 200, B - 1):
            one, one_lp = check(ks, z[b:b + 1], u[b], **rule)
            assert torch.equal(one, ids[b:b + 1]) and torch.equal(one_lp, lp[b:b + 1])


def check_again(ks, z, u, T, k=0, p=1.0):
    B = z.shape[0]

    def column(v, dtype):
        return torch.full((B,), v, dtype=dtype, device="cuda")
    return ks.class_sample(z, torch.tensor(u, device="cuda"), temperature=column(T, torch.float32), top_k=column(k, torch.int32), top_p=column(p, torch.float32))


def test_more_rows_than_a_launch_takes(ks):
    gen = torch.Generator("cuda").manual_seed(32)
    B, C = 33_000, 24
    z = logits_of(gen, B, C, torch.float32)
    u = torch.rand(B, generator=gen, device="cuda").tolist()
    check(ks, z, u, T=1.5, k=9, p=0.9)
    # the rows of the second launch that keep more than LDS holds: the same as by themselves
    C = 6_000
    z = logits_of(gen, 8, C, torch.bfloat16, spread=0.3).repeat(4_200, 1)
    u = torch.rand(z.shape[0], generator=gen, device="cuda")
    ids, lp = ks.class_sample(z, u, top_p=torch.full((z.shape[0],), 0.97, device="cuda"))
    for first in (0, 32_760, 33_592):
        part = slice(first, first + 8)
        own = check(ks, z[part], u[part].tolist(), p=0.97)
        assert torch.equal(own[0], ids[part]) and torch.equal(own[1], lp[part])


def test_many_classes_of_few_logits_in_long_parts(ks):
    """Parts of 1,024 classes and bins of a million equal logits."""
    C = 2_500_000
    gen = torch.Generator("cuda").manual_seed(33)
    equal = torch.full((1, C), -0.75, dtype=torch.bfloat16, device="cuda")
    five = torch.randint(-2, 3, (1, C), generator=gen, device="cuda").to(torch.bfloat16)
    near = 0.01 * torch.randint(0, 3, (1, C), generator=gen, device="cuda").to(torch.float32)
    for z in (equal, five, near, five[:, 3:C - 2]):
        for rule in (dict(k=C // 3), dict(p=0.37), dict(k=C // 2, p=0.5), dict(m=0.3)):
            print(rule, flush=True)
            check(ks, z, 0.618, **rule)
    check(ks, torch.cat([equal, five]), [0.0, LAST], k=C // 3, p=0.9)


@pytest.mark.parametrize("C", [8, 5_000, 40_000])
def test_the_least_weights_and_min_p(ks, C):
    """Whole weights are compared with m: one of 0.6 of 2^-s is 1 and stays for m = 0.7 of 2^-s, 2.6 is 3 and stays for 2.9, 1.4 is 1 and goes for 1.2."""
    s = min(48, 62 - math.ceil(math.log2(C)))
    for weight, m, stays in ((0.6, 0.7, True), (0.55, 1.0, True), (2.6, 2.9, True), (1.4, 1.2, False), (0.4, 0.3, False), (9.6, 9.99, True)):
        z = torch.full((1, C), -200.0, device="cuda")
        z[0, 1], z[0, 5], z[0, C - 1] = math.log(weight) - s * math.log(2.0), 0.0, -1.0
        for rule in (dict(), dict(k=3), dict(k=4), dict(p=1 - 2.0 ** -24)):
            ids, _ = check(ks, z, 0.0, m=m * 2.0 ** -s, **rule)
            assert ids.item() == (1 if stays and "p" not in rule else 5), (weight, m, rule)
