"""GPU parity of include/class_distill.h against a plain implementation in 64 bits, with tolerances that count its roundings."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32, TYPES = 2.0 ** -24, {torch.float32: 0.0, torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2}
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ks():
    import paper_2102_06025_amd as ks
    ks.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return ks


@pytest.fixture(autouse=True)
def name_the_case(request):
    print(f"[distill] {request.node.name}", flush=True)


# ---------------------------------------------------------------------------------------------------- plain form
def plain(z, ids, t, T, grad_scale):
    """-> loss, gradient, and what their roundings are relative to."""
    B, C = z.shape
    z, t = z.double() / T, torch.where(ids >= 0, t.double() / T, -INF)
    at = ids.clamp(min=0).long()
    top = z.amax(1, keepdim=True)
    base = torch.where(top > -INF, top, 0.0)
    e = (z - base).exp()
    S = e.sum(1, keepdim=True)
    p = torch.where(S > 0, e / S, 0.0)
    t_top = t.amax(1, keepdim=True)
    some = t_top > -INF
    w = torch.where(some, (t - torch.where(some, t_top, 0.0)).exp(), 0.0)
    q = torch.where(some, w / w.sum(1, keepdim=True), 0.0)
    log_q = t - torch.where(some, t_top, 0.0) - torch.where(some, w.sum(1, keepdim=True).log(), 0.0)
    log_p = torch.where(S > 0, z.gather(1, at) - base - S.log(), -INF)
    loss = T * T * torch.where(q != 0, q * (log_q - log_p), 0.0).sum(1)
    target = torch.zeros_like(z).scatter_add_(1, at, torch.where(ids >= 0, q, 0.0))
    g = grad_scale * T / B
    grad = torch.where(some, p - target, 0.0) * g
    # powers: 3 roundings of the exponent, times ln 2; sums: up to 64 terms one after the other and 30 on the way up, of terms that
    # are as far off as the average exponent, at most log2 C below the largest in the mean; 10 for quotients, products and the power itself
    depth = ((z - base) * math.log2(math.e)).abs().clamp(max=200.0)
    size = (p * (104 + 2.1 * (depth + 20)) + target * (60 + 2.1 * (17 + 20 * 2))) * abs(g)
    K_sum = torch.where(q != 0, q * (log_q.abs() + z.gather(1, at).abs()), 0.0).sum(1)
    loss_size = T * T * (150 + 4.2 * 20 + 120 * K_sum) + loss.abs()
    return loss, grad, size, loss_size


def close(got, want, size, step, tag):
    assert torch.equal(got.isnan(), want.isnan()), tag
    got, finite = got.double(), want.isfinite()
    assert torch.equal(got[~finite & ~want.isnan()], want[~finite & ~want.isnan()]), tag
    off = (got - want).abs() - 1.01 * (U32 * size + step * want.abs()) - 2.0 ** -120
    assert off[finite].numel() == 0 or off[finite].max().item() <= 0, (tag, off[finite].max().item())


def check(ks, z, ids, t, T=1.0, grad_scale=1.0, **more):
    want, grad, size, loss_size = plain(z, ids.where(ids < z.shape[1], -1), t, T, grad_scale)
    o = ks.class_distill_fwd_bwd(z, ids, t, temperature=T, grad_scale=grad_scale, **more)
    close(o["loss_per_sample"], want, loss_size, 0.0, "loss")
    close(o["loss_mean"], want.mean()[None], loss_size.mean()[None], 0.0, "mean")
    close(o["dlogits"], grad, size, TYPES[z.dtype], "gradient")
    return o


def matrix(B, C, dtype, ld, shift, fill=None):
    store = torch.full((B * ld + shift,), 7.0, dtype=dtype, device="cuda")
    m = torch.as_strided(store, (B, C), (ld, 1), shift)
    if fill is not None:
        m.copy_(fill)
    return store, m


def inputs(gen, B, C, K, dtype, t_dtype=torch.float32, again=False):
    z = (2 * torch.randn((B, C), generator=gen, device="cuda")).to(dtype)
    if again:
        ids = torch.randint(0, C, (B, K), generator=gen, device="cuda")
    else:
        ids = (torch.arange(K, device="cuda") * (C // K) + torch.randint(0, C // K, (B, K), generator=gen, device="cuda"))
        ids = ids.gather(1, torch.rand((B, K), generator=gen, device="cuda").argsort(1))
    t = (4 * torch.randn((B, K), generator=gen, device="cuda")).to(t_dtype)
    z.scatter_(1, ids, (0.7 * t.float()).to(dtype))
    return z, ids.to(torch.int32), t


# ---------------------------------------------------------------------------------------------------- parity
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,K", [(1, 1, 1), (2, 2, 1), (3, 7, 3), (5, 100, 10), (4, 255, 7), (33, 1_000, 32), (17, 4_097, 64), (64, 10_000, 32), (3, 8_193, 1_000),
                                   (9, 16_385, 100), (77, 50_021, 100), (2, 390_625, 4_096), (260, 3_000, 50)])
def test_loss_and_gradient(ks, B, C, K, dtype):
    gen = torch.Generator("cuda").manual_seed(B + C)
    z, ids, t = inputs(gen, B, C, K, dtype, torch.bfloat16 if C % 2 else torch.float32)
    for T, scale in ((1.0, 1.0), (2.5, 1_024.0), (0.5, -3.0)):
        check(ks, z, ids, t, T, scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C,pad,shift,pad2,shift2", [(1_000, 0, 0, 0, 0), (999, 0, 0, 0, 0), (9_001, 0, 3, 0, 3), (9_001, 0, 1, 7, 0), (17_000, 5, 1, 5, 1), (20_003, 1, 2, 9, 2),
                                                     (6, 0, 1, 0, 1), (5, 3, 0, 3, 1), (16_384, 8, 0, 16, 0)])
def test_rows_that_lie_apart_or_beside_each_other(ks, C, pad, shift, pad2, shift2, dtype):
    gen = torch.Generator("cuda").manual_seed(C + shift)
    B, K = 5, min(20, C // 2)
    z, ids, t = inputs(gen, B, C, K, dtype)
    _, z = matrix(B, C, dtype, C + pad, shift, z)
    store, d = matrix(B, C, dtype, C + pad2, shift2)
    out = dict(loss_per_sample=torch.empty(B, device="cuda"), loss_mean=torch.empty(1, device="cuda"), dlogits=d)
    o = check(ks, z, ids, t, 1.5, out=out)
    assert o["dlogits"] is d
    d.fill_(7.0)
    assert (store == 7.0).all(), "written outside the gradient"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C", [50, 10_000, 40_001])
def test_in_place_is_the_same(ks, C, dtype):
    gen = torch.Generator("cuda").manual_seed(C)
    z, ids, t = inputs(gen, 12, C, 24, dtype)
    want = ks.class_distill_fwd_bwd(z, ids, t, temperature=2.0)
    keep = want["loss_per_sample"].clone()
    out = dict(loss_per_sample=torch.empty(12, device="cuda"), loss_mean=torch.empty(1, device="cuda"), dlogits=z)
    ks.class_distill_fwd_bwd(z, ids, t, temperature=2.0, out=out)
    assert torch.equal(z, want["dlogits"]) and torch.equal(out["loss_per_sample"], keep)


def test_classes_that_are_named_again(ks):
    gen = torch.Generator("cuda").manual_seed(2)
    for C, K in ((3, 40), (30, 64), (20_000, 2_000), (9_000, 4_096)):
        z, ids, t = inputs(gen, 6, C, K, torch.float32, again=True)
        first = check(ks, z, ids, t, 1.3)
        again = ks.class_distill_fwd_bwd(z, ids, t, temperature=1.3)
        assert torch.equal(first["dlogits"], again["dlogits"])
    ids[:] = 17
    check(ks, z, ids, t, 1.0)


def test_empty_entries_and_padding(ks):
    gen = torch.Generator("cuda").manual_seed(3)
    B, C, K = 12, 5_000, 33
    z, ids, t = inputs(gen, B, C, K, torch.float32)
    ids[0] = -1
    ids[1, 1:] = -7
    ids[2, ::2] = -2 ** 31
    t[3] = -INF
    t[4, 5:] = -INF
    t[5, 0], ids[5, 0] = NAN, -1  # nobody reads what an empty entry holds
    t[6] *= 1e4
    t[7] = 0.0
    o = check(ks, z, ids, t, 2.0)
    assert o["loss_per_sample"][[0, 3]].tolist() == [0.0, 0.0] and not o["dlogits"][[0, 3]].any()
    assert int(o["dev_status"]) == 0
    # padding may hold anything
    z[0, 7], z[3] = NAN, INF
    o = ks.class_distill_fwd_bwd(z, ids, t, temperature=2.0)
    assert o["loss_per_sample"][[0, 3]].tolist() == [0.0, 0.0] and not o["dlogits"][[0, 3]].any()
    assert o["loss_mean"].isfinite().all()


def test_masked_classes(ks):
    gen = torch.Generator("cuda").manual_seed(4)
    B, C, K = 8, 3_000, 16
    z, ids, t = inputs(gen, B, C, K, torch.float32)
    mask = torch.rand((B, C), generator=gen, device="cuda") < 0.7
    mask.scatter_(1, ids.long(), False)
    z.masked_fill_(mask, -INF)
    z[1, ids[1, 3].long()] = -INF   # a class that the teacher names
    z[2] = -INF                     # a mask that leaves nothing
    z[3] = -INF
    z[3, ids[3, 0].long()] = 2.0    # and one that leaves one
    z[4] = torch.where(mask[4], -3.4028234e38, z[4])
    o = check(ks, z, ids, t)
    assert o["loss_per_sample"][[1, 2, 3]].tolist() == [INF] * 3 and o["loss_mean"].item() == INF
    assert o["dlogits"].isfinite().all() and not o["dlogits"][0][mask[0]].any()
    ids[3, 1:] = -1
    assert ks.class_distill_fwd_bwd(z, ids, t)["loss_per_sample"][3].item() == 0.0


def test_infinities_and_nan(ks):
    gen = torch.Generator("cuda").manual_seed(5)
    z, ids, t = inputs(gen, 6, 2_000, 9, torch.float32)
    z[0, 100], z[1, 7], z[1, 8] = NAN, INF, INF
    t[2, 4], t[3, 1] = NAN, INF
    o = ks.class_distill_fwd_bwd(z, ids, t)
    assert o["loss_per_sample"].isnan().tolist() == [True] * 4 + [False] * 2
    assert o["dlogits"][:2].isnan().all() and not o["dlogits"][4:].isnan().any()
    for b in (2, 3):
        named = torch.zeros(2_000, dtype=torch.bool, device="cuda")
        named[ids[b].long()] = True
        assert torch.equal(o["dlogits"][b].isnan(), named)


def test_large_logits_and_temperatures(ks):
    gen = torch.Generator("cuda").manual_seed(6)
    z, ids, t = inputs(gen, 4, 3_000, 20, torch.float32)
    check(ks, z * 50, ids, t * 50, 1.0)
    check(ks, z + 1e4, ids, t - 1e4, 1.0)
    check(ks, z, ids, t, 100.0)
    check(ks, z, ids, t, 0.02)


def test_ids_beyond_the_classes_are_reported(ks):
    gen = torch.Generator("cuda").manual_seed(7)
    z, ids, t = inputs(gen, 3, 1_000, 5, torch.float32)
    ids[1, 2], ids[2, 0] = 1_000, 2 ** 31 - 1
    o = check(ks, z, ids, t)
    assert int(o["dev_status"]) == ks.KS_DEV_BAD_LABEL


def test_gradient_against_differences(ks):
    """Central differences of the GPU's losses.  Third derivatives of a loss are below 1 / T; losses are off by 2e-5 at most here."""
    gen = torch.Generator("cuda").manual_seed(8)
    C, K, T, eps = 12, 5, 1.5, 0.03
    z, ids, t = inputs(gen, 1, C, K, torch.float32)
    grad = ks.class_distill_fwd_bwd(z, ids, t, temperature=T)["dlogits"][0]
    step = torch.eye(C, device="cuda") * eps
    up = ks.class_distill_fwd_bwd(z + step, ids.expand(C, K).contiguous(), t.expand(C, K).contiguous(), temperature=T)["loss_per_sample"]
    down = ks.class_distill_fwd_bwd(z - step, ids.expand(C, K).contiguous(), t.expand(C, K).contiguous(), temperature=T)["loss_per_sample"]
    assert ((up - down) / (2 * eps) - grad).abs().max().item() <= eps ** 2 / (6 * T) + 2e-5 / eps


def test_one_named_class_is_the_ordinary_loss(ks):
    """A teacher that is sure of one class: the loss and gradient of the full softmax."""
    gen = torch.Generator("cuda").manual_seed(9)
    B, C, D, s = 32, 1_000, 64, 20.0
    W = torch.nn.functional.normalize(torch.randn((C, D), generator=gen, device="cuda")).to(torch.bfloat16)
    X = torch.nn.functional.normalize(torch.randn((B, D), generator=gen, device="cuda")).to(torch.bfloat16)
    y = torch.randint(0, C, (B,), generator=gen, device="cuda", dtype=torch.int32)
    full = ks.full_softmax_fwd_bwd(W, X, y, s)
    o = ks.class_distill_fwd_bwd(s * (X.float() @ W.float().t()), y[:, None].contiguous(), torch.zeros((B, 1), device="cuda"))
    assert torch.allclose(o["loss_per_sample"], full["loss_per_sample"], atol=1e-3)
    dX = s * (o["dlogits"] @ W.float())
    assert (dX - full["dX"]).abs().max() <= 2.0 ** -8 * 4 * full["dX"].abs().max()  # the full softmax keeps its gradient in bf16


def test_offsets_beyond_32_bits(ks):
    gen = torch.Generator("cuda").manual_seed(10)
    z, ids, t = inputs(gen, 2, 3_000, 5, torch.bfloat16)
    store = torch.empty((2, (1 << 31) + 64), dtype=torch.bfloat16, device="cuda")
    far = store[:, :3_000]
    far.copy_(z)
    check(ks, far, ids, t, out=dict(loss_per_sample=torch.empty(2, device="cuda"), loss_mean=torch.empty(1, device="cuda"), dlogits=far.clone()))
    check(ks, far, ids, t)


def test_more_rows_than_a_launch_takes(ks):
    gen = torch.Generator("cuda").manual_seed(12)
    z, ids, t = inputs(gen, 33_000, 20, 3, torch.float32)
    check(ks, z, ids, t, 2.0, 100.0)


def test_streams_graphs_and_shared_workspaces(ks):
    gen = torch.Generator("cuda").manual_seed(11)
    B, C, K = 10, 20_000, 30
    z, ids, t = inputs(gen, B, C, K, torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o = ks.class_distill_fwd_bwd(z, ids, t, stream=side)
    side.synchronize()
    want = ks.class_distill_fwd_bwd(z, ids, t)
    assert all(torch.equal(o[k], want[k]) for k in ("loss_per_sample", "loss_mean", "dlogits"))
    ws = torch.empty(ks.class_distill_workspace(C, B, K), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graphs = []
    for T in (1.0, 3.0):
        out = dict(loss_per_sample=torch.empty(B, device="cuda"), loss_mean=torch.empty(1, device="cuda"), dlogits=torch.empty_like(z))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ks.class_distill_fwd_bwd(z, ids, t, temperature=T, out=out, ws=ws, dev_status=status)
        graphs.append((g, T, out))
    for _ in range(3):
        new = inputs(gen, B, C, K, torch.bfloat16)
        for a, b in zip((z, ids, t), new):
            a.copy_(b)
        for g, T, out in graphs:
            g.replay()
            want = ks.class_distill_fwd_bwd(z, ids, t, temperature=T)
            torch.cuda.synchronize()
            assert all(torch.equal(out[k], want[k]) for k in ("loss_per_sample", "loss_mean", "dlogits"))
    assert int(status) == 0


def test_a_step_that_learns_from_a_larger_layer(ks):
    """The teacher answers in 4 bits, its top logits become the target; the student's gradient is that of the plain formulas."""
    gen = torch.Generator("cuda").manual_seed(13)
    B, C, D, K = 24, 2_000, 128, 20
    Wt = torch.nn.functional.normalize(torch.randn((C, D), generator=gen, device="cuda"))
    X = torch.nn.functional.normalize(Wt[torch.randint(0, C, (B,), generator=gen, device="cuda")] + 0.1 * torch.randn((B, D), generator=gen, device="cuda"))
    z = ks.class_logits_mxfp4(ks.class_quantize_mxfp4(X), ks.class_quantize_mxfp4(Wt, classes=True), B, C, D, 30.0)
    t, ids = z.topk(K, 1)
    W = torch.nn.functional.normalize(torch.randn((C, 32), generator=gen, device="cuda"))
    check(ks, 10.0 * X[:, :32] @ W.t(), ids.to(torch.int32), t.contiguous(), 2.0)


def test_refusals_of_tensors(ks):
    gen = torch.Generator("cuda").manual_seed(14)
    z, ids, t = inputs(gen, 3, 100, 5, torch.float32)
    with pytest.raises(ValueError):
        ks.class_distill_fwd_bwd(z, ids[:2], t[:2])
    with pytest.raises(ValueError):
        ks.class_distill_fwd_bwd(z, ids, t[:, :4])
    with pytest.raises(TypeError):
        ks.class_distill_fwd_bwd(z, ids.long(), t)
    with pytest.raises(TypeError):
        ks.class_distill_fwd_bwd(z, ids, t.half())
    with pytest.raises(ValueError):
        ks.class_distill_fwd_bwd(z, ids, t, out=dict(loss_per_sample=torch.empty(3, device="cuda"), loss_mean=torch.empty(1, device="cuda"),
                                                     dlogits=torch.empty((3, 100), dtype=torch.bfloat16, device="cuda")))
    for T in (0.0, NAN, INF):
        with pytest.raises(ks.KsError) as e:
            ks.class_distill_fwd_bwd(z, ids, t, temperature=T)
        assert e.value.code == ks.KS_INVALID_ARG
    with pytest.raises(ks.KsError) as e:
        ks.class_distill_fwd_bwd(z, torch.zeros((3, 4_097), dtype=torch.int32, device="cuda"), torch.zeros((3, 4_097), device="cuda"))
    assert e.value.code == ks.KS_UNSUPPORTED


def loss_rounding(z, ids, t, T):
    """What the loss is off by at most, whatever is added to all logits of a row.  A power of x = (z - m) / T: three roundings of x, and the
    power itself (two); a sum of them: 64 one after the other and 30 on the way up.  With them the row's sum, the teacher's sum and each q."""
    z, t = z.double() / T, t.double() / T
    p, depth = torch.softmax(z, 1), (z - z.amax(1, keepdim=True)).abs().clamp(max=120.0)
    q, depth_t = torch.softmax(t, 1), (t - t.amax(1, keepdim=True)).abs().clamp(max=120.0)
    of_sum = 96 + 3 * (p * depth).sum(1)
    of_t = 2 + 3 * (q * depth_t).sum(1)
    log_ratio = torch.log_softmax(t, 1) - torch.log_softmax(z, 1).gather(1, ids.long())
    of_q = (q * (2 + 3 * depth_t + of_t[:, None]) * log_ratio.abs()).sum(1)
    loss = (q * log_ratio).sum(1)
    return T * T * loss, T * T * (1.05 * U32 * (of_sum + of_t + of_q + loss.abs()) + 2.0 ** -50 * (z.abs().amax(1) + 50))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_number_added_to_all_logits_changes_no_loss(ks, dtype):
    gen = torch.Generator("cuda").manual_seed(21)
    for C, K, T in ((1_000, 128, 1.0), (20_000, 60, 2.0), (300, 300, 1.0), (50, 1, 0.7)):
        z, ids, t = inputs(gen, 16, C, K, dtype)
        for add in (0.0, 30.0, -1e3, 1e4, 3e5):
            shifted = (z.float() + add).to(dtype)
            want, off = loss_rounding(shifted, ids, t, T)
            got = ks.class_distill_fwd_bwd(shifted, ids, t, temperature=T)["loss_per_sample"].double()
            worst = ((got - want).abs() - off).max().item()
            assert worst <= 0, (C, K, T, add, (got - want).abs().max().item(), off.max().item())


def test_a_student_that_matches_its_teacher(ks):
    """The teacher names every class with the student's own logits: no loss, wherever they lie."""
    gen = torch.Generator("cuda").manual_seed(22)
    for C, add, T in ((128, 0.0, 1.0), (128, 30.0, 1.0), (1_000, -1e3, 2.0), (4_096, 1e4, 1.0)):
        z = (2 * torch.randn((8, C), generator=gen, device="cuda") + add)
        ids = torch.rand((8, C), generator=gen, device="cuda").argsort(1).to(torch.int32)
        t = z.gather(1, ids.long())
        want, off = loss_rounding(z, ids, t, T)
        o = ks.class_distill_fwd_bwd(z, ids, t, temperature=T)
        assert ((o["loss_per_sample"].double() - want).abs() <= off).all(), (C, add, o["loss_per_sample"].abs().max().item(), off.max().item())
        assert want.abs().max().item() <= 1e-12 * (1 + abs(add))
