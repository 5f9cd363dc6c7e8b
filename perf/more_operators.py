"""Answering with a trained layer in 4 bits, drawing a class from its logits, and learning from a teacher's top logits, as cases
to time and to compare.

  codes    rows as microscaled 4-bit floating point (blocks of 32 elements, a power of two each) and back: what a layer keeps of
           itself in 4 bits, as training for 4 bits computes it every step (class_quantize_mxfp4, class_dequantize_mxfp4)
  answer   the logits of a batch of features against every class from the 4-bit codes of the class weights: the features are
           quantised, the codes multiplied (class_quantize_mxfp4, class_logits_mxfp4)
  draw     one class per request from its row of the logits, with temperature, top-k, top-p and min-p, by a given random number
           (class_sample)
  distill  loss and gradient of a batch of logits that learns from a teacher's top logits (class_distill_fwd_bwd)

Sizes are those of the repository's configurations (10,000 to 1,000,000 classes, D = 128 to 512, batches up to 2,048), of one
request at a time, and of an output layer of generic size (131,072 classes of depth 4,096).  Inputs are made on the GPU from the
seed alone.
"""
import math

import torch

own = False

SCALE = 30.0
MAX_PRODUCT = 2_048 * 131_072 * 4_096  # B * C * D of the largest listed product
MAX_ROWS = 390_625 * 512               # n * D of the largest listed rows
MAX_DRAW = 256 * 390_625               # B * C of the largest listed draw
MAX_DISTILL = 1_024 * 390_625          # B * C of the largest listed distillation


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the features of one batch
        {"name": "codes_batch", "kind": "codes", "n": 1_024, "D": 512, "bf16": True, "classes": False},
        # fp32 weights of one GPU's share of 100 M classes
        {"name": "codes_shard", "kind": "codes", "n": 390_625, "D": 512, "bf16": False, "classes": True},
        # one request against the smallest configuration: launches and latency
        {"name": "answer4_one_small", "kind": "answer", "B": 1, "C": 10_000, "D": 128, "bf16": False, "prior": False},
        # one request against the shard: the codes are read once, at the rate of the memory
        {"name": "answer4_one_shard", "kind": "answer", "B": 1, "C": 390_625, "D": 512, "bf16": True, "prior": True},
        # the benchmark's batch against the shard (an evaluation pass): the logits are what moves
        {"name": "answer4_shard", "kind": "answer", "B": 1_024, "C": 390_625, "D": 512, "bf16": True, "prior": False},
        # an output layer of generic size over deep features: the matrix pipes are what counts
        {"name": "answer4_deep", "kind": "answer", "B": 2_048, "C": 131_072, "D": 4_096, "bf16": True, "prior": False},
        # one request of a small layer, with the usual filters
        {"name": "draw_one", "kind": "draw", "B": 1, "C": 10_000, "bf16": False, "spread": 1.3, "top_k": 50, "top_p": 0.95, "min_p": 0.0,
         "mixed": False, "masked": 0.0},
        # requests of every kind in one batch over the shard, half of the classes masked out
        {"name": "draw_shard", "kind": "draw", "B": 256, "C": 390_625, "bf16": True, "spread": 1.3, "top_k": 500, "top_p": 0.9, "min_p": 0.05,
         "mixed": True, "masked": 0.5},
        # a flat distribution of which most has to be kept: no few candidates hold the answer
        {"name": "draw_flat", "kind": "draw", "B": 16, "C": 100_000, "bf16": False, "spread": 0.7, "top_k": 0, "top_p": 0.98, "min_p": 0.0,
         "mixed": False, "masked": 0.0},
        # a small student
        {"name": "distill_small", "kind": "distill", "B": 64, "C": 10_000, "K": 32, "bf16": False, "temperature": 2.0, "ragged": False},
        # a ragged batch: some teachers name fewer classes, a few rows are padding
        {"name": "distill_ragged", "kind": "distill", "B": 77, "C": 50_021, "K": 100, "bf16": False, "temperature": 1.0, "ragged": True},
        # the benchmark's batch over the shard
        {"name": "distill_shard", "kind": "distill", "B": 1_024, "C": 390_625, "K": 128, "bf16": True, "temperature": 3.0, "ragged": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("codes", "answer", "answer", "draw", "draw", "distill", "distill"))
    bf16 = rng.random() < 0.5
    D = rng.choice((64, 96, 128, 256, 320, 512, 512, 1_024, _log(rng, 33, 4_096)))
    C = _log(rng, 2_000, 1_000_000)
    if kind == "codes":
        return {"kind": kind, "n": min(_log(rng, 1, 390_625), MAX_ROWS // D), "D": D, "bf16": bf16, "classes": rng.random() < 0.5}
    B = rng.choice((1, _log(rng, 2, 64), _log(rng, 2, 2_048), _log(rng, 64, 2_048)))
    if kind == "answer":
        # deep layers have fewer classes; a batch is cut to the work of the largest listed product and to 4 GB of logits
        C = min(C, 1_000_000 * 512 // D)
        B = max(1, min(B, MAX_PRODUCT // (C * D), (1 << 30) // C))
        return {"kind": kind, "B": B, "C": C, "D": D, "bf16": bf16, "prior": rng.random() < 0.5}
    if kind == "draw":
        return {"kind": kind, "B": min(B, 512, MAX_DRAW // C), "C": C, "bf16": bf16, "spread": rng.choice((0.5, 1.0, 1.3, 2.0, 4.0)),
                "top_k": rng.choice((0, 0, _log(rng, 1, 1_000), _log(rng, 1, 20_000))),
                "top_p": rng.choice((1.0, round(rng.uniform(0.05, 0.999), 3))),
                "min_p": rng.choice((0.0, 0.0, round(rng.uniform(0.001, 0.5), 3))), "mixed": rng.random() < 0.4,
                "masked": rng.choice((0.0, 0.0, 0.3, 0.9, 0.999))}
    return {"kind": kind, "B": min(B, MAX_DISTILL // C), "C": C, "K": _log(rng, 1, 1_000), "bf16": bf16,
            "temperature": rng.choice((1.0, 2.0, round(rng.uniform(0.5, 8.0), 2))), "ragged": rng.random() < 0.4}


# ---------------------------------------------------------------------------------------------------- inputs
def _unit(gen, n, D):
    return torch.nn.functional.normalize(torch.randn((n, D), generator=gen, device="cuda"))


def _features(gen, W, B):
    """Features of a trained model: near a class's own weight, some more than others."""
    C, D = W.shape
    label = torch.randint(0, C, (B,), generator=gen, device="cuda")
    near = torch.rand((B, 1), generator=gen, device="cuda")
    return torch.nn.functional.normalize(W[label] * near + _unit(gen, B, D) * (1 - near)).to(torch.bfloat16)


def _buffer(B, C, dtype):
    """A matrix whose rows begin on 128-byte lines."""
    return torch.empty((B, (C + 63) // 64 * 64), dtype=dtype, device="cuda")[:, :C]


def _near(gen, B, C, K):
    """K different classes a row, in any order."""
    step = C // K
    ids = torch.arange(K, device="cuda") * step + torch.randint(0, step, (B, K), generator=gen, device="cuda")
    return ids.gather(1, torch.rand((B, K), generator=gen, device="cuda").argsort(1))


def _draw_inputs(gen, case, s):
    B, C = case["B"], case["C"]
    z = _buffer(B, C, s["type"])
    z.copy_(case["spread"] * torch.randn((B, C), generator=gen, device="cuda"))
    # a sample's near classes stand out from the others, the nearest most
    near = min(60, C // 2)
    peak = 4.0 + 16.0 * torch.rand((B, 1), generator=gen, device="cuda")
    z.scatter_(1, _near(gen, B, C, near), (peak * torch.rand((B, near), generator=gen, device="cuda") ** 2).to(s["type"]))
    if case["masked"]:
        z.masked_fill_(torch.rand((B, C), generator=gen, device="cuda") < case["masked"], -math.inf)
    s["logits"] = z
    s["u"] = torch.rand(B, generator=gen, device="cuda")
    s["temperature"] = 0.5 + torch.rand(B, generator=gen, device="cuda")
    s["top_k"] = torch.full((B,), case["top_k"], dtype=torch.int32, device="cuda")
    s["top_p"] = torch.full((B,), case["top_p"], device="cuda")
    s["min_p"] = torch.full((B,), case["min_p"], device="cuda")
    if case["mixed"]:  # each request has its own settings, one in sixteen wants the largest logit
        def some(share):
            return torch.rand(B, generator=gen, device="cuda") < share
        few = (torch.rand(B, generator=gen, device="cuda") * (case["top_k"] + 1)).to(torch.int32)
        s["top_k"] = torch.where(some(0.5), few, 0).to(torch.int32)
        s["top_p"] = torch.where(some(0.5), 1.0, s["top_p"])
        s["min_p"] = torch.where(some(0.5), 0.0, s["min_p"])
        s["temperature"] = torch.where(some(0.0625), 0.0, s["temperature"])


def _distill_inputs(gen, case, s):
    B, C, K = case["B"], case["C"], case["K"]
    z = _buffer(B, C, s["type"])
    z.copy_(1.3 * torch.randn((B, C), generator=gen, device="cuda"))
    ids = _near(gen, B, C, K)
    top = 20.0 * torch.rand((B, 1), generator=gen, device="cuda")
    t = (top - 12.0 * torch.rand((B, K), generator=gen, device="cuda") ** 0.5).sort(1, descending=True).values
    # the student knows some of it
    z.scatter_(1, ids, (0.6 * t + torch.randn((B, K), generator=gen, device="cuda")).to(s["type"]))
    if case["ragged"]:
        count = (torch.rand((B, 1), generator=gen, device="cuda") * (K + 1)).to(torch.int64)
        ids = torch.where(torch.arange(K, device="cuda") < count, ids, -1)
    s["logits"], s["ids"], s["teacher"] = z, ids.to(torch.int32), t


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    s = {"case": case, "kind": kind, "type": torch.bfloat16 if case["bf16"] else torch.float32, "prior": None}
    if kind == "codes":
        s["V"] = (_unit(gen, case["n"], case["D"]) * torch.exp(2.0 * torch.rand((case["n"], 1), generator=gen, device="cuda") - 1.0)).to(s["type"])
    elif kind == "answer":
        W = _unit(gen, case["C"], case["D"])
        s["X"], s["W"] = _features(gen, W, case["B"]), W.to(torch.bfloat16)
        if case["prior"]:
            s["prior"] = -3.0 * torch.rand(case["C"], generator=gen, device="cuda")
    elif kind == "draw":
        _draw_inputs(gen, case, s)
    else:
        _distill_inputs(gen, case, s)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if not own:
        if kind == "answer":  # the checkpoint's codes, twice their values as whole numbers, and exponents
            s["W"] = [_plain_codes(part) for part in s["W"].split(1 << 16)]
            s["W"] = torch.cat([c for c, _ in s["W"]]), torch.cat([e for _, e in s["W"]])
        return s
    import paper_2102_06025_amd as ks
    # what a program allocates and lays out once
    s["ks"] = ks
    if kind == "codes":
        s["codes"] = torch.empty(ks.class_mxfp4_bytes(case["n"], case["D"], case["classes"]), dtype=torch.uint8, device="cuda")
        s["values"] = torch.empty((case["n"], case["D"]), dtype=torch.bfloat16, device="cuda")
    elif kind == "answer":
        s["w4"] = ks.class_quantize_mxfp4(s.pop("W"), classes=True)
        s["x4"] = ks.class_quantize_mxfp4(s["X"])
        s["out"] = _buffer(case["B"], case["C"], s["type"])
    elif kind == "draw":
        s["ids"] = torch.empty(case["B"], dtype=torch.int32, device="cuda")
        s["logprob"] = torch.empty(case["B"], dtype=torch.float32, device="cuda")
        s["ws"] = torch.empty(ks.class_sample_workspace(case["C"], case["B"]), dtype=torch.uint8, device="cuda")
    else:
        s["out"] = {"loss_per_sample": torch.empty(case["B"], device="cuda"), "loss_mean": torch.empty(1, device="cuda"),
                    "dlogits": _buffer(case["B"], case["C"], s["type"])}
        s["ws"] = torch.empty(ks.class_distill_workspace(case["C"], case["B"], case["K"]), dtype=torch.uint8, device="cuda")
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def _plain_codes(V):
    """Rows in blocks of 32 along the depth: twice the 4-bit values as whole numbers, and the blocks' exponents."""
    n, D = V.shape
    v = torch.nn.functional.pad(V.float(), (0, -D % 32)).view(n, -1, 32)
    largest = v.abs().amax(2)
    e = torch.where(largest > 0, torch.frexp(largest).exponent - 3, 0)
    a = torch.ldexp(v, -e[:, :, None])
    # the values are 0, 0.5, 1, 1.5, 2, 3, 4, 6: steps of 0.5 below 2, of 1 below 4, of 2 above
    size = a.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    code = (torch.round(a / step) * step).clamp_(-6.0, 6.0) * 2.0
    return code.to(torch.int8), e.to(torch.int8)


def _plain_values(code, e, D):
    return torch.ldexp(code.float() * 0.5, e[:, :, None].to(torch.int32)).flatten(1)[:, :D]


def _plain_draw(s):
    z = s["logits"].double()
    B, C = z.shape
    z, order = z.sort(dim=1, descending=True, stable=True)
    largest, t = z[:, :1], s["temperature"].double()[:, None]
    largest, none = torch.where(largest == -math.inf, 0.0, largest), largest == -math.inf  # a mask may leave nothing
    greedy = t <= 0
    place = torch.arange(C, device="cuda")
    w = torch.where(greedy, ((place == 0) & ~none).double(), ((z - largest) / torch.where(greedy, 1.0, t)).exp())
    del z
    k = s["top_k"][:, None]
    keep = (place < k) | (k <= 0)
    w = torch.where(keep, w, 0.0)
    p = s["top_p"].double()[:, None]
    before = w.cumsum(1) - w
    keep &= (before < p * w.sum(1, keepdim=True)) | (p >= 1) | (place == 0)
    del before
    keep &= w >= s["min_p"].double()[:, None].clamp(max=1.0)
    w = torch.where(keep, w, 0.0)
    by_id = torch.zeros_like(w).scatter_(1, order, w)
    del order, w, keep
    cum = by_id.cumsum(1)
    total = cum[:, -1:]
    ids = (cum <= s["u"].double()[:, None] * total).sum(1, keepdim=True)
    logprob = torch.where(none, -math.inf, (by_id.gather(1, ids.clamp(max=C - 1)) / total).log())
    return torch.where(none, -1, ids)[:, 0].to(torch.int32), logprob[:, 0].float()


def _plain_distill(s):
    case = s["case"]
    z = s["logits"].float() / case["temperature"]
    B, C = z.shape
    largest = z.amax(1, keepdim=True)
    lse = largest + (z - largest).exp_().sum(1, keepdim=True, dtype=torch.float64).log_().float()
    there = s["ids"] >= 0
    at = s["ids"].clamp(min=0).long()
    t = torch.where(there, s["teacher"] / case["temperature"], -math.inf)
    t = t - t.amax(1, keepdim=True).nan_to_num(neginf=0.0)
    q = t.exp()
    total = q.sum(1, keepdim=True)
    some = (total > 0).float()
    log_q = t - torch.where(total > 0, total, 1.0).log()
    q = q / torch.where(total > 0, total, 1.0)
    loss = torch.where(q > 0, q * (log_q - (z.gather(1, at) - lse)), 0.0).sum(1) * case["temperature"] ** 2
    p = z.sub_(lse).exp_().mul_(some).scatter_add_(1, at, -q)
    return loss, loss.mean()[None], p.mul_(case["temperature"] / B).to(s["type"])


def run(s):
    kind = s["kind"]
    if own:
        ks = s["ks"]
        if kind == "codes":
            case = s["case"]
            ks.class_quantize_mxfp4(s["V"], classes=case["classes"], codes=s["codes"])
            return ks.class_dequantize_mxfp4(s["codes"], case["n"], case["D"], classes=case["classes"], out=s["values"])
        if kind == "answer":
            case = s["case"]
            ks.class_quantize_mxfp4(s["X"], codes=s["x4"])
            return ks.class_logits_mxfp4(s["x4"], s["w4"], case["B"], case["C"], case["D"], SCALE, bias=s["prior"], out=s["out"])
        if kind == "draw":
            return ks.class_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                                   ids=s["ids"], logprob=s["logprob"], ws=s["ws"])
        out = ks.class_distill_fwd_bwd(s["logits"], s["ids"], s["teacher"], temperature=s["case"]["temperature"], out=s["out"], ws=s["ws"],
                                       dev_status=s["status"])
        return out["loss_per_sample"], out["loss_mean"], out["dlogits"]
    if kind == "codes":
        return _plain_values(*_plain_codes(s["V"]), s["case"]["D"]).to(torch.bfloat16)
    if kind == "answer":
        D = s["case"]["D"]
        z = (_plain_values(*_plain_codes(s["X"]), D) @ _plain_values(*s["W"], D).t()).mul_(SCALE)
        if s["prior"] is not None:
            z.add_(s["prior"][None, :])
        return z.to(s["type"])
    return _plain_draw(s) if kind == "draw" else _plain_distill(s)


def work(case):
    kind, size = case["kind"], 2 if case["bf16"] else 4
    if kind == "codes":
        return {"bytes": case["n"] * case["D"] * (size + 2), "flops": 2 * case["n"] * case["D"]}
    B, C = case["B"], case["C"]
    if kind == "answer":
        D = case["D"]
        blocks = (D + 31) // 32 * 17  # 32 elements and their exponent
        return {"bytes": C * blocks + 2 * B * D + B * C * size + (4 * C if case["prior"] else 0), "flops": 2 * B * C * D}
    if kind == "draw":
        return {"bytes": B * C * size + 28 * B, "flops": 3 * B * C}
    return {"bytes": 2 * B * C * size + B * case["K"] * 8 + 4 * B, "flops": 6 * B * C}


# ---------------------------------------------------------------------------------------------------- 64 bits
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_values(V):
    """The nearest of the 4-bit values times the block's power of two, of two equally near ones that with an even code."""
    grid = torch.tensor(_GRID, dtype=torch.float64, device="cuda")
    middle = (grid[1:] + grid[:-1]) / 2
    parts = []
    for v in V.split(1 << 14):
        n, D = v.shape
        x = torch.zeros((n, (D + 31) // 32 * 32), dtype=torch.float64, device="cuda")
        x[:, :D] = v
        x = x.view(n, -1, 32)
        peak = torch.maximum(x.max(dim=2).values, -x.min(dim=2).values)
        unit = torch.exp2(torch.floor(torch.log2(torch.where(peak > 0, peak, 1.0))) - 2.0)[:, :, None]
        a = x.abs() / unit
        below, above = torch.bucketize(a, middle), torch.bucketize(a, middle, right=True)
        code = torch.where(below % 2 == 0, below, above)
        parts.append((torch.sign(x) * grid[code] * unit).reshape(n, -1)[:, :D])
    return parts


def _exact_draw(s):
    B, C = s["logits"].shape
    ids, logprob = [], []
    for b in range(B):
        z = s["logits"][b].to(torch.float64)
        order = torch.argsort(-z, stable=True)
        if z[order[0]] == -math.inf:  # nothing to draw
            ids.append(order[0] * 0 - 1)
            logprob.append(z[order[0]])
            continue
        t, k, p = float(s["temperature"][b]), int(s["top_k"][b]), float(s["top_p"][b])
        n = 1 if t <= 0 else k if 0 < k < C else C
        order = order[:n]
        w = torch.exp((z[order] - z[order[0]]) / (t if t > 0 else 1.0))
        total = torch.cumsum(w, 0)
        if p < 1.0:
            n = 1 + int((total < p * total[-1]).sum())
        n = min(n, int((w >= min(float(s["min_p"][b]), 1.0)).sum()))
        kept, at = torch.sort(order[:n])
        w = w[:n][at]
        total = torch.cumsum(w, 0)
        place = int(torch.searchsorted(total, float(s["u"][b]) * total[-1:], right=True))
        ids.append(kept[place])
        logprob.append(torch.log(w[place]) - torch.log(total[-1]))
    return torch.stack(ids).to(torch.int32), torch.stack(logprob)


def _exact_distill(s):
    B, C = s["logits"].shape
    t = s["case"]["temperature"]
    loss, grad = [], []
    for b in range(0, B, 128):
        z = s["logits"][b:b + 128].to(torch.float64) / t
        log_p = torch.log_softmax(z, dim=1)
        target = torch.zeros_like(log_p)
        for r in range(log_p.shape[0]):
            named = s["ids"][b + r] >= 0
            ids = s["ids"][b + r][named].long()
            if ids.numel() == 0:
                log_p[r] = -math.inf
                continue
            target[r].index_add_(0, ids, torch.softmax(s["teacher"][b + r][named].double() / t, 0))
        loss.append(t * t * (torch.xlogy(target, target) - torch.where(target > 0, target * log_p, 0.0)).sum(1))
        grad.append((log_p.exp() - target) * (t / B))
    loss = torch.cat(loss)
    return loss, loss.sum().reshape(1) / B, torch.cat(grad)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "codes":
        return torch.cat(_exact_values(s["V"]))
    if kind == "answer":
        x = torch.cat(_exact_values(s["X"]))
        z = torch.cat([torch.mm(x, w.transpose(0, 1).contiguous()) for w in _exact_values(s["W"])], 1) * SCALE
        return z if s["prior"] is None else z + s["prior"].to(torch.float64).unsqueeze(0)
    return _exact_draw(s) if kind == "draw" else _exact_distill(s)
