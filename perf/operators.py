"""Answering with a trained output layer, as cases to time and to compare.

  answer   the logits of a batch of features against every class from 8-bit codes of the class weights: the features are
           quantised row by row, the codes multiplied in integers, the scales of both sides applied
           (class_quantize_rows, class_logits_int8)
  refresh  the same right after training moved the fp32 weights: their rows are normalised and quantised first
  adjust   penalties for classes that a request has seen already, biases of single classes, and masks of allowed classes,
           from one logits matrix into another (class_logits_adjust)
  decode   one step of a serving loop: answer, then adjust in place

Sizes are those of the repository's configurations (10,000 to 1,000,000 classes, D = 128 to 512, batches up to 2,048), of one
request at a time, and of an output layer of generic size (131,072 classes of depth 4,096).  Inputs are made on the GPU from the
seed alone.
"""
import math

import torch

own = False

SCALE = 30.0
MAX_PRODUCT = 2_048 * 131_072 * 4_096  # B * C * D of the largest listed product
MAX_LOGITS = 256 * 390_625             # B * C of the largest listed adjustment


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one request against the smallest configuration: launches and latency
        {"name": "answer_one_small", "kind": "answer", "B": 1, "C": 10_000, "D": 128, "bf16": False, "prior": False},
        # one request against one GPU's share of 100 M classes: the codes are read once, at the rate of the memory
        {"name": "answer_one_shard", "kind": "answer", "B": 1, "C": 390_625, "D": 512, "bf16": True, "prior": True},
        # a ragged batch against an odd-sized layer of a depth that is no multiple of anything
        {"name": "answer_ragged", "kind": "answer", "B": 77, "C": 50_021, "D": 333, "bf16": False, "prior": True},
        # the benchmark's batch against the shard (an evaluation pass): the logits are what moves
        {"name": "answer_shard", "kind": "answer", "B": 1_024, "C": 390_625, "D": 512, "bf16": True, "prior": False},
        # a million classes on one GPU, logits in fp32: the largest output
        {"name": "answer_million", "kind": "answer", "B": 1_024, "C": 1_000_000, "D": 512, "bf16": False, "prior": False},
        # an output layer of generic size over deep features: the matrix pipes are what counts
        {"name": "answer_deep", "kind": "answer", "B": 2_048, "C": 131_072, "D": 4_096, "bf16": True, "prior": False},
        # validation inside a training loop, small: weights requantised, one batch answered
        {"name": "refresh_small", "kind": "refresh", "B": 64, "C": 10_000, "D": 128, "w_bf16": False, "bf16": False},
        # the same on the shard's fp32 weights
        {"name": "refresh_shard", "kind": "refresh", "B": 64, "C": 390_625, "D": 512, "w_bf16": False, "bf16": True},
        # one request of a small layer: a history and a grammar that allows few classes
        {"name": "adjust_one", "kind": "adjust", "B": 1, "C": 10_000, "nodes": 1, "bf16": False, "seen": 300, "biases": 20,
         "allow": 0.02},
        # a batch over one of four nodes of a sharded layer (ids of the whole problem), long histories, half of the classes out
        {"name": "adjust_node", "kind": "adjust", "B": 256, "C": 390_625, "nodes": 4, "bf16": True, "seen": 6_000, "biases": 300,
         "allow": 0.5},
        # one step of a serving loop for sixteen requests on the shard
        {"name": "decode_shard", "kind": "decode", "B": 16, "C": 390_625, "nodes": 1, "D": 512, "bf16": True, "seen": 1_024,
         "biases": 64, "allow": 0.9},
        # the same on the middle configuration with a category filter, fp32 logits
        {"name": "decode_small", "kind": "decode", "B": 5, "C": 100_000, "nodes": 1, "D": 256, "bf16": False, "seen": 200,
         "biases": 0, "allow": 0.1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("answer", "answer", "answer", "refresh", "adjust", "adjust", "decode"))
    bf16 = rng.random() < 0.5
    C = _log(rng, 2_000, 1_000_000 if kind == "answer" else 390_625)
    D = rng.choice((64, 96, 128, 256, 320, 512, 512, 1_024, _log(rng, 33, 4_096)))
    B = rng.choice((1, _log(rng, 2, 64), _log(rng, 2, 2_048), _log(rng, 64, 2_048)))
    if kind == "adjust":
        B = min(B, MAX_LOGITS // C, 512)
    else:
        # deep layers have fewer classes; a batch is cut to the work of the largest listed product and to 4 GB of logits
        C = min(C, 1_000_000 * 512 // D)
        B = max(1, min(B, MAX_PRODUCT // (C * D), (1 << 30) // C))
    case = {"kind": kind, "B": B, "C": C, "bf16": bf16}
    if kind != "adjust":
        case["D"] = D
    if kind == "answer":
        case["prior"] = rng.random() < 0.5
    elif kind == "refresh":
        case["w_bf16"] = rng.random() < 0.4
    else:
        case["nodes"] = rng.choice((1, 1, 2, 4)) if kind == "adjust" else 1
        case["seen"] = rng.choice((0, _log(rng, 1, 100), _log(rng, 100, 2_000), _log(rng, 2_000, 20_000)))
        case["biases"] = rng.choice((0, _log(rng, 1, 300)))
        case["allow"] = rng.choice((0.001, 0.02, 0.1, 0.5, 0.9, 0.99, 1.0))
        if kind == "decode":
            case["B"] = B = min(B, 64)
    return case


# ---------------------------------------------------------------------------------------------------- inputs
def _codes(V):
    """Rows as 8-bit codes and a scale each, as a checkpoint of an 8-bit layer holds them."""
    largest = V.abs().amax(1, keepdim=True).clamp_(min=1e-30)
    return torch.round(V * (127.0 / largest)).to(torch.int8), (largest[:, 0] / 127.0).contiguous()


def _unit(gen, n, D):
    return torch.nn.functional.normalize(torch.randn((n, D), generator=gen, device="cuda"))


def _features(gen, W, B):
    """Features of a trained model: near a class's own weight, some more than others."""
    C, D = W.shape
    label = torch.randint(0, C, (B,), generator=gen, device="cuda")
    near = torch.rand((B, 1), generator=gen, device="cuda")
    own_row = torch.nn.functional.normalize(W[label].float())
    return torch.nn.functional.normalize(own_row * near + _unit(gen, B, D) * (1 - near)).to(torch.bfloat16)


def _requests(gen, case):
    """What the requests of a batch bring: the classes that they have seen (the first part of each list from the prompt),
    penalties, biases for single classes, allowed classes.  Lists lie end to end."""
    B, C, nodes = case["B"], case["C"], case["nodes"]
    Cg, c0 = C * nodes, C * (nodes // 2)
    s = {"c0": c0, "Cg": Cg, "seen_max": case["seen"], "bias_max": case["biases"]}

    def offsets(most):
        n = torch.randint(0, most + 1, (B,), generator=gen, device="cuda")
        n[0] = most
        o = torch.zeros(B + 1, dtype=torch.int64, device="cuda")
        o[1:] = n.cumsum(0)
        return o

    s["seen_offsets"] = offsets(case["seen"])
    total = int(s["seen_offsets"][-1])
    # few classes make up most of a history, and they come again and again
    u = torch.rand(total, generator=gen, device="cuda", dtype=torch.float64)
    s["seen_ids"] = ((u ** 3 * Cg).to(torch.int64) * 7_919 % Cg).to(torch.int32)
    length = s["seen_offsets"].diff()
    s["n_prompt"] = (length * torch.rand(B, generator=gen, device="cuda")).to(torch.int32)
    s["repetition"] = 1.0 + 0.5 * torch.rand(B, generator=gen, device="cuda")
    s["presence"] = torch.rand(B, generator=gen, device="cuda")
    s["frequency"] = 0.5 * torch.rand(B, generator=gen, device="cuda")
    s["bias_offsets"] = offsets(case["biases"])
    total = int(s["bias_offsets"][-1])
    # a request names a class once: the ids of one list are spread over the classes by a step that shares no factor with Cg
    step, at = Cg // 3 | 1, torch.arange(total, device="cuda")
    while math.gcd(step, Cg) != 1:
        step += 2
    s["bias_ids"] = ((at + int(torch.randint(0, Cg, (1,), generator=gen, device="cuda"))) * step % Cg).to(torch.int32)
    s["bias_values"] = 5.0 * torch.randn(total, generator=gen, device="cuda")
    # masks: shared by requests of one grammar; one request in eight has none; each mask allows whole runs of classes, and some
    # of the others one by one
    words = (C + 31) // 32
    n_masks = max(1, B // 2)
    if case["allow"] < 1.0:
        runs = torch.rand((n_masks, words), generator=gen, device="cuda") < case["allow"] * 0.5
        ones = torch.rand((n_masks, words, 32), generator=gen, device="cuda") < case["allow"] * 0.5
        bits = (runs[:, :, None] | ones).to(torch.int64) << torch.arange(32, device="cuda")
        s["allowed"] = bits.sum(2).to(torch.int32)
        row = torch.randint(0, n_masks, (B,), generator=gen, device="cuda")
        none = torch.rand(B, generator=gen, device="cuda") < 0.125
        none[0] = False
        s["mask_row"] = torch.where(none, -1, row).to(torch.int32)
    else:
        s["allowed"] = s["mask_row"] = None
    return s


def _buffer(B, C, bf16):
    """A logits matrix whose rows begin on 128-byte lines."""
    return torch.empty((B, (C + 63) // 64 * 64), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")[:, :C]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    B, C, kind = case["B"], case["C"], case["kind"]
    s = {"case": case, "kind": kind, "type": torch.bfloat16 if case["bf16"] else torch.float32, "prior": None}
    if kind in ("adjust", "decode"):
        s.update(_requests(gen, case))
    if kind == "adjust":
        s["logits"] = _buffer(B, C, case["bf16"])
        s["logits"].copy_(4.0 * torch.randn((B, C), generator=gen, device="cuda"))
        return s
    W = _unit(gen, C, case["D"])
    s["X"] = _features(gen, W, B)
    if case.get("prior"):
        s["prior"] = -3.0 * torch.rand(C, generator=gen, device="cuda")
    if kind == "refresh":
        s["W"] = W * torch.exp(2.0 * torch.rand((C, 1), generator=gen, device="cuda") - 1.0)
        if case["w_bf16"]:
            s["W"] = s["W"].to(torch.bfloat16)
    else:
        s["W"], s["w_scale"] = _codes(W)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2102_06025_amd as ks
        # what a serving program allocates and lays out once
        s["ks"] = ks
        s["out"] = _buffer(case["B"], case["C"], case["bf16"])
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if "X" in s:
            s["X8"], s["x_scale"] = ks.class_quantize_rows(s["X"])
        if s["kind"] == "refresh":
            s["W8"], s["w_scale"] = ks.class_quantize_rows(s["W"], classes=True, normalize=True)
        elif "W" in s:
            s["W8"] = ks.class_quantize_rows(s.pop("W"), classes=True)[0]  # the checkpoint's codes in the product's order
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def _plain_codes(V, normalize=False):
    """Codes (as numbers) and scales of rows; in 64 bits, since values lie next to the border of two codes."""
    v = V.double()
    largest = v.abs().amax(1, keepdim=True)
    codes = torch.round(v * 127.0 / torch.where(largest > 0, largest, 1.0))
    scale = largest[:, 0] / 127.0
    if normalize:
        norm = (v * v).sum(1).sqrt()
        scale = scale / torch.where(norm > 0, norm, 1.0)
    return codes.float(), scale.float()


def _plain_logits(s):
    x, xs = _plain_codes(s["X"])
    if s["kind"] == "refresh":
        w, ws = _plain_codes(s["W"], normalize=True)
    else:
        w, ws = s["W"].float(), s["w_scale"]
    z = (x @ w.t()).mul_((SCALE * xs)[:, None]).mul_(ws[None, :])
    if s["prior"] is not None:
        z.add_(s["prior"][None, :])
    return z.to(s["type"]), ws


def _plain_adjust(s, logits):
    B, C = logits.shape
    z = logits.float()
    rows = torch.arange(B, device="cuda")
    # how often each class of this node was seen, in all and behind the prompt
    length = s["seen_offsets"].diff()
    row = torch.repeat_interleave(rows, length)
    place = torch.arange(row.numel(), device="cuda") - s["seen_offsets"][row]
    col = s["seen_ids"].long() - s["c0"]
    here = (col >= 0) & (col < C)
    row, col, place = row[here], col[here], place[here]
    flat = row * C + col
    seen = torch.zeros(B * C, dtype=torch.int32, device="cuda").scatter_add_(0, flat, torch.ones_like(flat, dtype=torch.int32))
    said = (place >= s["n_prompt"][row]).to(torch.int32)
    count = torch.zeros(B * C, dtype=torch.int32, device="cuda").scatter_add_(0, flat, said).view(B, C).float()
    r = s["repetition"][:, None]
    z = torch.where(seen.view(B, C) > 0, torch.where(z > 0, z / r, z * r), z)
    z = z - s["frequency"][:, None] * count - torch.where(count > 0, s["presence"][:, None], 0.0)
    # biases of single classes
    row = torch.repeat_interleave(rows, s["bias_offsets"].diff())
    col = s["bias_ids"].long() - s["c0"]
    here = (col >= 0) & (col < C)
    z[row[here], col[here]] += s["bias_values"][here]
    if s["allowed"] is not None:
        at = torch.arange(C, device="cuda")
        allowed = (s["allowed"][:, at // 32] >> (at % 32).to(torch.int32) & 1).bool()
        out = ~allowed[s["mask_row"].clamp(min=0).long()] & (s["mask_row"] >= 0)[:, None]
        z = z.masked_fill_(out, -math.inf)
    return z.to(logits.dtype)


def _own_adjust(s, logits, out):
    return s["ks"].class_logits_adjust(logits, seen=(s["seen_ids"], s["seen_offsets"]), seen_max=s["seen_max"],
                                       n_prompt=s["n_prompt"], repetition=s["repetition"], presence=s["presence"],
                                       frequency=s["frequency"], bias=(s["bias_ids"], s["bias_values"], s["bias_offsets"]),
                                       bias_max=s["bias_max"], allowed=s["allowed"], mask_row=s["mask_row"], c0=s["c0"],
                                       Cg=s["Cg"], out=out, dev_status=s["status"])


def run(s):
    kind = s["kind"]
    if not own:
        if kind == "adjust":
            return _plain_adjust(s, s["logits"])
        z, ws = _plain_logits(s)
        return _plain_adjust(s, z) if kind == "decode" else (z, ws) if kind == "refresh" else z
    if kind == "adjust":
        return _own_adjust(s, s["logits"], s["out"])
    ks = s["ks"]
    if kind == "refresh":
        ks.class_quantize_rows(s["W"], classes=True, normalize=True, codes=s["W8"], row_scale=s["w_scale"])
    ks.class_quantize_rows(s["X"], codes=s["X8"], row_scale=s["x_scale"])
    z = ks.class_logits_int8(s["X8"], s["x_scale"], s["W8"], s["w_scale"], SCALE, bias=s["prior"], out=s["out"])
    if kind == "decode":
        return _own_adjust(s, z, z)
    return (z, s["w_scale"]) if kind == "refresh" else z


def work(case):
    B, C, kind = case["B"], case["C"], case["kind"]
    logits = B * C * (2 if case["bf16"] else 4)
    lists = 0
    if kind in ("adjust", "decode"):
        masks = max(1, B // 2) * ((C + 31) // 32) * 4 if case["allow"] < 1.0 else 0
        lists = B * (case["seen"] * 4 + case["biases"] * 8) // 2 + masks
    if kind == "adjust":
        return {"bytes": 2 * logits + lists, "flops": B * C}
    D = case["D"]
    weights = C * D + 4 * C
    if kind == "refresh":
        weights += C * D * (2 if case["w_bf16"] else 4)  # the weights in, the codes out
    return {"bytes": weights + 2 * B * D + logits + lists, "flops": 2 * B * C * D}


# ---------------------------------------------------------------------------------------------------- 64 bits
def _exact_logits(s, W, w_scale):
    """In 64 bits; the whole numbers of the codes multiply exactly there."""
    X = s["X"].to(torch.float64)
    peak = torch.maximum(X.max(dim=1).values, -X.min(dim=1).values)
    qx = torch.round(X * 127.0 / peak[:, None])
    z = torch.mm(qx, W.to(torch.float64).transpose(0, 1))
    z *= (peak / 127.0 * SCALE).unsqueeze(1)
    z *= w_scale.to(torch.float64).unsqueeze(0)
    return z if s["prior"] is None else z + s["prior"].to(torch.float64).unsqueeze(0)


def _exact_adjust(s, z):
    C, c0 = z.shape[1], s["c0"]
    z = z.to(torch.float64)
    for b in range(z.shape[0]):
        lo, hi = int(s["seen_offsets"][b]), int(s["seen_offsets"][b + 1])
        prompt = int(s["n_prompt"][b])
        ids = s["seen_ids"][lo:hi].long()
        mine = ids[(ids >= c0) & (ids < c0 + C)].unique() - c0
        v = z[b, mine]
        r = s["repetition"][b].double()
        z[b, mine] = torch.where(v > 0, v / r, v * r)
        ids = ids[prompt:]
        mine, n = ids[(ids >= c0) & (ids < c0 + C)].unique(return_counts=True)
        z[b, mine - c0] -= s["frequency"][b].double() * n + s["presence"][b].double()
        lo, hi = int(s["bias_offsets"][b]), int(s["bias_offsets"][b + 1])
        ids = s["bias_ids"][lo:hi].long()
        keep = (ids >= c0) & (ids < c0 + C)
        z[b, ids[keep] - c0] += s["bias_values"][lo:hi][keep].double()
        m = -1 if s["mask_row"] is None else int(s["mask_row"][b])
        if m >= 0:
            bits = s["allowed"][m][:, None].bitwise_right_shift(torch.arange(32, dtype=torch.int32, device="cuda")) % 2
            z[b] = torch.where(bits.reshape(-1)[:C] != 0, z[b], -math.inf)
    return z


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "adjust":
        return _exact_adjust(s, s["logits"])
    if kind == "refresh":
        W = s["W"].to(torch.float64)
        norm, peak = torch.linalg.vector_norm(W, dim=1), torch.maximum(W.max(dim=1).values, -W.min(dim=1).values)
        w_scale = peak / (127.0 * norm)
        return _exact_logits(s, torch.round(W * 127.0 / peak[:, None]), w_scale), w_scale
    z = _exact_logits(s, s["W"], s["w_scale"])
    if kind != "decode":
        return z
    # the logits are stored in their type before they are adjusted
    return _exact_adjust(s, z.to(s["type"]))
