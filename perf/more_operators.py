"""More operators of a linear model with many classes, as cases that can be timed and compared: training on the answers that the
model draws, noise on its rows, and serving it in four bits.

  policy      clipped policy loss of drawn classes, with a KL term against a reference, and its gradient in the scores
  preference  loss of paired log ratios (a preferred sequence of rows against another), and its gradient in the scores
  dropout     rows, or the gradient of such rows, with elements dropped by a counter-based generator; no mask is kept
  served      rows times class vectors of four bits with a scale for each group of 32, 64 or 128
  fresh       new class vectors put into four bits, and a first batch of rows scored by them

Sizes are this repository's own (rows of 4096 and 65536 elements) or generic ones around them.  Data are drawn on the
GPU from the seed.  Where `own` is false, run() computes the plain forms in elementary operations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
BLOCK = 128                                # elements of a row in whose 64 bytes the 4-bit codes have an order of their own
LEAST = 2.0 ** -126                        # the least scale of a group


def listed():
    return [
        # One small batch of answers, right after they were drawn: latency.
        dict(name="policy_small", op="policy", rows=64, classes=1000, storage="f32", masked=False, kl=0.0),
        # An odd vocabulary, classes masked out by -inf, padding, rows weighted, a KL term.
        dict(name="policy_masked", op="policy", rows=1023, classes=32001, storage="bf16", masked=True, kl=0.05),
        # A training batch over the wide output layer: 1 GiB of scores in, 1 GiB of gradient out.
        dict(name="policy_batch", op="policy", rows=8192, classes=65536, storage="bf16", masked=False, kl=0.02),
        # A few pairs of short answers of uneven length: latency.
        dict(name="preference_small", op="preference", pairs=6, length=9, classes=1001, storage="f32", kind="hinge", masked=True),
        # Pairs of a few hundred rows each over the wide output layer.
        dict(name="preference_batch", op="preference", pairs=16, length=256, classes=65536, storage="bf16", kind="logistic", masked=False),
        # One mini-batch picked by the sample stream on its way into the products.
        dict(name="dropout_small", op="dropout", rows=64, d=4096, storage="bf16", pad=0, picked=True, p=0.1),
        # The gradient of rows nobody padded: odd lengths, fp32, a stride of their own.
        dict(name="dropout_ragged", op="dropout", rows=4097, d=5003, storage="f32", pad=7, picked=False, p=0.5),
        # A large batch of wide rows.
        dict(name="dropout_large", op="dropout", rows=32768, d=8192, storage="bf16", pad=0, picked=False, p=0.1),
        # Serving, one row at a time: latency, and the class vectors read once.
        dict(name="served_one_row", op="served", rows=1, classes=4096, d=4096, storage="bf16", pad=0, group=128, out="bf16"),
        # Serving, a few rows against a wide output layer: the class vectors' 134 MB bound it.
        dict(name="served_few_rows", op="served", rows=16, classes=65536, d=4096, storage="bf16", pad=0, group=32, out="bf16"),
        # Class vectors of odd lengths from training, fp32 rows with a stride of their own.
        dict(name="fresh_ragged", op="fresh", rows=37, classes=5003, d=3001, storage="f32", pad=7, group=64, out="f32"),
        # The wide output layer as a worker has trained it, 1 GiB, made ready to serve.
        dict(name="fresh_wide", op="fresh", rows=8, classes=65536, d=4096, storage="f32", pad=0, group=128, out="f32"),
    ]


def draw(rng):
    def size(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["policy", "preference", "dropout", "served", "fresh"])
    storage = rng.choice(["f32", "bf16"])
    if op == "policy":
        return dict(op=op, rows=size(1, 4096), classes=size(2, 65536), storage=storage, masked=rng.random() < 0.5, kl=rng.choice([0.0, 0.02, 0.2]))
    if op == "preference":
        return dict(op=op, pairs=size(1, 32), length=size(1, 60), classes=size(2, 65536), storage=storage, kind=rng.choice(["hinge", "logistic", "logistic"]),
                    masked=rng.random() < 0.5)
    if op == "dropout":
        return dict(op=op, rows=size(1, 8192), d=size(1, 16000), storage=storage, pad=rng.choice([0, 0, 1, 8]), picked=rng.random() < 0.5,
                    p=rng.choice([0.05, 0.1, 0.3, 0.5]))
    case = dict(op=op, rows=size(1, 64), classes=size(64, 65536), d=size(64, 4096), storage=storage, pad=rng.choice([0, 0, 1, 8]),
                group=rng.choice([32, 64, 128]), out=rng.choice(["bf16", "f32"]))
    if op == "fresh":
        case["rows"] = min(case["rows"], 40)
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(gen, rows, cols, storage, scale=1.0, pad=0):
    """rows x cols normal values in rows of cols + pad elements."""
    full = torch.randn(rows, cols + pad, generator=gen, device="cuda") * scale
    return full.to(TYPES[storage])[:, :cols]


def prepare(case, seed):
    gen = _generator(seed)
    make = {"policy": _prepare_policy, "preference": _prepare_preference, "dropout": _prepare_dropout, "served": _prepare_served,
            "fresh": _prepare_fresh}[case["op"]]
    return {"case": case, **make(case, gen)}


def _scores(case, n, gen):
    """Scores of n rows, a class drawn from each row's softmax, and that class's log probability."""
    c = case["classes"]
    Z = torch.randn(n, c, generator=gen, device="cuda") * 3.0
    if case["masked"]:                                                          # a run of classes that may not be answered
        first = torch.randint(0, c, (n, 1), generator=gen, device="cuda")
        at = torch.arange(c, device="cuda")[None, :]
        Z.masked_fill_((at >= first) & (at < first + c // 3), -math.inf)
    Z = Z.to(TYPES[case["storage"]])
    race = torch.empty(n, c, device="cuda").exponential_(generator=gen)
    drawn = (Z.float() - race.log_()).argmax(1)
    del race
    log_p = Z.gather(1, drawn[:, None])[:, 0].float() - torch.logsumexp(Z.float(), 1)
    return Z, drawn, log_p


def _prepare_policy(case, gen):
    n = case["rows"]
    Z, drawn, log_p = _scores(case, n, gen)

    def near(width):                                                            # log probabilities under a model not far off
        return log_p + width * torch.randn(n, generator=gen, device="cuda")

    s = {"Z": Z, "drawn": drawn, "old": near(0.2), "ref": near(0.4) if case["kl"] else None,
         "advantage": torch.randn(n, generator=gen, device="cuda"), "weights": None, "low": 0.2, "high": 0.25, "kl": case["kl"], "scale": 1.0 / n}
    if case["masked"]:
        drawn[::13] = -1                                                        # padding
        s["weights"] = torch.rand(n, generator=gen, device="cuda") + 0.5
    return s


def _prepare_preference(case, gen):
    pairs, length = case["pairs"], case["length"]
    lengths = torch.randint(max(1, length // 2), length + length // 2 + 1, (2 * pairs,), generator=gen, device="cuda")
    lengths += (length - lengths.double().mean()).round().long()                # about pairs * 2 * length rows in all
    lengths.clamp_(min=0)
    offsets = torch.zeros(2 * pairs + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = lengths.cumsum(0)
    n = 2 * pairs * length + 3                                                  # a batch of one size, however long its sequences
    offsets.clamp_(max=n)
    Z, labels, log_p = _scores(case, n, gen)
    labels[n // 3::29] = -100                                                   # rows that do not count
    width = 4.0 / math.sqrt(length)
    ref = log_p + width * torch.randn(n, generator=gen, device="cuda")
    return {"Z": Z, "labels": labels, "offsets": offsets, "ref": ref, "beta": 0.1, "smoothing": 0.05 if case["masked"] else 0.0,
            "scale": 1.0 / pairs, "pair_weights": torch.rand(pairs, generator=gen, device="cuda") + 0.5 if case["masked"] else None}


def _prepare_dropout(case, gen):
    n, d = case["rows"], case["d"]
    X = _normal(gen, max(4096, n) if case["picked"] else n, d, case["storage"], 1.0, case["pad"])
    picked = torch.randint(0, X.shape[0], (n,), generator=gen, device="cuda") if case["picked"] else None
    word = torch.randint(0, 2 ** 31, (4,), generator=gen, device="cuda").tolist()
    return {"X": X, "picked": picked, "p": case["p"], "seed": word[0] << 32 | word[1], "chain": word[2] % 64, "step": word[3] % 100000}


def _rows(case, gen):
    m = max(4096, case["rows"])                                                 # the data set that the rows are picked from
    return {"X": _normal(gen, m, case["d"], case["storage"], 1.0, case["pad"]), "picked": torch.randint(0, m, (case["rows"],), generator=gen, device="cuda")}


def _prepare_served(case, gen):
    W = torch.randn(case["classes"], case["d"], generator=gen, device="cuda") / math.sqrt(case["d"])
    codes, scales = _to_four_bits(W, case["group"])                             # the class vectors as a serving program keeps them
    return {**_rows(case, gen), "codes": codes, "scales": scales}


def _prepare_fresh(case, gen):
    W = torch.randn(case["classes"], case["d"], generator=gen, device="cuda") / math.sqrt(case["d"])
    return {**_rows(case, gen), "W": W}


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"policy": _own_policy, "preference": _own_preference, "dropout": _own_dropout, "served": _own_served, "fresh": _own_fresh}[op](state)
    return {"policy": _plain_policy, "preference": _plain_preference, "dropout": _plain_dropout, "served": _plain_served, "fresh": _plain_fresh}[op](state)


def _own_policy(s):
    from paper_1708_04801_amd import api
    return api.wpsgd_policy_loss(s["Z"], s["drawn"], s["advantage"], old_log=s["old"], ref_log=s["ref"], row_weights=s["weights"], clip_low=s["low"],
                                 clip_high=s["high"], kl=s["kl"], scale=s["scale"])


def _own_preference(s):
    from paper_1708_04801_amd import api
    kind = api.HINGE if s["case"]["kind"] == "hinge" else api.LOGISTIC
    return api.wpsgd_preference_loss(s["Z"], s["labels"], s["offsets"], ref_log=s["ref"], pair_weights=s["pair_weights"], kind=kind, beta=s["beta"],
                                     smoothing=s["smoothing"], scale=s["scale"])


def _own_dropout(s):
    from paper_1708_04801_amd import api
    X = api.Matrix(s["X"].shape[0], s["X"].shape[1], dense=s["X"])
    return api.wpsgd_dropout(X, s["p"], s["seed"], chain=s["chain"], step=s["step"], rows=s["picked"])


def _own_served(s):
    from paper_1708_04801_amd import api
    X = api.Matrix(s["X"].shape[0], s["X"].shape[1], dense=s["X"])
    W = api.NibbleMatrix(s["case"]["classes"], s["case"]["d"], s["case"]["group"], s["codes"], s["scales"])
    return api.wpsgd_nibble_matmul(X, W, rows=s["picked"], dtype=TYPES[s["case"]["out"]])


def _own_fresh(s):
    from paper_1708_04801_amd import api
    X = api.Matrix(s["X"].shape[0], s["X"].shape[1], dense=s["X"])
    W = api.wpsgd_quantize_nibbles(api.Matrix(s["W"].shape[0], s["W"].shape[1], dense=s["W"]), group=s["case"]["group"])
    return api.wpsgd_nibble_matmul(X, W, rows=s["picked"], dtype=TYPES[s["case"]["out"]])


def _softmax(z):
    """exponentials relative to the rows' largest scores, their sums (in 64 bits), and the log of the softmax's denominator"""
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    return e, total, (top.double() + torch.log(total))[:, 0]


def _plain_policy(s):
    """The ratio is formed in 64 bits, since it is compared with borders."""
    z, drawn = s["Z"].float(), s["drawn"]
    counts = drawn >= 0
    r = s["weights"].double() if s["weights"] is not None else torch.ones(len(z), dtype=torch.float64, device=z.device)
    r = torch.where(counts, r, torch.zeros_like(r))
    e, total, lse = _softmax(z)
    at = drawn.clamp(min=0)[:, None]
    log_p = z.gather(1, at)[:, 0].double() - lse
    A = s["advantage"].double()
    ratio = torch.exp(log_p - s["old"].double())
    free, held = ratio * A, ratio.clamp(1.0 - s["low"], 1.0 + s["high"]) * A
    loss = -torch.minimum(free, held)
    slope = -torch.where(free <= held, free, torch.zeros_like(free))
    if s["ref"] is not None:
        gap = s["ref"].double() - log_p
        loss = loss + s["kl"] * (torch.exp(gap) - gap - 1.0)
        slope = slope + s["kl"] * (1.0 - torch.exp(gap))
    factor = (-s["scale"] * r * slope)[:, None]
    grad = e * (factor / total).float()
    grad.scatter_add_(1, at, -factor.float())
    return (loss * r).float(), torch.where(counts, log_p, torch.zeros_like(log_p)).float(), grad.to(s["Z"].dtype)


def _plain_preference(s):
    z, labels, offsets = s["Z"].float(), s["labels"], s["offsets"]
    pairs = (len(offsets) - 1) // 2
    e, total, lse = _softmax(z)
    at = labels.clamp(min=0)[:, None]
    place = torch.searchsorted(offsets, torch.arange(len(z), device=z.device), right=True) - 1       # which sequence a row is in
    counts = (labels >= 0) & (place < 2 * pairs)
    place = place.clamp(max=2 * pairs - 1)
    gain = z.gather(1, at)[:, 0].double() - lse - s["ref"].double()
    sums = torch.zeros(2 * pairs, dtype=torch.float64, device=z.device).index_add_(0, place, torch.where(counts, gain, torch.zeros_like(gain)))
    margin = s["beta"] * (sums[0::2] - sums[1::2])
    weight = s["pair_weights"].double() if s["pair_weights"] is not None else torch.ones_like(margin)
    loss, slope = torch.zeros_like(margin), torch.zeros_like(margin)
    for part, sign in ((1.0 - s["smoothing"], 1.0), (s["smoothing"], -1.0)):
        h = sign * margin
        if s["case"]["kind"] == "hinge":
            value, by_h = torch.clamp(1.0 - h, min=0.0), -(h < 1.0).double()
        else:
            value, by_h = torch.clamp(-h, min=0.0) + torch.log1p(torch.exp(-h.abs())), -1.0 / (1.0 + torch.exp(h))
        loss, slope = loss + part * value, slope + part * sign * by_h
    factor = (s["scale"] * s["beta"] * weight * slope)[place // 2] * torch.where(place % 2 == 0, -1.0, 1.0)
    factor = torch.where(counts, factor, torch.zeros_like(factor))[:, None]
    grad = e * (factor / total).float()
    grad.scatter_add_(1, at, -factor.float())
    return (loss * weight).float(), margin.float(), grad.to(s["Z"].dtype)


def _philox(c0, c1, c2, c3, seed):
    """Ten rounds of Philox4x32 in 64-bit whole numbers: tensors or numbers in, the four output words."""
    mask = 0xFFFFFFFF
    k0, k1 = seed & mask, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                                 # (mod 2^64)
        c0, c1, c2, c3 = ((b >> 32) & mask) ^ c1 ^ k0, b & mask, ((a >> 32) & mask) ^ c3 ^ k1, a & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return c0, c1, c2, c3


def _plain_dropout(s):
    x = s["X"] if s["picked"] is None else s["X"][s["picked"]]
    n, d = x.shape
    blocks = -(-d // 8)                                                         # eight elements to a call of the generator
    block = torch.arange(blocks, device=x.device)[None, :].expand(n, blocks)
    row = torch.arange(n, device=x.device)[:, None].expand(n, blocks)
    zero = torch.zeros_like(block)
    words = _philox(block, row, zero + s["chain"], zero + ((1 << 30) + s["step"] % (1 << 30)), s["seed"])
    drop = math.floor(s["p"] * 65536 + 0.5)
    keep = torch.stack([(w >> shift) & 0xFFFF for w in words for shift in (0, 16)], 2).reshape(n, 8 * blocks)[:, :d] >= drop
    factor = 65536.0 / (65536 - drop) if drop < 65536 else 0.0
    y = x.float() * factor
    return torch.where(keep, y, torch.zeros_like(y)).to(x.dtype)


def _to_four_bits(W, group):
    """Codes (sign, and which of 0, 1/2, 1, 3/2, 2, 3, 4, 6) and scales of the rows of W.  A block of 128 elements fills 64 bytes: element 32 j + 8 k + i of it is in byte
    16 k + 4 j + i / 2, the even one in the lower half.  A group's scale is the least bfloat16 value s (2^-126 or more) with 6 s >= its largest size, 1 for a group of
    zeros; a code is the nearest, half to even.  Rows of scales are padded to whole eights, with zeros."""
    r, c = W.shape
    blocks = -(-c // BLOCK)
    w = torch.nn.functional.pad(W.float(), (0, blocks * BLOCK - c)).reshape(r, -1, group)
    top = w.abs().amax(-1)
    s = ((top / 6.0).view(torch.int32) & -65536).view(torch.float32).clamp(min=LEAST)     # cut to bfloat16, then up as far as it takes
    for _ in range(2):
        s = torch.where(6.0 * s < top, (s.view(torch.int32) + 65536).view(torch.float32), s)
    s = torch.where(top > 0, s, torch.ones_like(s))
    size = w.abs()
    code = torch.zeros_like(w, dtype=torch.uint8)
    for i, border in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):                   # (halves of an odd place go up, to the even one)
        edge = (s * border)[..., None]
        code += (size >= edge if i % 2 else size > edge).to(torch.uint8)
    code += torch.signbit(w).to(torch.uint8) * 8
    code = code.reshape(r, blocks, 4, 4, 4, 2).transpose(2, 3)                             # j, k of 32 j + 8 k + 2 byte + half
    codes = (code[..., 0] | code[..., 1] << 4).reshape(r, blocks * 64)
    n = s.shape[1]
    used = -(-c // group)                                                                  # (groups of padding: 0)
    scales = torch.zeros(r, -(-n // 8) * 8, dtype=torch.bfloat16, device=W.device)
    scales[:, :used] = s[:, :used].to(torch.bfloat16)
    return codes, scales


def _from_four_bits(codes, scales, group, c):
    values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    r = codes.shape[0]
    code = torch.stack([codes & 15, codes >> 4], -1).reshape(r, -1, 4, 4, 4, 2).transpose(2, 3).reshape(r, -1, group)
    w = values[code.int()] * scales[:, :code.shape[1], None].float()
    return w.reshape(r, -1)[:, :c]


def _plain_served(s):
    case = s["case"]
    w = _from_four_bits(s["codes"], s["scales"], case["group"], case["d"])
    return (s["X"][s["picked"]].float() @ w.t()).to(TYPES[case["out"]])


def _plain_fresh(s):
    case = s["case"]
    w = _from_four_bits(*_to_four_bits(s["W"], case["group"]), case["group"], case["d"])
    return (s["X"][s["picked"]].float() @ w.t()).to(TYPES[case["out"]])


# ---- what one pass cannot do without ----------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "policy":
        n, c = case["rows"], case["classes"]
        return {"bytes": n * (2.0 * c * SIZE[case["storage"]] + 24 + (4 if case["kl"] else 0) + (4 if case["masked"] else 0)), "flops": 6.0 * n * c}
    if op == "preference":
        n, c = 2 * case["pairs"] * case["length"] + 3, case["classes"]
        return {"bytes": n * (2.0 * c * SIZE[case["storage"]] + 12) + case["pairs"] * 28.0, "flops": 6.0 * n * c}
    if op == "dropout":
        n, d = case["rows"], case["d"]
        return {"bytes": 2.0 * n * d * SIZE[case["storage"]] + (8 * n if case["picked"] else 0), "flops": 1.0 * n * d}
    n, c, d = case["rows"], case["classes"], case["d"]
    weights = d * 4.0 if op == "fresh" else d / 2 + 2.0 * -(-d // case["group"])
    return {"bytes": n * d * SIZE[case["storage"]] + 8 * n + c * weights + n * c * SIZE[case["out"]], "flops": 2.0 * n * c * d}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"policy": _exact_policy, "preference": _exact_preference, "dropout": _exact_dropout, "served": _exact_served, "fresh": _exact_fresh}[case["op"]](s)


def _exact_logs(Z):
    """Z becomes its rows' log probabilities, in 64 bits."""
    z = Z.double()
    z -= torch.logsumexp(z, 1, keepdim=True)
    return z


def _exact_gradient(log_p, labels, by_log):
    """d/dz of sum_i by_log_i log p_i,label, from all log probabilities (overwritten)."""
    rows = torch.arange(len(log_p), device=log_p.device)
    grad = log_p.exp_().mul_(-by_log[:, None])
    grad[rows, labels.clamp(min=0)] += by_log
    return grad


def _exact_policy(s):
    every = _exact_logs(s["Z"])
    rows, on = torch.arange(len(every), device="cuda"), s["drawn"] >= 0
    log_p = every[rows, s["drawn"].clamp(min=0)]
    r = (s["weights"].double() if s["weights"] is not None else torch.ones_like(log_p)) * on
    A = s["advantage"].double()
    ratio = (log_p - s["old"].double()).exp()
    low, high = 1.0 - s["low"], 1.0 + s["high"]
    # a gain beyond the border that it moves towards counts no further
    beyond = ((A > 0) & (ratio > high)) | ((A < 0) & (ratio < low))
    gain = torch.where(beyond, torch.where(A > 0, torch.full_like(A, high), torch.full_like(A, low)), ratio) * A
    loss, by_log = -gain, torch.where(beyond, torch.zeros_like(A), -ratio * A)
    if s["ref"] is not None:
        gap = s["ref"].double() - log_p
        loss = loss + s["kl"] * (torch.expm1(gap) - gap)
        by_log = by_log - s["kl"] * torch.expm1(gap)
    return r * loss, torch.where(on, log_p, torch.zeros_like(log_p)), _exact_gradient(every, s["drawn"], s["scale"] * r * by_log)


def _exact_preference(s):
    every = _exact_logs(s["Z"])
    n = len(every)
    rows, on = torch.arange(n, device="cuda"), s["labels"] >= 0
    gain = (every[rows, s["labels"].clamp(min=0)] - s["ref"].double()) * on
    ends = s["offsets"].tolist()
    by_log = torch.zeros(n, dtype=torch.float64, device="cuda")
    losses, margins = [], []
    for p in range((len(ends) - 1) // 2):
        a, b, c = ends[2 * p:2 * p + 3]
        h = s["beta"] * float(gain[a:b].sum() - gain[b:c].sum())
        w = float(s["pair_weights"][p]) if s["pair_weights"] is not None else 1.0
        eps = s["smoothing"]
        if s["case"]["kind"] == "hinge":
            loss, slope = (1 - eps) * max(0.0, 1 - h) + eps * max(0.0, 1 + h), (-(1 - eps) if h < 1 else 0.0) + (eps if h > -1 else 0.0)
        else:
            soft = max(-h, 0.0) + math.log1p(math.exp(-abs(h)))                 # -log sigma(h), and -log sigma(-h) = that + h
            loss, slope = soft + eps * h, -1.0 / (1.0 + math.exp(h)) + eps
        losses.append(w * loss)
        margins.append(h)
        by_log[a:b] = s["scale"] * w * slope * s["beta"]
        by_log[b:c] = -s["scale"] * w * slope * s["beta"]
    made = [torch.tensor(v, dtype=torch.float64, device="cuda") for v in (losses, margins)]
    return made[0], made[1], _exact_gradient(every, s["labels"], by_log * on)


def _exact_dropout(s):
    """The generator in unsigned 64-bit whole numbers of numpy, some rows at a time."""
    x = s["X"] if s["picked"] is None else s["X"][s["picked"]]
    n, d = x.shape
    blocks, u = (d + 7) // 8, np.uint64
    drop = int(s["p"] * 65536 + 0.5)
    low, half = u(0xFFFFFFFF), u(32)
    out = torch.zeros(n, d, dtype=torch.float64, device="cuda")
    some = max(1, (1 << 20) // blocks)
    for first in range(0, n, some):
        rows = min(some, n - first)
        v = np.zeros((4, rows * blocks), dtype=u)
        v[0] = np.tile(np.arange(blocks, dtype=u), rows)
        v[1] = np.repeat(np.arange(first, first + rows, dtype=u), blocks)
        v[2], v[3] = u(s["chain"]), u(2 ** 30 + s["step"] % 2 ** 30)
        for i in range(10):
            left, right = v[0] * u(0xD2511F53), v[2] * u(0xCD9E8D57)
            key = (s["seed"] + i * 0x9E3779B9) % 2 ** 32, ((s["seed"] >> 32) + i * 0xBB67AE85) % 2 ** 32
            v[0], v[2] = (right >> half) ^ v[1] ^ u(key[0]), (left >> half) ^ v[3] ^ u(key[1])
            v[1], v[3] = right & low, left & low
        bits = np.ascontiguousarray(v.T).astype("<u4").view("<u2").reshape(rows, 8 * blocks)[:, :d]
        out[first:first + rows] = torch.from_numpy(bits >= drop).cuda()
    out *= x.double()
    return out.mul_(65536.0 / (65536.0 - drop)) if drop < 65536 else out


_SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_rows(s):
    return s["X"][s["picked"]].double()


def _exact_served(s):
    d, group = s["case"]["d"], s["case"]["group"]
    value = torch.tensor([*_SIZES, *(-v for v in _SIZES)], dtype=torch.float64, device="cuda")
    at = torch.arange(d, device="cuda")
    within = at % 128
    byte = at // 128 * 64 + within % 32 // 8 * 16 + within // 32 * 4 + within % 8 // 2
    code = (s["codes"][:, byte] >> (4 * (within % 2)).to(torch.uint8)) & 15
    return _exact_rows(s) @ (value[code.long()] * s["scales"].double()[:, at // group]).t()


def _exact_fresh(s):
    W, group = s["W"].double(), s["case"]["group"]
    r, d = W.shape
    groups = -(-d // group)
    w = torch.zeros(r, groups * group, dtype=torch.float64, device="cuda")
    w[:, :d] = W
    w = w.reshape(r, groups, group)
    top = w.abs().amax(-1, keepdim=True)
    # the least multiple of the spacing of eight significant bits that six times reach the top
    _, e = torch.frexp(top / 6.0)
    unit = ((e.to(torch.int64) - 8 + 1023) << 52).view(torch.float64)           # 2^(e - 8) from its bits: a power function may be off
    scale = torch.ceil(top / (6.0 * unit)) * unit
    scale = torch.where(6.0 * (scale - unit) >= top, scale - unit, scale).clamp(min=LEAST)
    scale = torch.where(top > 0, scale, torch.ones_like(scale))
    v = w / scale                                                               # in 64 bits no quotient rounds onto a half that it is not
    size = v.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    value = torch.round(size / step) * step * torch.sign(v)
    return _exact_rows(s) @ (value * scale).reshape(r, -1)[:, :d].t()
