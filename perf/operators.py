"""The operators of a linear model with many classes (the output layer of a language model, trained by the workers
of weighted parallel SGD), as cases that can be timed and compared.

  scores    rows of the data set, picked by the sample stream, times the class vectors: both in 8-bit floating point
            with one power-of-two scale for each block of 128 along the summed axis
  gradient  the class vectors' gradient: the transposed loss gradient times the transposed rows, the same way
  loss      softmax cross-entropy of the scores, with its gradient
  step      global gradient norm over many tensors, clipping, and the regularised SGD update of all of them
  classes   a class drawn for each row from its scores: temperature, top-k, min-p and top-p, from given random numbers

Sizes are this repository's own (rows of 4096 and 65536 elements) or generic ones around them.  Data are drawn on the
GPU from the seed.  Where `own` is false, run() computes the plain forms in elementary operations.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
LOG2E = 1.4426950408889634
WEIGHT_ONE = 2.0 ** 31                     # what the largest score's weight is as a whole number

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # Serving, one row at a time: latency, and the class vectors read once.
        dict(name="scores_one_row", op="scores", rows=1, classes=4096, d=4096, storage="bf16", pad=0, out="bf16"),
        # Serving, a few rows against a wide output layer: the class vectors' 268 MB bound it.
        dict(name="scores_few_rows", op="scores", rows=16, classes=65536, d=4096, storage="bf16", pad=0, out="bf16"),
        # Training: a large batch against the same output layer, bound by the products.
        dict(name="scores_batch", op="scores", rows=8192, classes=65536, d=4096, storage="bf16", pad=0, out="bf16"),
        # A data set nobody padded: odd lengths all round, fp32 rows with a stride of their own.
        dict(name="gradient_ragged", op="gradient", rows=1001, classes=5003, d=3001, storage="f32", pad=7, out="f32"),
        # The class vectors' gradient of a training batch.
        dict(name="gradient_batch", op="gradient", rows=8192, classes=16384, d=4096, storage="bf16", pad=0, out="f32"),
        # A small batch over few classes: launch latency.
        dict(name="loss_small", op="loss", rows=64, classes=1000, storage="f32", masked=False),
        # An odd vocabulary, classes masked out by -inf, rows that do not count, a row with no class left.
        dict(name="loss_masked", op="loss", rows=1023, classes=32001, storage="bf16", masked=True),
        # A training batch over the wide output layer: 1 GiB of scores in, 1 GiB of gradient out.
        dict(name="loss_batch", op="loss", rows=8192, classes=65536, storage="bf16", masked=False),
        # Three hundred small tensors packed without gaps, so that most start anywhere.
        dict(name="step_many", op="step", tensors=300, total=3_000_000, storage="f32", clips=True),
        # A few large tensors: gradients in bfloat16, weights in fp32.
        dict(name="step_large", op="step", tensors=12, total=268_435_456, storage="bf16", clips=True),
        # One row's answer: latency.
        dict(name="classes_one_row", op="classes", rows=1, classes=32000, storage="f32", mixed=False),
        # A batch of requests, each with settings of its own, over a large vocabulary.
        dict(name="classes_batch", op="classes", rows=256, classes=131072, storage="bf16", mixed=True),
    ]


def draw(rng):
    def size(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["scores", "gradient", "loss", "step", "classes"])
    storage = rng.choice(["f32", "bf16"])
    if op == "scores":
        return dict(op=op, rows=size(1, 8192), classes=size(64, 65536), d=size(64, 4096), storage=storage,
                    pad=rng.choice([0, 0, 1, 8]), out=rng.choice(["bf16", "f32"]))
    if op == "gradient":
        return dict(op=op, rows=size(1, 8192), classes=size(64, 16384), d=size(64, 4096), storage=storage,
                    pad=rng.choice([0, 0, 3, 8]), out=rng.choice(["bf16", "f32"]))
    if op == "loss":
        return dict(op=op, rows=size(1, 4096), classes=size(2, 131072), storage=storage, masked=rng.random() < 0.5)
    if op == "step":
        return dict(op=op, tensors=size(1, 500), total=size(1000, 200_000_000), storage=storage, clips=rng.random() < 0.7)
    return dict(op=op, rows=size(1, 512), classes=size(100, 131072), storage=storage, mixed=rng.random() < 0.7)


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
    make = {"scores": _prepare_scores, "gradient": _prepare_gradient, "loss": _prepare_loss, "step": _prepare_step,
            "classes": _prepare_classes}[case["op"]]
    state = {"case": case, **make(case, gen)}
    if own and case["op"] == "step":       # the list that a training program makes once, its tensors staying where they are
        from paper_1708_04801_amd import api
        state["list"] = api.wpsgd_tensor_list(state["grads"], state["weights"])
    return state


def _prepare_scores(case, gen):
    m = max(4096, case["rows"])            # the data set the rows are picked from
    X = _normal(gen, m, case["d"], case["storage"], 1.0, case["pad"])
    W = torch.randn(case["classes"], case["d"], generator=gen, device="cuda") / math.sqrt(case["d"])
    codes, exps = _to_blocks(W)            # the class vectors as a serving program keeps them
    picked = torch.randint(0, m, (case["rows"],), generator=gen, device="cuda")
    return {"X": X, "picked": picked, "codes": codes, "exps": exps}


def _prepare_gradient(case, gen):
    m = max(4096, case["rows"])
    X = _normal(gen, m, case["d"], case["storage"], 1.0, case["pad"])
    picked = torch.randint(0, m, (case["rows"],), generator=gen, device="cuda")
    # a loss gradient: mostly small, a large negative entry at the label
    G = torch.exp(torch.randn(case["rows"], case["classes"], generator=gen, device="cuda") * 2.0)
    G /= G.sum(1, keepdim=True)
    label = torch.randint(0, case["classes"], (case["rows"], 1), generator=gen, device="cuda")
    G.scatter_add_(1, label, torch.full_like(label, -1, dtype=torch.float32))
    G = (G / case["rows"]).to(torch.bfloat16)
    return {"X": X, "picked": picked, "G": G}


def _prepare_loss(case, gen):
    n, c = case["rows"], case["classes"]
    Z = torch.randn(n, c, generator=gen, device="cuda") * 3.0
    labels = torch.randint(0, c, (n,), generator=gen, device="cuda")
    weights = None
    if case["masked"]:
        first = torch.randint(0, c, (n, 1), generator=gen, device="cuda")       # a run of classes that may not be answered
        at = torch.arange(c, device="cuda")[None, :]
        off = (at >= first) & (at < first + c // 3) & (at != labels[:, None])
        Z.masked_fill_(off, -math.inf)
        Z[n // 2] = -math.inf                                                   # a row with nothing left
        labels[::17] = -100                                                     # rows that do not count
        weights = torch.rand(n, generator=gen, device="cuda") + 0.5
    return {"Z": Z.to(TYPES[case["storage"]]), "labels": labels, "weights": weights, "scale": 1.0 / n}


def _prepare_step(case, gen):
    n, total = case["tensors"], case["total"]
    share = torch.rand(n, generator=gen, device="cuda").double().cumsum(0)
    ends = [0] + [int(v) for v in (share / share[-1] * total).tolist()]
    ends[-1] = total
    flat_g = (torch.randn(total, generator=gen, device="cuda") * 0.01).to(TYPES[case["storage"]])
    flat_w = torch.randn(total, generator=gen, device="cuda") * 0.02
    spans = [(a, b) for a, b in zip(ends, ends[1:]) if b > a]
    grads = [flat_g[a:b] for a, b in spans]
    weights = [flat_w[a:b] for a, b in spans]
    return {"grads": grads, "weights": weights, "flat_w": flat_w, "eta": 0.05, "lam": 1e-4,
            "max_norm": 0.005 * math.sqrt(total) if case["clips"] else 0.02 * math.sqrt(total)}


def _prepare_classes(case, gen):
    n, c = case["rows"], case["classes"]
    spread = torch.rand(n, 1, generator=gen, device="cuda") * 3.0 + 1.0         # flat rows and peaked ones
    Z = (torch.randn(n, c, generator=gen, device="cuda") * spread).to(TYPES[case["storage"]])
    u = torch.rand(n, generator=gen, device="cuda")
    if not case["mixed"]:
        return {"Z": Z, "u": u, "temperature": 0.8, "top_k": 50, "top_p": 0.95, "min_p": 0.0}

    def pick(values, dtype):
        t = torch.tensor(values, dtype=dtype, device="cuda")
        return t[torch.randint(0, len(values), (n,), generator=gen, device="cuda")]

    return {"Z": Z, "u": u, "temperature": pick([0.0, 0.6, 0.8, 1.0, 1.0, 1.5], torch.float32),
            "top_k": pick([0, 0, 1, 40, 50, 1000], torch.int32), "top_p": pick([1.0, 0.95, 0.9, 0.5], torch.float32),
            "min_p": pick([0.0, 0.0, 0.02, 0.1], torch.float32)}


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"scores": _own_scores, "gradient": _own_gradient, "loss": _own_loss, "step": _own_step, "classes": _own_classes}[op](state)
    return {"scores": _plain_scores, "gradient": _plain_gradient, "loss": _plain_loss, "step": _plain_step,
            "classes": _plain_classes}[op](state)


def _own_scores(s):
    from paper_1708_04801_amd import api
    X = api.Matrix(s["X"].shape[0], s["X"].shape[1], dense=s["X"])
    a = api.wpsgd_quantize(X, rows=s["picked"])
    b = api.BlockMatrix(s["case"]["classes"], s["case"]["d"], s["codes"], s["exps"])
    return api.wpsgd_block_matmul(a, b, dtype=TYPES[s["case"]["out"]])


def _own_gradient(s):
    from paper_1708_04801_amd import api
    X = api.Matrix(s["X"].shape[0], s["X"].shape[1], dense=s["X"])
    G = api.Matrix(s["G"].shape[0], s["G"].shape[1], dense=s["G"])
    g = api.wpsgd_quantize(G, transpose=True)
    x = api.wpsgd_quantize(X, rows=s["picked"], transpose=True)
    return api.wpsgd_block_matmul(g, x, dtype=TYPES[s["case"]["out"]])


def _own_loss(s):
    from paper_1708_04801_amd import api
    return api.wpsgd_softmax_loss(s["Z"], s["labels"], scale=s["scale"], row_weights=s["weights"])


def _own_step(s):
    from paper_1708_04801_amd import api
    norm = api.wpsgd_clipped_step(s["list"], s["eta"], s["lam"], s["max_norm"])
    return norm, s["flat_w"]


def _own_classes(s):
    from paper_1708_04801_amd import api
    return api.wpsgd_draw_classes(s["Z"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])


def _power_of_two(e):
    """2^e as fp32, for whole e from -126 to 127, put together from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _to_blocks(x):
    """e4m3 codes (padded to whole blocks) and biased exponents (padded to whole words) of the rows of x."""
    x = x.float()
    r, c = x.shape
    b = -(-c // BLOCK)
    x = torch.nn.functional.pad(x, (0, b * BLOCK - c)).reshape(r, b, BLOCK)
    size = x.abs()
    top = torch.where(torch.isfinite(size), size, torch.zeros_like(size)).amax(-1)
    mantissa, exponent = torch.frexp(top)                                   # top = mantissa * 2^exponent, 448 = 0.875 * 2^9
    e = exponent - 9 + (mantissa > 0.875).to(exponent.dtype)
    e = torch.where(top > 0, e, torch.zeros_like(e)).clamp(min=-126)
    codes = (x * _power_of_two(-e)[..., None]).to(torch.float8_e4m3fn).reshape(r, b * BLOCK)
    exps = torch.full((r, -(-b // 4) * 4), 127, dtype=torch.uint8, device=x.device)
    exps[:, :b] = (e + 127).to(torch.uint8)
    return codes, exps


def _from_blocks(codes, exps):
    r, n = codes.shape
    e = exps[:, :n // BLOCK].to(torch.int32) - 127
    return (codes.float().reshape(r, -1, BLOCK) * _power_of_two(e)[..., None]).reshape(r, n)


def _plain_scores(s):
    a = _from_blocks(*_to_blocks(s["X"][s["picked"]]))
    return (a @ _from_blocks(s["codes"], s["exps"]).t()).to(TYPES[s["case"]["out"]])


def _plain_gradient(s):
    g = _from_blocks(*_to_blocks(s["G"].t()))
    x = _from_blocks(*_to_blocks(s["X"][s["picked"]].t()))
    return (g @ x.t()).to(TYPES[s["case"]["out"]])


def _plain_loss(s):
    z, labels = s["Z"].float(), s["labels"]
    r = s["weights"] if s["weights"] is not None else torch.ones(len(z), device=z.device)
    counts = (labels >= 0) & (r != 0)
    at = labels.clamp(min=0)[:, None]
    top = z.amax(1, keepdim=True)
    empty = torch.isneginf(top)
    e = torch.exp(z - torch.where(empty, torch.zeros_like(top), top))
    total = e.sum(1, keepdim=True)
    loss = (top + torch.log(total) - z.gather(1, at))[:, 0] * r
    loss = torch.where(empty[:, 0], torch.full_like(loss, math.inf), loss)
    loss = torch.where(counts, loss, torch.zeros_like(loss))
    grad = e / total
    grad.scatter_add_(1, at, torch.full_like(top, -1.0))
    grad = grad * (s["scale"] * r)[:, None]
    grad = torch.where(counts[:, None] & ~empty, grad, torch.zeros_like(grad))
    return loss, grad.to(s["Z"].dtype)


def _plain_step(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.clamp(s["max_norm"] / norm, max=1.0) * s["eta"]
    factor = torch.where(torch.isfinite(norm), factor, torch.zeros_like(factor))
    shrink = torch.where(torch.isfinite(norm), torch.full_like(norm, 1.0 - s["eta"] * s["lam"]), torch.ones_like(norm))
    [w.mul_(shrink).sub_(g.float() * factor) for g, w in zip(s["grads"], s["weights"])]
    return norm, s["flat_w"]


def _column(v, n, dtype):
    if isinstance(v, torch.Tensor):
        return v.to(dtype)[:, None]
    return torch.full((n, 1), v, dtype=dtype, device="cuda")


def _plain_classes(s):
    """Classes in order of score, the lower index first among equals: the first top_k of them, those of them whose weight is at least min_p of the
    largest, and the shortest run from the front that holds top_p of what is left; one of those is drawn, by weight."""
    x = s["Z"].float() + 0.0
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    n, c = x.shape
    T = _column(s["temperature"], n, torch.float32)
    k, p, low = _column(s["top_k"], n, torch.int64), _column(s["top_p"], n, torch.float32), _column(s["min_p"], n, torch.float32)
    k = torch.where((k <= 0) | (T == 0), torch.where(T == 0, torch.ones_like(k), torch.full_like(k, c)), k)
    top = x.amax(1, keepdim=True)
    e = torch.exp2((x - top) * (torch.full_like(T, LOG2E) / torch.where(T == 0, torch.ones_like(T), T)))
    e = torch.where(x == top, torch.ones_like(e), e)
    q = torch.floor(e * WEIGHT_ONE + 0.5).to(torch.int64)
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    q_sorted = q.gather(1, order)
    place = torch.arange(c, device=x.device)[None, :]
    fits = (place < k) & (e.gather(1, order) >= low)
    q_sorted = torch.where(fits, q_sorted, torch.zeros_like(q_sorted))
    before = q_sorted.cumsum(1) - q_sorted
    total = q_sorted.sum(1, keepdim=True)
    need = torch.where(p < 1, torch.ceil(p.double() * total.double()).to(torch.int64), total)
    need = torch.minimum(torch.clamp(need, min=1), total)
    kept = fits & (before < need)
    q_kept = torch.zeros_like(q).scatter_(1, order, torch.where(kept, q_sorted, torch.zeros_like(q_sorted)))
    total = q_kept.sum(1, keepdim=True)
    target = torch.minimum((s["u"].double()[:, None] * total.double()).to(torch.int64), total - 1)
    answer = (q_kept.cumsum(1) <= target).sum(1)
    answer = torch.clamp(answer, max=c - 1)
    prob = (q_kept.gather(1, answer[:, None]).double() / total.double())[:, 0].float()
    empty = torch.isneginf(top)[:, 0]
    return torch.where(empty, torch.full_like(answer, -1), answer), torch.where(empty, torch.zeros_like(prob), prob)


# ---- what one pass cannot do without ----------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "scores":
        n, c, d = case["rows"], case["classes"], case["d"]
        return {"bytes": n * d * SIZE[case["storage"]] + 8 * n + c * d * (1 + 1 / BLOCK) + n * c * SIZE[case["out"]], "flops": 2.0 * n * c * d}
    if op == "gradient":
        n, c, d = case["rows"], case["classes"], case["d"]
        return {"bytes": n * d * SIZE[case["storage"]] + 8 * n + n * c * 2 + c * d * SIZE[case["out"]], "flops": 2.0 * n * c * d}
    if op == "loss":
        return {"bytes": case["rows"] * (2.0 * case["classes"] * SIZE[case["storage"]] + 12), "flops": 6.0 * case["rows"] * case["classes"]}
    if op == "step":
        return {"bytes": case["total"] * (SIZE[case["storage"]] + 8.0), "flops": 5.0 * case["total"]}
    return {"bytes": case["rows"] * (case["classes"] * float(SIZE[case["storage"]]) + 28), "flops": 6.0 * case["rows"] * case["classes"]}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"scores": _exact_scores, "gradient": _exact_gradient, "loss": _exact_loss, "step": _exact_step,
            "classes": _exact_classes}[case["op"]](s)


def _exact_two(e):
    """2^e in 64 bits, for whole e, put together from its bits: a power function may be off in the last place, and a half would not be one."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_blocks(x):
    """What the 8-bit values of the rows of x stand for: for each block the least power of two that brings its largest size to 448 or under,
    and the nearest multiple of the spacing that three mantissa bits leave (half to even; spacing 2^-9 below 2^-6)."""
    r, c = x.shape
    b = -(-c // BLOCK)
    y = torch.zeros(r, b * BLOCK, dtype=torch.float64, device=x.device)
    y[:, :c] = x.double()
    y = y.reshape(r, b, BLOCK)
    top = y.abs().amax(-1, keepdim=True)
    safe = torch.where(top > 0, top, torch.full_like(top, E4M3_MAX))
    e = torch.ceil(torch.log2(safe / E4M3_MAX))
    e = e + (safe > E4M3_MAX * _exact_two(e)).double() - (safe <= E4M3_MAX * _exact_two(e - 1)).double()
    unit = _exact_two(e)
    v = y / unit
    _, p = torch.frexp(v)
    step = _exact_two((p - 1).clamp(min=-6) - 3)
    return (torch.round(v / step) * step * unit).reshape(r, b * BLOCK)


def _exact_scores(s):
    a = _exact_blocks(s["X"][s["picked"]])
    n = s["codes"].shape[1]
    scale = _exact_two(s["exps"][:, :n // BLOCK].to(torch.int64) - 127)
    b = (s["codes"].double().reshape(-1, n // BLOCK, BLOCK) * scale[..., None]).reshape(-1, n)
    return a @ b.t()


def _exact_gradient(s):
    return _exact_blocks(s["G"].t()) @ _exact_blocks(s["X"][s["picked"]].t()).t()


def _exact_loss(s):
    z, labels = s["Z"].double(), s["labels"]
    r = s["weights"].double() if s["weights"] is not None else torch.ones(len(z), dtype=torch.float64, device="cuda")
    lse = torch.logsumexp(z, 1)
    at = labels.clamp(min=0)
    rows = torch.arange(len(z), device="cuda")
    none = torch.isinf(lse)
    loss = torch.where(none, torch.full_like(lse, math.inf), (lse - z[rows, at]) * r)
    loss = torch.where(labels < 0, torch.zeros_like(loss), loss)
    z -= torch.where(none, torch.zeros_like(lse), lse)[:, None]
    z.exp_()
    z[rows, at] -= 1.0
    z *= (s["scale"] * r * ((labels >= 0) & ~none))[:, None]
    return loss, z


def _exact_step(s):
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.clamp(s["max_norm"] / norm, max=1.0) * s["eta"]
    done = [w.double() * (1.0 - s["eta"] * s["lam"]) - factor * g.double() for g, w in zip(s["grads"], s["weights"])]
    return norm, torch.cat(done)


def _exact_classes(s):
    """Only the drawn class's probability is a computed number."""
    x = torch.nan_to_num(s["Z"].double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    n, c = x.shape
    T, p, low = (_column(s[v], n, torch.float32).double() for v in ("temperature", "top_p", "min_p"))
    k = _column(s["top_k"], n, torch.int64)
    greedy = T == 0
    top = x.amax(1, keepdim=True)
    weight = torch.exp((x - top) / torch.where(greedy, torch.ones_like(T), T))
    w, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = weight.gather(1, order)
    place = torch.arange(c, device=x.device)[None, :]
    first = torch.where(greedy, torch.ones_like(k), torch.where(k > 0, k, torch.full_like(k, c)))
    w = w * ((place < first) & (w >= low))
    sums = w.cumsum(1)
    w = w * ((sums - w < p * sums[:, -1:]) | (p >= 1))
    w = torch.zeros_like(w).scatter_(1, order, w)
    sums = w.cumsum(1)
    at = (sums <= s["u"].double()[:, None] * sums[:, -1:]).sum(1, keepdim=True).clamp(max=c - 1)
    return None, (w.gather(1, at) / sums[:, -1:])[:, 0]
