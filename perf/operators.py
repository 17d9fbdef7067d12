"""The operators of a worker's local step in preference tuning, measured through
the framework's public calls: linear layers with microscaled 4-bit operands
(forward, single tokens, both gradients, the codec itself), the preference loss
over paired sequences with its gradient, and the clipping of each worker's
gradient over its many tensors.

A case is a dict of plain values:
  op      "linear" (y = x W^T, W kept in 4 bits), "linear_grad" (dx and dW from
          dy), "codec" (to 4 bits and back), "preference" (losses, log-probabilities
          and the logits' gradient), "logps" (a reference model's log-probabilities),
          "clip" (global norms over many tensors, clipping, packing)
  rows, inp, out       linear layers: tokens, input and output features
  rows, cols           codec: the matrix
  pairs, longest, vocab, prompt   preference: pairs of sequences, the longest one
          a sequence may be, the vocabulary, the share of each that is prompt
  layers, d, ffn, kv, vocab, k    clip: the model whose parameters' gradients are
          clipped, and the workers
  dtype   of activations, logits or gradients, "f32" or "bf16"

Where `own` is false the operators are computed from elementary torch operations
in 32 bits, rounded once at the end."""
import math
import random

import torch

own = False

BETA, SMOOTH = 0.1, 0.05
MAX_NORM = 1.0
NORMS = (4.0, 0.5, 2.0, 0.9)     # the workers' gradient norms, about the clipping threshold
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # the magnitudes of a 4-bit element


def listed():
    return [
        # one token through an up projection of the 1.1B shape: latency and the weight's bytes
        {"name": "token 1.1b up", "op": "linear", "rows": 1, "inp": 2048, "out": 5632, "dtype": "bf16"},
        # thirteen sequences decoding together, the 7B shape
        {"name": "tokens 13 7b up", "op": "linear", "rows": 13, "inp": 4096, "out": 11008, "dtype": "bf16"},
        # a training batch through the head of GPT-2 small: odd rows, an odd vocabulary
        {"name": "head gpt2 1003 rows", "op": "linear", "rows": 1003, "inp": 768, "out": 50257, "dtype": "f32"},
        # a training batch through the 7B up projection: the matrix product itself
        {"name": "linear 7b up 4096", "op": "linear", "rows": 4096, "inp": 4096, "out": 11008, "dtype": "bf16"},
        # both gradients of the 1.1B up projection
        {"name": "grads 1.1b up 2048", "op": "linear_grad", "rows": 2048, "inp": 2048, "out": 5632, "dtype": "bf16"},
        # both gradients of a small odd layer with a short batch
        {"name": "grads odd 300", "op": "linear_grad", "rows": 300, "inp": 771, "out": 1030, "dtype": "f32"},
        # a pseudo-gradient of the GPT-2 embedding as a 4-bit payload, and what its receiver reads
        {"name": "codec gpt2 wte", "op": "codec", "rows": 50257, "cols": 768, "dtype": "f32"},
        # a single short pair: launches count
        {"name": "preference 1 pair", "op": "preference", "pairs": 1, "longest": 24, "vocab": 32000, "prompt": 0.5,
         "dtype": "bf16"},
        # a micro-batch of GPT-2 small: rows that start at odd addresses
        {"name": "preference gpt2", "op": "preference", "pairs": 4, "longest": 512, "vocab": 50257, "prompt": 0.3,
         "dtype": "f32"},
        # a micro-batch of the 1.1B model
        {"name": "preference 1.1b", "op": "preference", "pairs": 16, "longest": 1024, "vocab": 32000, "prompt": 0.4,
         "dtype": "bf16"},
        # four workers' gradients of a toy model: launches count
        {"name": "clip toy k4", "op": "clip", "layers": 3, "d": 97, "ffn": 260, "kv": 33, "vocab": 501, "k": 4,
         "dtype": "f32"},
        # two workers' bf16 gradients of the 1.1B model, packed for the optimiser
        {"name": "clip 1.1b k2", "op": "clip", "layers": 22, "d": 2048, "ffn": 5632, "kv": 256, "vocab": 32000, "k": 2,
         "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size spread over its logarithm: as drawn, or rounded down to a usual multiple."""
    n = _log(rng, lo, hi)
    m = rng.choice([1, 1, 2, 32, 128])
    n = n - n % m if n >= 2 * m and n - n % m >= lo else n
    return n if n != 3072 else n + 1


def draw(rng):
    """A case of the same ranges, sizes over their logarithm, odd ones among them."""
    op = rng.choice(["linear", "linear", "linear", "linear_grad", "linear_grad", "codec", "preference", "preference",
                     "logps", "clip", "clip"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op == "linear":
        rows = rng.choice([_log(rng, 1, 16), _size(rng, 1, 4096)])
        return {"op": op, "rows": rows, "inp": _size(rng, 200, 4096), "out": _size(rng, 200, 11008), "dtype": dtype}
    if op == "linear_grad":
        return {"op": op, "rows": _size(rng, 30, 2048), "inp": _size(rng, 200, 2048), "out": _size(rng, 200, 5632),
                "dtype": dtype}
    if op == "codec":
        return {"op": op, "rows": _size(rng, 1, 20000), "cols": _size(rng, 30, 1900), "dtype": dtype}
    if op in ("preference", "logps"):
        vocab, longest = _size(rng, 300, 50257), _size(rng, 8, 1024)
        most = 16 * 1024 * 32000 // (vocab * longest * (2 if dtype == "f32" else 1))
        return {"op": op, "pairs": rng.randint(1, max(1, min(16, most))), "longest": longest, "vocab": vocab,
                "prompt": round(rng.uniform(0.1, 0.7), 2), "dtype": dtype}
    k, d = rng.choice([1, 2, 3, 4]), _size(rng, 64, 1024)
    return {"op": op, "layers": rng.randint(1, 12), "d": d, "ffn": _size(rng, 2 * d, 4 * d),
            "kv": _size(rng, max(2, d // 8), d), "vocab": _size(rng, 500, 32000), "k": k, "dtype": dtype}


# ------------------------------------------------------------------- inputs --
def _gen(seed, role):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1_000_003 + role * 101) & 0x7FFF_FFFF_FFFF_FFFF)
    return g


def _normal(shape, std, seed, role, dtype=torch.float32):
    return torch.randn(shape, generator=_gen(seed, role), device="cuda").mul_(std).to(dtype)


def _tensors(c):
    """Element counts of the model's parameters, one after another."""
    d, ffn, kv, vocab = c["d"], c["ffn"], c["kv"], c["vocab"]
    layer = [d * d, kv * d, kv * d, d * d, ffn * d, ffn * d, d * ffn, d, d]
    return [vocab * d] + layer * c["layers"] + [d, vocab * d]


def _lengths(c):
    """(length, prompt tokens) of each sequence, the pairs' first ones, then their second ones: of the case alone."""
    r = random.Random(str(sorted((k, v) for k, v in c.items() if k != "name")))
    n = [r.randint(max(1, c["longest"] // 4), c["longest"]) for _ in range(2 * c["pairs"])]
    return [(t, int(t * c["prompt"] * r.uniform(0.5, 1.0))) for t in n]


def _pack(v):
    """The 4-bit form of v [rows, cols] as a program keeps it: codes [rows, 64 ceil(cols / 128)], two a byte, the first
    in the low half; scales [ceil(cols / 128), rows, 4], a power of two plus 127 for each 32 columns; and the values they stand for."""
    rows, cols = v.shape
    groups = -(-cols // 128)
    x = torch.nn.functional.pad(v.float(), (0, groups * 128 - cols)).view(rows, groups * 4, 32)
    e = torch.frexp(x.abs().amax(2, keepdim=True))[1].float() - 3
    e = torch.where(x.abs().amax(2, keepdim=True) > 0, e.clamp(-126, 127), torch.zeros_like(e))
    y = x * torch.exp2(-e)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = ((a / step).round() * step).clamp(max=6.0)
    code = torch.searchsorted(torch.tensor(GRID, device=v.device), a.contiguous()).to(torch.uint8)
    code = (code + 8 * torch.signbit(y).to(torch.uint8)).view(rows, groups * 64, 2)
    values = (torch.copysign(a, y) * torch.exp2(e)).view(rows, groups * 128)[:, :cols].contiguous()
    scales = (e + 127).to(torch.uint8).view(rows, groups, 4).transpose(0, 1).contiguous()
    return {"rows": rows, "cols": cols, "codes": (code[..., 0] + 16 * code[..., 1]).contiguous(), "scales": scales,
            "values": values}


def _room(rows, cols):
    """Buffers for the 4-bit form of a matrix."""
    groups = -(-cols // 128)
    return {"rows": rows, "cols": cols, "codes": torch.empty((rows, 64 * groups), dtype=torch.uint8, device="cuda"),
            "scales": torch.empty((groups, rows, 4), dtype=torch.uint8, device="cuda")}


def _prepare_linear(c, seed, s):
    rows, inp, out, dt = c["rows"], c["inp"], c["out"], DTYPES[c["dtype"]]
    s["x"] = _normal((rows, inp), 1.0, seed, 1, dt)
    w = _normal((out, inp), 0.02, seed, 2)
    if c["op"] == "linear":
        # the weight as a program keeps it after an optimiser step, for the framework and for the plain form
        s.update(w=_pack(w), xq=_room(rows, inp), y=torch.empty((rows, out), dtype=dt, device="cuda"))
        return
    s["dy"] = _normal((rows, out), 1e-2, seed, 3, dt)
    s.update(wt=_pack(w.t().contiguous()), dyq=_room(rows, out), dyt=_room(out, rows), xt=_room(inp, rows),
             dx=torch.empty((rows, inp), dtype=dt, device="cuda"), dw=torch.empty((out, inp), device="cuda"))


def _prepare_preference(c, seed, s):
    dt, vocab, lens = DTYPES[c["dtype"]], c["vocab"], _lengths(c)
    rows = sum(t for t, _ in lens)
    s["labels"] = torch.randint(0, vocab, (rows,), generator=_gen(seed, 1), device="cuda")
    s["logits"] = torch.empty((rows, vocab), dtype=dt, device="cuda")
    g = _gen(seed, 2)
    for a in range(0, rows, 4096):   # a model that knows its tokens: one to two nats each, as in language
        b = min(rows, a + 4096)
        x = torch.randn((b - a, vocab), generator=g, device="cuda").mul_(2.0)
        x[torch.arange(b - a, device="cuda"), s["labels"][a:b]] += math.log(vocab) + 1.0
        s["logits"][a:b] = x
    ends = [0]
    for t, _ in lens:
        ends.append(ends[-1] + t)
    s["offsets"] = torch.tensor(ends, dtype=torch.int64, device="cuda")
    # what the plain form adds up by: each row's sequence and its place in it
    s["seq"] = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor([t for t, _ in lens], device="cuda"))
    s["place"] = torch.arange(rows, device="cuda") - s["offsets"][s["seq"]]
    s["labels"][s["place"] < torch.tensor([p for _, p in lens], device="cuda")[s["seq"]]] = -100
    s["logps"] = torch.empty(len(lens), device="cuda")
    s["work"] = torch.empty(2 * rows + len(lens), device="cuda")
    if c["op"] == "preference":
        # the frozen reference model gives each sequence about what the policy does
        own_lp = torch.cat([_row_logps(s["logits"][a:a + 4096], s["labels"][a:a + 4096])[0] for a in range(0, rows, 4096)])
        s["ref"] = _by_sequence(s, own_lp) + _normal((len(lens),), 5.0, seed, 3)
        s["losses"] = torch.empty(c["pairs"], device="cuda")
        s["grads"] = torch.empty_like(s["logits"])


def _prepare_clip(c, seed, s):
    sizes, k, dt = _tensors(c), c["k"], DTYPES[c["dtype"]]
    n = sum(sizes)
    s["grads"] = torch.empty((k, n), dtype=dt, device="cuda")
    for w in range(k):
        s["grads"][w] = _normal((n,), NORMS[w % 4] / math.sqrt(n), seed, 1 + w, dt)
    s["packed"] = torch.empty((k, n), device="cuda")
    s["norms"] = torch.empty(k, device="cuda")
    if own:   # the handle over the gradients' tensors that a training program keeps between steps
        al = _framework()
        s["list"] = al.autoloco_grads_create(_context(), [list(g.split(sizes)) for g in s["grads"]], list(s["packed"]))


def prepare(case, seed):
    c = dict(case)
    s = {"case": c}
    if c["op"] in ("linear", "linear_grad"):
        _prepare_linear(c, seed, s)
    elif c["op"] == "codec":
        s["x"] = _normal((c["rows"], c["cols"]), 1e-3, seed, 1, DTYPES[c["dtype"]])   # a pseudo-gradient
        s.update(q=_room(c["rows"], c["cols"]), back=torch.empty((c["rows"], c["cols"]), device="cuda"))
    elif c["op"] == "clip":
        _prepare_clip(c, seed, s)
    else:
        _prepare_preference(c, seed, s)
    return s


# ---------------------------------------------------------- the framework's --
_ctx = None


def _framework():
    import paper_2609_36662_amd as al
    return al


def _context():
    global _ctx
    if _ctx is None:
        _ctx = _framework().autoloco_create(0)
    return _ctx


def _run_own(s):
    al, ctx, c = _framework(), _context(), s["case"]
    mx = lambda q: al.Mxfp4(q["rows"], q["cols"], q["codes"], q["scales"])  # noqa: E731
    if c["op"] == "linear":
        al.autoloco_mxfp4_linear(ctx, s["x"], mx(s["w"]), s["y"], mx(s["xq"]))
        return s["y"]
    if c["op"] == "linear_grad":
        dyq, dyt, xt = mx(s["dyq"]), mx(s["dyt"]), mx(s["xt"])
        al.autoloco_mxfp4_quantize(ctx, s["dy"], dyq, dyt)
        al.autoloco_mxfp4_quantize(ctx, s["x"], None, xt)
        al.autoloco_mxfp4_matmul(ctx, dyq, mx(s["wt"]), s["dx"])
        al.autoloco_mxfp4_matmul(ctx, dyt, xt, s["dw"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if c["op"] == "codec":
        q = mx(s["q"])
        al.autoloco_mxfp4_quantize(ctx, s["x"], q)
        al.autoloco_mxfp4_dequantize(ctx, q, s["back"])
        return s["back"]
    if c["op"] == "logps":
        al.autoloco_sequence_logps(ctx, s["logits"], s["labels"], s["offsets"], s["logps"], s["work"])
        return s["logps"]
    if c["op"] == "preference":
        al.autoloco_preference_loss(ctx, s["logits"], s["labels"], s["offsets"], s["ref"], s["losses"], s["logps"],
                                    s["work"], grads=s["grads"], beta=BETA, label_smoothing=SMOOTH,
                                    grad_scale=1.0 / c["pairs"])
        return {"losses": s["losses"], "logps": s["logps"], "grads": s["grads"]}
    al.autoloco_clip_grad_norm(ctx, s["list"], MAX_NORM, norms=s["norms"], stats=False)
    return {"grads": s["packed"], "norms": s["norms"]}


# ----------------------------------------------------------- the plain form --
def _values(v):
    """What the 4-bit form of v stands for: along each row 32 values share the power of two that brings the largest
    magnitude below 8, and each is rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code."""
    rows, cols = v.shape
    x = torch.nn.functional.pad(v.float(), (0, -cols % 32)).view(rows, -1, 32)
    e = torch.frexp(x.abs().amax(2, keepdim=True))[1] - 3
    y = torch.ldexp(x, -e)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = ((a / step).round() * step).clamp(max=6.0)
    return torch.ldexp(torch.copysign(a, y), e).view(rows, -1)[:, :cols]


def _row_logps(logits, labels):
    """log-probability of each row's label (0 where it is masked), exp(x - max) and its sum."""
    x = logits.float()
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    z = e.sum(1, keepdim=True)
    lab = x.gather(1, labels.clamp(min=0)[:, None]) - m - z.log()
    return torch.where(labels >= 0, lab[:, 0], 0.0), e, z


def _by_sequence(s, v):
    table = torch.zeros((s["offsets"].numel() - 1, s["case"]["longest"]), dtype=v.dtype, device=v.device)
    table[s["seq"], s["place"]] = v
    return table.sum(1)


def _run_plain(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    if c["op"] == "linear":
        return (_values(s["x"]) @ s["w"]["values"].t()).to(dt)
    if c["op"] == "linear_grad":
        return {"dx": (_values(s["dy"]) @ s["wt"]["values"].t()).to(dt),
                "dw": _values(s["dy"].t()) @ _values(s["x"].t()).t()}
    if c["op"] == "codec":
        return _values(s["x"]).contiguous()
    if c["op"] == "clip":
        g = s["grads"].float()
        norms = g.square().sum(1).sqrt()
        return {"grads": g * (MAX_NORM / (norms + 1e-6)).clamp(max=1.0)[:, None], "norms": norms}
    lp, e, z = _row_logps(s["logits"], s["labels"])
    logps = _by_sequence(s, lp)
    if c["op"] == "logps":
        return logps
    p = c["pairs"]
    margin = BETA * ((logps - s["ref"])[:p] - (logps - s["ref"])[p:])
    soft = (-margin.abs()).exp().log1p()
    losses = (1 - SMOOTH) * (soft - margin.clamp(max=0.0)) + SMOOTH * (soft + margin.clamp(min=0.0))
    slope = BETA / p * (1 / (1 + (-margin).exp()) - (1 - SMOOTH))   # of the mean loss, by a chosen sequence's log-probability
    per_row = torch.where(s["labels"] >= 0, torch.cat([slope, -slope])[s["seq"]], 0.0)
    grads = e.mul_(-(per_row / z[:, 0])[:, None])
    grads[torch.arange(grads.shape[0], device="cuda"), s["labels"].clamp(min=0)] += per_row
    return {"losses": losses, "logps": logps, "grads": grads.to(dt)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# -------------------------------------------------------------------- work --
def work(case):
    """Bytes and operations of one pass: inputs read once, outputs written once (a 4-bit matrix is 17 bytes for 32
    values; rows of logits whose label is masked are not read)."""
    c = case
    b = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "linear":
        r, i, o = c["rows"], c["inp"], c["out"]
        return {"bytes": r * i * b + o * i * 17 / 32 + r * o * b, "flops": 2.0 * r * i * o}
    if c["op"] == "linear_grad":
        r, i, o = c["rows"], c["inp"], c["out"]
        return {"bytes": r * i * b + r * o * b + o * i * 17 / 32 + r * i * b + o * i * 4, "flops": 4.0 * r * i * o}
    if c["op"] == "codec":
        return {"bytes": c["rows"] * c["cols"] * (b + 4.0), "flops": 0.0}
    if c["op"] == "clip":
        n = sum(_tensors(c)) * c["k"]
        return {"bytes": n * (b + 4.0), "flops": 3.0 * n}
    lens = _lengths(c)
    rows, live = sum(t for t, _ in lens), sum(t - p for t, p in lens)
    reads, writes = live * c["vocab"] * b, rows * c["vocab"] * b if c["op"] == "preference" else 0
    return {"bytes": float(reads + writes + rows * 8), "flops": (4.0 if c["op"] == "logps" else 7.0) * live * c["vocab"]}


# ------------------------------------------------------------------- exact --
def _exact_values(v):
    """The 4-bit form's values in 64 bits, from the midpoints between neighbouring magnitudes."""
    rows, cols = v.shape
    x = torch.nn.functional.pad(v.double(), (0, -cols % 32)).view(rows, -1, 32)
    scale = torch.exp2(torch.floor(torch.log2(x.abs().amax(2, keepdim=True).clamp(min=2.0 ** -120))) - 2)
    a = x.abs() / scale
    at = torch.zeros(a.shape, dtype=torch.int64, device=a.device)
    for i in range(7):
        mid = (GRID[i] + GRID[i + 1]) / 2
        at += (a >= mid) if i % 2 else (a > mid)
    out = torch.tensor(GRID, dtype=torch.float64, device=a.device)[at] * scale * x.sign()
    return out.reshape(rows, -1)[:, :cols].contiguous()


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "linear":
        return _exact_values(s["x"]) @ s["w"]["values"].double().t().contiguous()
    if c["op"] == "linear_grad":
        dyt, xt = _exact_values(s["dy"].t()), _exact_values(s["x"].t())
        return {"dx": _exact_values(s["dy"]) @ s["wt"]["values"].double().t().contiguous(), "dw": dyt @ xt.t().contiguous()}
    if c["op"] == "codec":
        return _exact_values(s["x"])
    if c["op"] == "clip":
        norms = torch.stack([g.double().pow(2).sum() for g in s["grads"]]).sqrt()
        return {"grads": torch.stack([g.double() * min(1.0, MAX_NORM / (float(n) + 1e-6)) for g, n in zip(s["grads"], norms)]),
                "norms": norms}
    rows, p = s["labels"].numel(), c["pairs"]
    lse = torch.empty(rows, dtype=torch.float64, device="cuda")
    for a in range(0, rows, 2048):
        lse[a:a + 2048] = torch.logsumexp(s["logits"][a:a + 2048].double(), 1)
    at = torch.arange(rows, device="cuda")
    lp = s["logits"][at, s["labels"].clamp(min=0)].double() - lse
    ends = s["offsets"].tolist()
    live = s["labels"] >= 0
    logps = torch.stack([lp[a:b][live[a:b]].sum() for a, b in zip(ends, ends[1:])])
    if c["op"] == "logps":
        return logps
    ratio = logps - s["ref"].double()
    margin = BETA * (ratio[:p] - ratio[p:])
    log_sig = torch.nn.functional.logsigmoid
    losses = -(1 - SMOOTH) * log_sig(margin) - SMOOTH * log_sig(-margin)
    slope = BETA / p * (torch.sigmoid(margin) - (1 - SMOOTH))
    grads = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    for q in range(2 * p):
        a, b = ends[q], ends[q + 1]
        keep = at[a:b][live[a:b]]
        if keep.numel():
            g = -(s["logits"][keep].double() - lse[keep, None]).exp()
            g[torch.arange(keep.numel(), device="cuda"), s["labels"][keep]] += 1.0
            grads[keep] = g * (slope[q] if q < p else -slope[q - p])
    return {"losses": losses, "logps": logps, "grads": grads}
