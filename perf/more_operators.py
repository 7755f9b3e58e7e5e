"""Operators of a language module's training step as measurable cases: each is one pass a training or an
evaluation step makes of them.

  ce_fwd   loss of a linear layer with softmax cross entropy over a vocabulary: logits z = x table^T, for
           every token lse(z) - (1 - s) z[target] - s mean(z) with label smoothing s, and their mean over the
           tokens whose target lies in the vocabulary (the others count as nothing)
  ce_grad  the same with the gradients of x and of the table
  grouped  products of rows sorted by expert with their expert's matrix w [groups, k, n]: `fwd` y = x w,
           `dgrad` dx = dy w^T, `wgrad` dw = x^T dy for every expert
  dropout  y = r + x * keep / (1 - p) (or without r, as for a gradient); keep from a counter-based generator

Dropout's random bits are those of Philox4x32-10 (Salmon, Moraes, Dror and Shaw, 2011): a block of eight
consecutive elements takes the four words at the counter (block, offset + site), both of 64 bits, low words
first, under the key seed; element 2i of the block has the low half of word i, element 2i + 1 the high half.
An element is kept where its 16 bits are at least p * 65536 rounded.
"""
import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
CUS = 256
IGNORED = -100


# ------------------------------------------------------------------------------- the cases
def _ce(op, T, h, V, ignored=0.0, smoothing=0.0, dtype="bf16", **kw):
    return dict(op=op, T=T, h=h, V=V, ignored=ignored, smoothing=smoothing, dtype=dtype, **kw)


def _grouped(form, T, groups, k, n, skew=1.0, dtype="bf16", **kw):
    return dict(op="grouped", form=form, T=T, groups=groups, k=k, n=n, skew=skew, dtype=dtype, **kw)


def _dropout(n, p, residual, dtype="bf16", **kw):
    return dict(op="dropout", n=n, p=p, residual=residual, dtype=dtype, **kw)


def listed():
    return [
        # one token scored by the 7B-shaped decoder: the table is read once
        _ce("ce_fwd", 1, 4096, 32000, name="ce_token"),
        # validation loss of the small language model on a ragged batch, odd vocabulary, a fifth of it image tokens
        _ce("ce_fwd", 3 * 1021, 2048, 50021, ignored=0.2, name="ce_eval_ragged"),
        # a training step of the tiny fp32 workload's decoder, with smoothed targets
        _ce("ce_grad", 2 * 128, 128, 1000, ignored=0.125, smoothing=0.1, dtype="f32", name="ce_grad_tiny_f32"),
        # transcripts of an audio sample: 1499 tokens, odd vocabulary, smoothed targets
        _ce("ce_grad", 1499, 1280, 51001, smoothing=0.1, name="ce_grad_ragged"),
        # the 7B-shaped decoder, 4 x 4096 tokens of which a quarter are images or prompts, a large vocabulary
        _ce("ce_grad", 4 * 4096, 4096, 128000, ignored=0.25, name="ce_grad_llm"),
        # a serving step: 24 sequences, two experts each, of eight experts: their matrices are read once
        _grouped("fwd", 48, 8, 4096, 1408, name="grouped_decode"),
        # gate and up products of 16 experts, 8 x 1024 tokens to two experts each
        _grouped("fwd", 2 * 8 * 1024, 16, 2048, 5632, name="grouped_fwd_llm"),
        # gradients of the experts' inputs, in fp32, sizes that no tile divides
        _grouped("dgrad", 2 * 1499, 12, 640, 1000, dtype="f32", name="grouped_dgrad_f32"),
        # the weight gradients of many small experts, some without a token
        _grouped("wgrad", 2 * 8 * 4096, 64, 2048, 1408, skew=1.5, name="grouped_wgrad_llm"),
        # a gradient of the tiny fp32 workload, one row short: nothing but latency
        _dropout(255 * 129, 0.25, 0, dtype="f32", name="dropout_tiny_f32"),
        # the residual stream of the 7B-shaped decoder, 4 x 4096 tokens
        _dropout(4 * 4096 * 4096, 0.1, 1, name="dropout_add_llm"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("ce_fwd", "ce_grad", "ce_grad", "grouped", "grouped", "grouped", "dropout"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if op == "dropout":
        return _dropout(_log(rng, 1, 1 << 26), rng.choice((0.0, 0.05, 0.1, 0.3, 0.5, 0.9)), rng.randint(0, 1), dtype)
    if op == "grouped":
        k, n = 8 * _log(rng, 8, 512), 8 * _log(rng, 8, 704)
        groups = _log(rng, 1, 128)
        while groups * k * n > 1 << 28:
            groups = (groups + 1) // 2
        most = (1 << 38) if dtype == "bf16" else (1 << 34)      # multiplications
        return _grouped(rng.choice(("fwd", "dgrad", "wgrad")), _log(rng, 1, max(2, min(65536, most // (k * n)))), groups, k, n, rng.choice((0.0, 1.0, 2.0)), dtype)
    h, V = 8 * _log(rng, 8, 512 if dtype == "bf16" else 160), _log(rng, 2, 131072)
    most = (1 << 42) if dtype == "bf16" else (1 << 35)
    case = _ce(op, _log(rng, 1, max(2, min(16384, most // (h * V)))), h, V, rng.choice((0.0, 0.0, 0.25, 0.9)), rng.choice((0.0, 0.0, 0.1)), dtype)
    return case if _counted(case) else {**case, "ignored": 0.0}


def _counted(case):
    """Tokens that the loss counts: of every stretch of 256, a share at its start is ignored."""
    T, skip = case["T"], _skip(case)
    return T // 256 * (256 - skip) + max(0, T % 256 - skip)


def _skip(case):
    return int(round(256 * case["ignored"]))


def work(case):
    es = SIZE[case["dtype"]]
    op = case["op"]
    if op in ("ce_fwd", "ce_grad"):      # of x only the counted tokens' rows are needed
        T, h, V, C = case["T"], case["h"], case["V"], _counted(case)
        read = (C * h + V * h) * es + 4 * T
        if op == "ce_fwd":
            return {"bytes": read + 4 * T, "flops": 2 * C * h * V}
        return {"bytes": read + 4 * T + (T * h + V * h) * es, "flops": 6 * C * h * V}
    if op == "grouped":
        T, k, n, sizes = case["T"], case["k"], case["n"], _sizes(case)
        used = len(sizes) if case["form"] == "wgrad" else sum(s > 0 for s in sizes)      # an expert without a token has a gradient, of zeros
        return {"bytes": (T * k + T * n + used * k * n) * es + 4 * (len(sizes) + 1), "flops": 2 * T * k * n}
    n = case["n"]
    return {"bytes": (3 if case["residual"] else 2) * n * es, "flops": 30 * n}


# ------------------------------------------------------------------------------- the inputs
def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(DT[dtype])


def _sizes(case):
    """Rows of every expert: popular and unpopular ones in no order, and every fifth of many has none where the load is skewed."""
    E, T = case["groups"], case["T"]
    weight = [math.exp(case["skew"] * math.sin(2.399963 * (e + 1))) for e in range(E)]
    if E >= 5 and case["skew"] > 1:
        weight = [0.0 if e % 5 == 3 else w for e, w in enumerate(weight)]
    total, ends, run = sum(weight), [], 0.0
    for w in weight:
        run += w
        ends.append(int(round(T * run / total)))
    ends[-1] = T if weight[-1] else ends[-1]
    return [b - a for a, b in zip([0] + ends, ends)]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt = case["op"], case["dtype"]
    if op == "dropout":
        n = case["n"]
        s = {"x": _normal(g, (n,), dt), "rng": torch.randint(0, 1 << 62, (2,), generator=g, device="cuda", dtype=torch.int64)}
        if case["residual"]:
            s["r"] = _normal(g, (n,), dt, 4.0)
        return s
    if op == "grouped":
        T, E, k, n = case["T"], case["groups"], case["k"], case["n"]
        sizes = _sizes(case)
        s = {"offsets": torch.tensor([0] + list(np.cumsum(sizes)), dtype=torch.int32, device="cuda")}
        if case["form"] != "dgrad":
            s["x"] = _normal(g, (T, k), dt)
        if case["form"] != "fwd":
            s["dy"] = _normal(g, (T, n), dt, 1e-3)
        if case["form"] != "wgrad":
            s["w"] = _normal(g, (E, k, n), dt, k ** -0.5)
        return s
    # a trained model's logits: most of a few units, the targets' from ordinary to far ahead of the rest
    T, h, V = case["T"], case["h"], case["V"]
    table = _normal(g, (V, h), dt, 2.0 * h ** -0.5)
    target = (V * torch.rand((T,), generator=g, device="cuda") ** 3).long().clamp(max=V - 1)
    sure = 3.0 * torch.rand((T, 1), generator=g, device="cuda")
    x = (torch.randn((T, h), generator=g, device="cuda") + sure * table[target].float()).to(DT[dt])
    skipped = torch.arange(T, device="cuda") % 256 < _skip(case)
    return {"x": x, "table": table, "target": torch.where(skipped, IGNORED, target).to(torch.int32)}


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if case["op"] == "grouped":
        state["sizes"] = _sizes(case)      # a router that ran on the host knows them
    if own:        # what a program that calls the framework keeps: scratch memory and buffers for what a call writes
        state["kept"] = _kept(case)
    return state


# ------------------------------------------------------------------------------- plain forms
def _plain_ce(case, s):
    x, table, target = s["x"].float(), s["table"].float(), s["target"].long()
    V, smooth = case["V"], case["smoothing"]
    counts = (target >= 0) & (target < V)
    D = counts.sum().clamp(min=1).float()
    at = target.clamp(0, V - 1).unsqueeze(1)
    z = x @ table.t()
    top = z.amax(1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(1, keepdim=True)
    losses = (top + torch.log(total)).squeeze(1) - (1.0 - smooth) * z.gather(1, at).squeeze(1)
    if smooth:
        losses = losses - smooth * z.mean(1)
    losses = torch.where(counts, losses, 0.0)
    out = {"loss": (losses.double().sum() / D).float(), "losses": losses}
    del z
    if case["op"] == "ce_fwd":
        return out
    p /= total
    p.scatter_add_(1, at, torch.full_like(p[:, :1], smooth - 1.0))
    if smooth:
        p -= smooth / V
    p *= counts.unsqueeze(1) / D
    out["dx"] = (p @ table).to(s["x"].dtype)
    out["dtable"] = (p.t() @ x).to(s["x"].dtype)
    return out


def _plain_grouped(case, s):
    out, form = [], case["form"]
    row = 0
    for e, size in enumerate(s["sizes"]):
        part = slice(row, row + size)
        row += size
        if form == "fwd":
            out.append(s["x"][part].float() @ s["w"][e].float())
        elif form == "dgrad":
            out.append(s["dy"][part].float() @ s["w"][e].float().t())
        else:
            out.append((s["x"][part].float().t() @ s["dy"][part].float()).unsqueeze(0))
    return {"y": torch.cat(out).to(DT[case["dtype"]])}


_M32 = 0xFFFFFFFF


def _philox(c, k):
    """Ten rounds on lists of four counter words and two key words, whole numbers of 32 bits in 64; a product's 64 bits wrap into the sign."""
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & _M32) ^ c[1] ^ k[0], b & _M32, ((a >> 32) & _M32) ^ c[3] ^ k[1], a & _M32]
        k = [(k[0] + 0x9E3779B9) & _M32, (k[1] + 0xBB67AE85) & _M32]
    return c


SITE = 5      # which of a program's dropouts this is


def _plain_dropout(case, s):
    n, seed, turn = case["n"], s["rng"][0], s["rng"][1] + SITE
    block = torch.arange((n + 7) // 8, device="cuda")
    words = _philox([block & _M32, block >> 32, turn & _M32, (turn >> 32) & _M32], [seed & _M32, (seed >> 32) & _M32])
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=1).reshape(-1)[:n]
    drop = int(round(case["p"] * 65536))
    y = torch.where(halves >= drop, s["x"].float() * (65536.0 / (65536 - drop)), 0.0)
    if case["residual"]:
        y = s["r"].float() + y
    return {"y": y.to(s["x"].dtype)}


def run(state):
    case = state["case"]
    if own:
        return _call(case, state, state["kept"])
    op = case["op"]
    if op == "dropout":
        return _plain_dropout(case, state)
    return _plain_grouped(case, state) if op == "grouped" else _plain_ce(case, state)


# ------------------------------------------------------------------------------- the framework's calls
def _binding():
    from paper_2605_18710_amd import binding
    return binding


def _kept(case):
    mb = _binding()
    op, dt = case["op"], DT[case["dtype"]]

    def empty(*shape, dtype=dt):
        return torch.empty(shape, device="cuda", dtype=dtype)

    if op == "dropout":
        return {"y": empty(case["n"])}
    if op == "grouped":
        T, E, k, n = case["T"], case["groups"], case["k"], case["n"]
        return {"y": {"fwd": lambda: empty(T, n), "dgrad": lambda: empty(T, k), "wgrad": lambda: empty(E, k, n)}[case["form"]]()}
    T, h, V = case["T"], case["h"], case["V"]
    kept = {"loss": empty(dtype=torch.float32), "losses": empty(T, dtype=torch.float32)}
    if op == "ce_fwd":
        size = mb.linear_ce_fwd_scratch_bytes(case["dtype"], T, h, V)
    else:
        size = mb.linear_ce_grad_scratch_bytes(case["dtype"], T, h, V)
        kept.update(dx=empty(T, h), dtable=empty(V, h))
    kept["scratch"] = empty(size, dtype=torch.uint8)
    return kept


def _call(case, s, kept):
    mb = _binding()
    op, dt = case["op"], case["dtype"]
    stream = torch.cuda.current_stream().cuda_stream
    if op == "dropout":
        mb.op_dropout(stream, CUS, dt, case["n"], case["p"], SITE, s["rng"], s["x"], s.get("r"), kept["y"])
        return {"y": kept["y"]}
    if op == "grouped":
        sizes = (case["T"], case["groups"], case["k"], case["n"], s["offsets"])
        if case["form"] == "fwd":
            mb.op_grouped_linear_fwd(stream, CUS, dt, *sizes, s["x"], s["w"], kept["y"])
        elif case["form"] == "dgrad":
            mb.op_grouped_linear_dgrad(stream, CUS, dt, *sizes, s["dy"], s["w"], kept["y"])
        else:
            mb.op_grouped_linear_wgrad(stream, CUS, dt, *sizes, s["x"], s["dy"], kept["y"])
        return {"y": kept["y"]}
    sizes = (case["T"], case["h"], case["V"], case["smoothing"], 0.0)      # 0: the mean over the counted tokens
    if op == "ce_fwd":
        mb.op_linear_ce_fwd(stream, CUS, dt, *sizes, s["target"], s["x"], s["table"], kept["loss"], kept["losses"], kept["scratch"])
        return {"loss": kept["loss"], "losses": kept["losses"]}
    mb.op_linear_ce_grad(stream, CUS, dt, *sizes, s["target"], s["x"], s["table"], kept["loss"], kept["losses"], kept["dx"], kept["dtable"], kept["scratch"])
    return {"loss": kept["loss"], "losses": kept["losses"], "dx": kept["dx"], "dtable": kept["dtable"]}


# ------------------------------------------------------------------------------- in 64 bits
def _exact_ce(case, i):
    """Gradients by automatic differentiation through the definition, the counted tokens alone, a piece of them at a time."""
    T, V, smooth = case["T"], case["V"], case["smoothing"]
    grad = case["op"] == "ce_grad"
    rows = torch.nonzero((i["target"] >= 0) & (i["target"] < V)).squeeze(1)
    table = i["table"].double().requires_grad_(grad)
    losses = torch.zeros(T, device="cuda", dtype=torch.float64)
    dx = torch.zeros_like(i["x"], dtype=torch.float64) if grad else None
    step = max(1, (1 << 29) // V)
    for r in rows.split(step):
        x = i["x"][r].double().requires_grad_(grad)
        with torch.set_grad_enabled(grad):
            logp = torch.log_softmax(x @ table.t(), dim=1)
            q = logp[torch.arange(len(r), device="cuda"), i["target"][r].long()]
            each = -(1.0 - smooth) * q - (smooth / V) * logp.sum(1) if smooth else -q
        losses[r] = each.detach()
        if grad:
            (each.sum() / len(rows)).backward()
            dx[r] = x.grad
    out = {"loss": losses.sum() / max(1, len(rows)), "losses": losses}
    if grad:
        out.update(dx=dx, dtable=table.grad if table.grad is not None else torch.zeros_like(table))
    return {key: v.detach() for key, v in out.items()}


def _exact_grouped(case, i):
    ends = i["offsets"].tolist()
    form = case["form"]
    first = i["dy"] if form == "dgrad" else i["x"]
    if form == "wgrad":
        y = torch.zeros((case["groups"], case["k"], case["n"]), device="cuda", dtype=torch.float64)
    else:
        y = torch.zeros((case["T"], case["n"] if form == "fwd" else case["k"]), device="cuda", dtype=torch.float64)
    for e in range(case["groups"]):
        a, b = ends[e], ends[e + 1]
        if a == b:
            continue
        rows = first[a:b].double()
        if form == "wgrad":
            y[e] = torch.mm(rows.t().contiguous(), i["dy"][a:b].double())
        else:
            w = i["w"][e].double()
            y[a:b] = torch.mm(rows, w if form == "fwd" else w.t().contiguous())
    return {"y": y}


def _exact_dropout(case, i):
    """The generator over unsigned numbers on the host; products of 32 bits by 64-bit unsigned ones."""
    n = case["n"]
    seed, offset = (int(v) for v in i["rng"].cpu())
    turn = (offset + SITE) % (1 << 64)
    u = np.uint64
    low, half = u(0xFFFFFFFF), u(32)
    x0 = np.arange((n + 7) // 8, dtype=np.uint64)
    x1, x0 = x0 >> half, x0 & low
    x2, x3 = np.full_like(x0, turn & 0xFFFFFFFF), np.full_like(x0, turn >> 32)
    key = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        p, q = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (q >> half) ^ x1 ^ u(key[0]), q & low, (p >> half) ^ x3 ^ u(key[1]), p & low
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    bits = np.stack([w.astype(np.uint32) for w in (x0, x1, x2, x3)], axis=1).astype("<u4").view("<u2").reshape(-1)[:n]
    drop = int(round(case["p"] * 65536))
    keep = torch.from_numpy(bits >= drop).cuda()
    y = i["x"].double() * keep / (1 - drop / 65536)
    return {"y": i["r"].double() + y if case["residual"] else y}


def exact(case, seed):
    i = _inputs(case, seed)
    if case["op"] == "dropout":
        return _exact_dropout(case, i)
    return _exact_grouped(case, i) if case["op"] == "grouped" else _exact_ce(case, i)
