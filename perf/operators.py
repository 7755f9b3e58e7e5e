"""Operators around a layer's products as measurable cases: each is one pass a training step or a
serving loop makes of them.

  rotate      rotary positions with several axes (time, height, width) on the q and k parts of
              packed rows [q (H heads) | k (Hkv heads) | v (Hkv heads)], forward or turned back
  qk_fwd      norm of every query and key head, then the rotation, in one pass
  qk_bwd      its backward pass: the gradient of the rows and of the norms' gains (and shifts)
  save_load   an activation checkpoint: packed to 8 bits in blocks of 32, and unpacked
  mlp         activation of an MLP that keeps its input in 8 bits, and its backward pass from
              there, which forms the activation's output again
  wgrad       weight gradient of a linear layer whose input was kept in 8 bits

Pair i of a head of d elements is elements (2i, 2i+1) (`adjacent`) or (i, i + d/2) (`halves`); it
turns by position[axis of i] * frequency of i.  `order` says how pairs are dealt to axes with
`sections` pairs each: `split`, runs of pairs in the order of the axes, pair i at base^(-2i/d);
`own`, the same runs, each with a spectrum of its own, pair j of s at base^(-j/s); `dealt`, one pair
to each axis in turn while it has room, pair i at base^(-2i/d).  Pairs past the sections stay.

A block of 32 consecutive elements in 8 bits has one exponent e, the smallest (from -127 on) with
max |x| <= 127.5 * 2^e, kept as the byte e + 127, and the whole numbers nearest to x / 2^e (ties to
even, at most 127 in size).  A block with a NaN or an infinity has the byte 255 and is NaN.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
CUS = 256


# ------------------------------------------------------------------------------- the cases
def _heads(op, T, H, Hkv, d, sections, order, pairing="halves", norm="none", dtype="bf16", base=1e6, **kw):
    return dict(op=op, T=T, H=H, Hkv=Hkv, d=d, axes=len(sections), sections=",".join(map(str, sections)), order=order, pairing=pairing, norm=norm,
                dtype=dtype, base=float(base), eps=1e-6, **kw)


def listed():
    return [
        # one token of a decoder that generates behind images: nothing but latency
        _heads("rotate", 1, 16, 4, 128, (24, 20, 20), "split", name="rotate_token", back=0),
        # gradients of a video encoder's q and k, 64 frames of 576 patches: each axis with a spectrum of its own
        _heads("rotate", 64 * 576, 16, 16, 64, (8, 12, 12), "own", "adjacent", base=1e4, name="rotate_back_video", back=1),
        # a serving step of 24 sequences with grouped key/value heads
        _heads("qk_fwd", 24, 16, 4, 128, (24, 20, 20), "dealt", norm="rmsnorm", name="qk_norm_decode"),
        # ViT-B queries and keys, 8 x 196 patches, LayerNorm, fp32
        _heads("qk_fwd", 8 * 196, 12, 12, 64, (16, 16), "own", "adjacent", norm="layernorm", dtype="f32", base=1e2, name="qk_norm_vit_f32"),
        # the 7B-shaped decoder, 8 x 4096 tokens of text and images, with eight key/value heads
        _heads("qk_fwd", 8 * 4096, 32, 8, 128, (24, 20, 20), "dealt", norm="rmsnorm", name="qk_norm_llm"),
        # audio encoder, 8 x 1500 frames, one axis (time), fp32
        _heads("qk_bwd", 8 * 1500, 20, 20, 64, (32,), "split", norm="layernorm", dtype="f32", base=1e4, name="qk_norm_back_audio_f32"),
        _heads("qk_bwd", 8 * 4096, 32, 8, 128, (24, 20, 20), "dealt", norm="rmsnorm", name="qk_norm_back_llm"),
        # a residual stream whose size is no multiple of a block
        dict(op="save_load", n=7 * 1499 * 1285, dtype="bf16", name="save_load_ragged"),
        # ViT-L MLP, 16 x 576 patches, GELU
        dict(op="mlp", T=16 * 576, f=4096, act="gelu", dtype="bf16", name="mlp_gelu_vit"),
        # MLP of the 7B-shaped decoder, 4 x 4096 tokens, SwiGLU: gate and up are half of what a layer keeps
        dict(op="mlp", T=4 * 4096, f=11008, act="swiglu", dtype="bf16", name="mlp_swiglu_llm"),
        # audio encoder, one sample, attention output projection with its bias
        dict(op="wgrad", T=1500, k=1280, n=1280, bias=1, dtype="bf16", name="wgrad_audio"),
        dict(op="wgrad", T=4 * 4096, k=4096, n=4096, bias=0, dtype="bf16", name="wgrad_llm"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_heads(rng, op):
    dtype = rng.choice(("bf16", "bf16", "f32"))
    d = rng.choice((32, 40, 64, 72, 80, 96, 128, 128, 256))
    Hkv = _log(rng, 1, 16)
    H = Hkv * rng.choice((1, 1, 2, 4, 5, 8))
    T = _log(rng, 1, max(2, (32768 * 6144 * 2) // ((H + 2 * Hkv) * d * SIZE[dtype] * 2)))
    axes, order = rng.randint(1, 3), rng.choice(("split", "own", "dealt"))
    left, sections = d // 2, []
    for a in range(axes):
        s = left // (axes - a) if rng.random() < 0.7 else rng.randint(1, max(1, left // (axes - a)))
        sections.append(s)
        left -= s
    more = dict(back=rng.randint(0, 1)) if op == "rotate" else {}
    norm = "none" if op == "rotate" else rng.choice(("rmsnorm", "rmsnorm", "layernorm"))
    return _heads(op, T, H, Hkv, d, tuple(sections), order, rng.choice(("adjacent", "halves")), norm, dtype, rng.choice((1e2, 1e4, 1e6)), **more)


def draw(rng):
    op = rng.choice(("rotate", "qk_fwd", "qk_bwd", "qk_bwd", "save_load", "mlp", "mlp", "wgrad"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op in ("rotate", "qk_fwd", "qk_bwd"):
        return _draw_heads(rng, op)
    if op == "save_load":
        return dict(op=op, n=_log(rng, 1, 1 << 27), dtype=dtype)
    if op == "mlp":
        f = 8 * _log(rng, 8, 2048)
        return dict(op=op, T=_log(rng, 1, max(2, (1 << 26) // f)), f=f, act=rng.choice(("gelu", "swiglu", "swiglu", "gelu_tanh")), dtype=dtype)
    k, n = 8 * _log(rng, 8, 640), 8 * _log(rng, 8, 640)
    most = (1 << 38) if dtype == "bf16" else (1 << 34)      # multiplications
    return dict(op=op, T=_log(rng, 1, max(2, min(32768, most // (k * n)))), k=k, n=n, bias=rng.randint(0, 1), dtype=dtype)


def work(case):
    es = SIZE[case["dtype"]]
    op = case["op"]
    if op in ("rotate", "qk_fwd", "qk_bwd"):
        T, d = case["T"], case["d"]
        qk, row = (case["H"] + case["Hkv"]) * d, (case["H"] + 2 * case["Hkv"]) * d
        ids = 4 * case["axes"] * T
        if op == "rotate":
            return {"bytes": 2 * T * row * es + ids, "flops": 3 * T * qk}
        if op == "qk_fwd":
            return {"bytes": 2 * T * row * es + ids, "flops": 7 * T * qk}
        return {"bytes": T * (2 * row + qk) * es + ids, "flops": 18 * T * qk}
    if op == "save_load":
        n = case["n"]
        return {"bytes": n * 2 * es + 2 * (n + n // 32), "flops": 4 * n}
    if op == "mlp":      # the checkpoint is written by the forward pass and read by the backward pass
        m = case["T"] * case["f"]
        z = 2 * m if case["act"] == "swiglu" else m
        return {"bytes": (2 * z + 3 * m) * es + 2 * (z + z // 32), "flops": 40 * m}
    T, k, n = case["T"], case["k"], case["n"]
    return {"bytes": T * k + T * k // 32 + (T * n + k * n + (n if case["bias"] else 0)) * es, "flops": 2 * T * k * n}


# ------------------------------------------------------------------------------- the inputs
def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(DT[dtype])


def _activations(g, T, width, dtype):
    """Activations: a few channels far larger than the rest, and the padding behind the last sequence is zero."""
    x = torch.randn((T, width), generator=g, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.8 * torch.randn((width,), generator=g, device="cuda", dtype=torch.float32))
    if T > 8:
        x[T - T // 16:] = 0
    return x.to(DT[dtype])


def _positions(g, T, axes):
    """Text and images in turn: 64 tokens of text, on all axes alike, then a grid of up to 16 x 16; frames follow each other in time."""
    t = torch.arange(T, device="cuda", dtype=torch.int64)
    start = torch.randint(0, 100000, (1,), generator=g, device="cuda")
    within, turn = t % 320, t // 320
    image = within >= 64
    first = start + 80 * turn
    cell = (within - 64).clamp(min=0)
    grid = torch.stack((first + 64, first + 64 + cell // 16, first + 64 + cell % 16))
    pos = torch.where(image, grid, first + within)
    return (pos[:axes] if axes > 1 else start + t.unsqueeze(0)).to(torch.int32).contiguous()


def _power(e):
    """2^e in 64 bits, exactly: its exponent's bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _pack(x):
    """Blocks of 32 along the flat elements: whole numbers (int8) and exponent bytes (uint8)."""
    n = x.numel()
    blocks = torch.nn.functional.pad(x.reshape(-1), (0, -n % 32)).reshape(-1, 32).float()
    top = blocks.abs().amax(1)
    mantissa, exponent = torch.frexp(top.double() / 127.5)
    e = torch.where(mantissa == 0.5, exponent - 1, exponent)
    e = torch.where(top == 0, -127, e).clamp(min=-127)
    q = torch.round(blocks.double() * _power(-e).unsqueeze(1)).clamp(-127, 127)
    bad = ~torch.isfinite(top)
    q = torch.where(bad.unsqueeze(1), 0.0, q).to(torch.int8)
    return q.reshape(-1)[:n].contiguous(), torch.where(bad, 255, e + 127).to(torch.uint8)


def _unpack(q, scale):
    """The values that packed numbers stand for, in 32 bits."""
    n = q.numel()
    blocks = torch.nn.functional.pad(q, (0, -n % 32)).reshape(-1, 32)
    v = blocks.double() * _power(scale.long() - 127).unsqueeze(1)
    v = torch.where((scale == 255).unsqueeze(1), math.nan, v)
    return v.reshape(-1)[:n].float()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt = case["op"], case["dtype"]
    if op in ("rotate", "qk_fwd", "qk_bwd"):
        T, d = case["T"], case["d"]
        row = (case["H"] + 2 * case["Hkv"]) * d
        x = {"x": _normal(g, (T, row), dt), "pos": _positions(g, T, case["axes"])}
        if op != "rotate":
            for part in ("q", "k"):
                x["gain_" + part] = (1 + 0.3 * torch.randn((d,), generator=g, device="cuda")).to(DT[dt])
                x["shift_" + part] = _normal(g, (d,), dt, 0.1)
        if op == "qk_bwd":
            x["dy"] = _normal(g, (T, row), dt, 1e-3)
        return x
    if op == "save_load":
        return {"x": _activations(g, 1, case["n"], dt).reshape(-1)}
    if op == "mlp":
        T, f = case["T"], case["f"]
        width = 2 * f if case["act"] == "swiglu" else f
        return {"z": _activations(g, T, width, dt), "da": _normal(g, (T, f), dt, 1e-3)}
    T, k, n = case["T"], case["k"], case["n"]
    q, scale = _pack(_activations(g, T, k, dt))
    return {"q": q, "scale": scale, "dy": _normal(g, (T, n), dt, 1e-3)}


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if "axes" in case:        # inverse frequencies, which a program keeps whatever computes the rotation
        state["pairs"] = _pairs(case)
    if own:        # what a program that calls the framework keeps: the frequencies' table, scratch memory, buffers for what a call writes
        state["kept"] = _kept(case)
    return state


# ------------------------------------------------------------------------------- plain forms
def _sections(case):
    return [int(s) for s in case["sections"].split(",")]


def _pairs(case):
    """(axis, frequency) of every pair of a head, on the GPU; a pair that stays has axis 0 and frequency 0."""
    d, base, order = case["d"], case["base"], case["order"]
    sections = _sections(case)
    dealt = [(a, j) for a, s in enumerate(sections) for j in range(s)]
    if order == "dealt":
        dealt.sort(key=lambda p: (p[1], p[0]))
    stay = d // 2 - len(dealt)
    freq = [base ** (-j / sections[a]) if order == "own" else base ** (-2.0 * i / d) for i, (a, j) in enumerate(dealt)]
    return (torch.tensor([a for a, _ in dealt] + [0] * stay, device="cuda"), torch.tensor(freq + [0.0] * stay, device="cuda", dtype=torch.float64))


def _angles(s):
    axis, freq = s["pairs"]
    return s["pos"][axis].t().double() * freq      # [T, d / 2]


def _rotate(case, s, x, sign):
    """x [T, heads, d] in 32 bits."""
    angle = _angles(s)
    cos, sin = torch.cos(angle).float().unsqueeze(1), (sign * torch.sin(angle)).float().unsqueeze(1)
    if case["pairing"] == "halves":
        a, b = x.chunk(2, dim=2)
        return torch.cat((a * cos - b * sin, a * sin + b * cos), dim=2)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * cos - b * sin, a * sin + b * cos), dim=3).flatten(2)


def _split(case, x):
    """The q and k parts [T, heads, d] in 32 bits, and the v part as it is."""
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    x = x.reshape(case["T"], H + 2 * Hkv, d)
    return x[:, :H].float(), x[:, H:H + Hkv].float(), x[:, H + Hkv:]


def _join(case, q, k, v):
    return torch.cat((q.to(v.dtype), k.to(v.dtype), v), dim=1).reshape(case["T"], -1)


def _normed(case, x):
    mean = x.mean(2, keepdim=True) if case["norm"] == "layernorm" else torch.zeros_like(x[..., :1])
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(2, keepdim=True) + case["eps"])
    return (x - mean) * rstd, rstd


def _qk_fwd(case, s):
    q, k, v = _split(case, s["x"])
    out = []
    for part, x in (("q", q), ("k", k)):
        y = _normed(case, x)[0] * s["gain_" + part].float()
        if case["norm"] == "layernorm":
            y = y + s["shift_" + part].float()
        out.append(_rotate(case, s, y, 1.0))
    return {"y": _join(case, *out, v)}


def _qk_bwd(case, s):
    q, k, _ = _split(case, s["x"])
    dq, dk, dv = _split(case, s["dy"])
    dx, grads = [], {}
    for part, x, dy in (("q", q, dq), ("k", k, dk)):
        xhat, rstd = _normed(case, x)
        g = _rotate(case, s, dy, -1.0)
        gain = s["gain_" + part]
        grads["dgain_" + part] = (g * xhat).sum((0, 1)).to(gain.dtype)
        if case["norm"] == "layernorm":
            grads["dshift_" + part] = g.sum((0, 1)).to(gain.dtype)
        w = g * gain.float()
        if case["norm"] == "layernorm":
            w = w - w.mean(2, keepdim=True)
        dx.append(rstd * (w - xhat * (w * xhat).mean(2, keepdim=True)))
    return {"dx": _join(case, *dx, dv), **grads}


def _activate(act, z):
    """a and a function that takes da to dz, in 32 bits."""
    if act == "swiglu":
        gate, up = z.chunk(2, dim=1)
        s = 1.0 / (1.0 + torch.exp(-gate))
        return gate * s * up, lambda da: torch.cat((da * up * (s * (1.0 + gate * (1.0 - s))), da * (gate * s)), dim=1)
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * p, lambda da: da * (p + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2 * math.pi)))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1.0 + t), lambda da: da * (0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z))


def _mlp(case, s):
    z, da = s["z"], s["da"]
    a, _ = _activate(case["act"], z.float())
    kept = _unpack(*_pack(z)).reshape(z.shape)
    again, back = _activate(case["act"], kept)
    return {"a": a.to(z.dtype), "dz": back(da.float()).to(z.dtype), "a_again": again.to(z.dtype)}


def _wgrad(case, s):
    x = _unpack(s["q"], s["scale"]).reshape(case["T"], case["k"])
    dy = s["dy"].float()
    out = {"dw": (x.t().contiguous() @ dy).to(s["dy"].dtype)}
    if case["bias"]:
        out["db"] = dy.sum(0).to(s["dy"].dtype)
    return out


def run(state):
    case = state["case"]
    if own:
        return _call(case, state, state["kept"])
    op = case["op"]
    if op == "rotate":
        q, k, v = _split(case, state["x"])
        sign = -1.0 if case["back"] else 1.0
        return {"y": _join(case, _rotate(case, state, q, sign), _rotate(case, state, k, sign), v)}
    if op == "save_load":
        return {"x": _unpack(*_pack(state["x"])).to(state["x"].dtype)}
    return {"qk_fwd": _qk_fwd, "qk_bwd": _qk_bwd, "mlp": _mlp, "wgrad": _wgrad}[op](case, state)


# ------------------------------------------------------------------------------- the framework's calls
def _binding():
    from paper_2605_18710_amd import binding
    return binding


def _kept(case):
    mb = _binding()
    op, dt = case["op"], DT[case["dtype"]]

    def empty(*shape, dtype=dt):
        return torch.empty(shape, device="cuda", dtype=dtype)

    def scratch(size):
        return torch.empty(max(size, 256), device="cuda", dtype=torch.uint8)

    if op in ("rotate", "qk_fwd", "qk_bwd"):
        T, d = case["T"], case["d"]
        table = scratch(mb.rope_axes_table_bytes(d))
        mb.op_rope_axes_table(torch.cuda.current_stream().cuda_stream, CUS, d, _sections(case), case["order"], case["base"], table)
        kept = {"table": table, "y": empty(T, (case["H"] + 2 * case["Hkv"]) * d)}
        if op == "qk_bwd":
            kept.update(scratch=scratch(mb.qk_norm_rope_bwd_scratch_bytes(d)), dgain_q=empty(d), dgain_k=empty(d), dshift_q=empty(d), dshift_k=empty(d))
        return kept
    if op == "save_load":
        n = case["n"]
        return {"q": empty(n, dtype=torch.int8), "scale": empty(mb.pack8_scale_bytes(n), dtype=torch.uint8), "x": empty(n)}
    if op == "mlp":
        T, f = case["T"], case["f"]
        width = 2 * f if case["act"] == "swiglu" else f
        return {"q": empty(T * width, dtype=torch.int8), "scale": empty(mb.pack8_scale_bytes(T * width), dtype=torch.uint8),
                "a": empty(T, f), "dz": empty(T, width), "a_again": empty(T, f)}
    T, k, n = case["T"], case["k"], case["n"]
    return {"dw": empty(k, n), "db": empty(n), "scratch": scratch(mb.linear_wgrad_pack8_scratch_bytes(case["dtype"], T, k, n))}


def _call(case, s, kept):
    mb = _binding()
    op, dt = case["op"], case["dtype"]
    stream = torch.cuda.current_stream().cuda_stream
    if op in ("rotate", "qk_fwd", "qk_bwd"):
        heads = (case["T"], case["H"], case["Hkv"], case["d"])
        norm, eps, pairing, axes = case["norm"], case["eps"], case["pairing"], case["axes"]
        y = kept["y"]
        if op == "rotate":
            mb.op_rope_axes(stream, CUS, dt, *heads, pairing, -1 if case["back"] else 1, axes, s["pos"], kept["table"], s["x"], y)
            return {"y": y}
        layer = norm == "layernorm"
        if op == "qk_fwd":
            mb.op_qk_norm_rope_fwd(stream, CUS, dt, norm, *heads, eps, pairing, axes, s["pos"], kept["table"], s["x"], s["gain_q"],
                                   s["shift_q"] if layer else None, s["gain_k"], s["shift_k"] if layer else None, y)
            return {"y": y}
        mb.op_qk_norm_rope_bwd(stream, CUS, dt, norm, *heads, eps, pairing, axes, s["pos"], kept["table"], s["x"], s["gain_q"], s["gain_k"], s["dy"], y,
                               kept["dgain_q"], kept["dshift_q"] if layer else None, kept["dgain_k"], kept["dshift_k"] if layer else None, kept["scratch"])
        out = {"dx": y, "dgain_q": kept["dgain_q"]}
        if layer:
            out["dshift_q"] = kept["dshift_q"]
        out["dgain_k"] = kept["dgain_k"]
        if layer:
            out["dshift_k"] = kept["dshift_k"]
        return out
    if op == "save_load":
        mb.op_pack8(stream, CUS, dt, case["n"], s["x"], kept["q"], kept["scale"])
        mb.op_unpack8(stream, CUS, dt, case["n"], kept["q"], kept["scale"], kept["x"])
        return {"x": kept["x"]}
    if op == "mlp":
        T, f, act = case["T"], case["f"], case["act"]
        mb.op_act_fwd_pack8(stream, CUS, dt, act, T, f, s["z"], kept["a"], kept["q"], kept["scale"])
        mb.op_act_bwd_pack8(stream, CUS, dt, act, T, f, kept["q"], kept["scale"], s["da"], kept["dz"], kept["a_again"])
        return {"a": kept["a"], "dz": kept["dz"], "a_again": kept["a_again"]}
    mb.op_linear_wgrad_pack8(stream, CUS, dt, case["T"], case["k"], case["n"], s["q"], s["scale"], s["dy"], kept["dw"], kept["db"] if case["bias"] else None,
                             kept["scratch"])
    return {"dw": kept["dw"], "db": kept["db"]} if case["bias"] else {"dw": kept["dw"]}


# ------------------------------------------------------------------------------- in 64 bits
def _turned(case, x, pos, sign):
    """Rotation as a product of complex numbers; the pairs dealt out one by one."""
    d, base, sections = case["d"], case["base"], _sections(case)
    angle = torch.zeros((case["T"], d // 2), device="cuda", dtype=torch.float64)
    left, a = list(sections), 0
    for i in range(sum(sections)):
        while left[a] == 0:
            a = (a + 1) % len(left)
        nth = sections[a] - left[a]
        angle[:, i] = sign * pos[a].double() * base ** (-nth / sections[a] if case["order"] == "own" else -2.0 * i / d)
        left[a] -= 1
        a = (a + 1) % len(left) if case["order"] == "dealt" else a
    if case["pairing"] == "halves":
        z = torch.complex(*x.unflatten(2, (2, -1)).unbind(2))
        return torch.view_as_real(z * torch.polar(torch.ones_like(angle), angle)[:, None]).movedim(3, 2).flatten(2)
    z = torch.view_as_complex(x.unflatten(2, (-1, 2)).contiguous())
    return torch.view_as_real(z * torch.polar(torch.ones_like(angle), angle)[:, None]).flatten(2)


def _exact_heads(case, i):
    H, Hkv, T, d = case["H"], case["Hkv"], case["T"], case["d"]
    parts = [p.double().unflatten(1, (-1, d)) for p in i["x"].split((H * d, Hkv * d, Hkv * d), dim=1)]
    if case["op"] == "rotate":
        sign = -1.0 if case["back"] else 1.0
        return {"y": torch.cat([_turned(case, p, i["pos"], sign).flatten(1) for p in parts[:2]] + [parts[2].flatten(1)], dim=1)}
    layer, out, grads = case["norm"] == "layernorm", [], {}
    upstream = i["dy"].double().split((H * d, Hkv * d, Hkv * d), dim=1) if case["op"] == "qk_bwd" else None
    for j, part in enumerate(("q", "k")):
        x, gain = parts[j].requires_grad_(upstream is not None), i["gain_" + part].double().requires_grad_(upstream is not None)
        shift = (i["shift_" + part].double() if layer else torch.zeros_like(gain)).requires_grad_(upstream is not None)
        centred = x - x.sum(2, keepdim=True) / d if layer else x
        y = _turned(case, centred * torch.rsqrt((centred * centred).sum(2, keepdim=True) / d + case["eps"]) * gain + shift, i["pos"], 1.0)
        if upstream is None:
            out.append(y.flatten(1))
            continue
        dx, dgain, dshift = torch.autograd.grad(y, (x, gain, shift), upstream[j].unflatten(1, (-1, d)))
        out.append(dx.flatten(1))
        grads["dgain_" + part] = dgain
        if layer:
            grads["dshift_" + part] = dshift
    if upstream is None:
        return {"y": torch.cat(out + [parts[2].flatten(1)], dim=1)}
    return {"dx": torch.cat(out + [upstream[2]], dim=1), **grads}


def _steps():
    """2^-128 to 2^128, from the host's own powers: ties between two whole numbers have to stay ties."""
    return torch.tensor([2.0 ** e for e in range(-128, 129)], device="cuda", dtype=torch.float64)


def _nearest(x):
    """What x stands for once it is kept in blocks of 32 whole numbers, from the definition: the first of the steps that is large enough."""
    flat = x.double().reshape(-1)
    rows = torch.cat((flat, flat.new_zeros(-flat.numel() % 32))).view(-1, 32)
    top = rows.abs().max(1, keepdim=True).values
    steps = _steps()[1:]
    step = steps[torch.searchsorted(127.5 * steps, top)]
    return ((rows / step).round().clamp(-127, 127) * step).view(-1)[:flat.numel()].view(x.shape)


def _exact_act(act, z):
    if act == "swiglu":
        gate, up = z.split(z.shape[1] // 2, dim=1)
        return gate * torch.sigmoid(gate) * up
    return torch.nn.functional.gelu(z, approximate="tanh" if act == "gelu_tanh" else "none")


def exact(case, seed):
    i = _inputs(case, seed)
    op = case["op"]
    if op in ("rotate", "qk_fwd", "qk_bwd"):
        return _exact_heads(case, i)
    if op == "save_load":
        return {"x": _nearest(i["x"])}
    if op == "mlp":
        a = _exact_act(case["act"], i["z"].double())
        kept = _nearest(i["z"]).requires_grad_(True)
        again = _exact_act(case["act"], kept)
        dz, = torch.autograd.grad(again, kept, i["da"].double())
        return {"a": a, "dz": dz, "a_again": again.detach()}
    T, k = case["T"], case["k"]
    step = _steps()[i["scale"].long() + 1]
    x = (i["q"].double() * step.repeat_interleave(32)[:T * k]).view(T, k)
    dy = i["dy"].double()
    out = {"dw": torch.mm(x.t().contiguous(), dy)}
    if case["bias"]:
        out["db"] = torch.mv(dy.t().contiguous(), torch.ones(T, device="cuda", dtype=torch.float64))
    return out
