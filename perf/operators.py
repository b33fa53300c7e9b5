"""The operators of a latent world model's transformer block, as a list of sized cases: attention of many heads to states of
another length, rotary positions, and the norm around a block with its gate and residual.  The decoder's user runs such a
model in front of it; a frame of 720x480 is a latent of 60x90, in patches of 2x2 1350 tokens.

A case's fields: op and what sizes it.  `run` computes the plain form in torch, or calls the library (`own`).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _attention(name, dtype, batch, q_len, kv_len, heads, kv_heads, dim, ragged):
    return {"name": name, "op": "attention", "dtype": dtype, "batch": batch, "q_len": q_len, "kv_len": kv_len, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "ragged": ragged}


def _rotary(name, dtype, batch, tokens, heads, kv_heads, dim, rotary, layout, axes, far):
    return {"name": name, "op": "rotary", "dtype": dtype, "batch": batch, "tokens": tokens, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "rotary": rotary, "layout": layout, "axes": axes, "far": far}


def _norm(name, dtype, stream, batch, tokens, group, channels, kind, post):
    return {"name": name, "op": "norm", "dtype": dtype, "stream": stream, "batch": batch, "tokens": tokens, "group": group,
            "channels": channels, "kind": kind, "post": post}


def listed():
    return [
        # one action token per session against its own short history: latency
        _attention("attn-bf16-token", "bf16", 8, 1, 512, 16, 16, 64, True),
        # one token per session against a long memory of past frames, heads in groups of four: the bytes of k and v
        _attention("attn-bf16-token-long", "bf16", 4, 1, 16384, 32, 8, 128, True),
        # eight frames of patches attend to a padded text prompt, with and without it (guidance)
        _attention("attn-bf16-text", "bf16", 2, 10800, 77, 30, 30, 64, True),
        # patches of a frame attend to each other, eight frames
        _attention("attn-bf16-frame", "bf16", 8, 1350, 1350, 30, 30, 64, False),
        # the latent pixels of a 720x480 frame attend to those of a 1280x720 one
        _attention("attn-bf16-history", "bf16", 1, 5400, 14400, 16, 16, 128, False),
        # single precision, as it is run to check the other, odd lengths
        _attention("attn-f32", "f32", 2, 1350, 777, 12, 4, 80, True),
        # q and k of one new token per session, far positions
        _rotary("rotary-bf16-token", "bf16", 8, 1, 32, 8, 128, 128, "half", 1, True),
        # q and k of eight frames of patches: time, row and column
        _rotary("rotary-bf16-frames", "bf16", 2, 10800, 30, 30, 64, 64, "interleaved", 3, False),
        # single precision, part of the head
        _rotary("rotary-f32-part", "f32", 3, 1013, 12, 4, 80, 32, "half", 1, True),
        # one token per session
        _norm("norm-bf16-token", "bf16", "f32", 8, 1, 1, 1920, "layer", False),
        # eight frames of patches, each frame with a noise level (modulation) of its own; residual stream in single precision
        _norm("norm-bf16-frames", "bf16", "f32", 2, 10800, 1350, 1920, "layer", False),
        # single precision, norms before and after the block, a width that no vector divides
        _norm("norm-f32-sandwich", "f32", "f32", 3, 1013, 1013, 1111, "rms", True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    cases = listed()
    most = {op: max(work(c)["bytes"] + work(c)["flops"] / 100 for c in cases if c["op"] == op) for op in ("attention", "rotary", "norm")}
    while True:
        op = rng.choice(("attention", "attention", "attention", "rotary", "norm"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        if op == "attention":
            kv_heads = _log_int(rng, 1, 32)
            heads = kv_heads * rng.choice((1, 1, 1, 2, 4, 5, 8))
            q_len = rng.choice((1, 1, _log_int(rng, 1, 16), _log_int(rng, 16, 11000), _log_int(rng, 16, 11000), _log_int(rng, 16, 11000)))
            c = _attention("", dtype, _log_int(rng, 1, 16), q_len, _log_int(rng, 1, 17000), heads, kv_heads,
                           rng.choice((32, 40, 64, 64, 72, 80, 96, 128, 128)), rng.random() < 0.6)
            if c["batch"] * heads * q_len * c["kv_len"] > 1.2e9 or (dtype == "f32" and work(c)["flops"] > 4e10):
                continue
        elif op == "rotary":
            dim = rng.choice((32, 40, 64, 80, 96, 128, 256))
            axes = rng.choice((1, 1, 2, 3))
            rotary = dim if rng.random() < 0.6 else 2 * rng.randint(axes, dim // 2)
            kv_heads = _log_int(rng, 1, 32)
            c = _rotary("", dtype, _log_int(rng, 1, 8), _log_int(rng, 1, 11000), kv_heads * rng.choice((1, 1, 2, 4)), kv_heads, dim, rotary,
                        rng.choice(("half", "interleaved")), axes, axes == 1 and rng.random() < 0.5)
        else:
            tokens = _log_int(rng, 1, 11000)
            channels = _log_int(rng, 64, 8192)
            c = _norm("", dtype, rng.choice((dtype, "f32")), _log_int(rng, 1, 8), tokens, rng.choice((tokens, max(1, tokens // 8))),
                      channels if rng.random() < 0.25 else max(64, channels // 64 * 64), rng.choice(("layer", "rms")), rng.random() < 0.4)
        c.pop("name")
        if work(c)["bytes"] + work(c)["flops"] / 100 <= most[op]:
            return c


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _axis_pairs(case):
    n, a = case["rotary"] // 2, case["axes"]
    return [n - (a - 1) * (n // a)] + [n // a] * (a - 1)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "attention":
        b, h, n, d = case["batch"], case["heads"], case["kv_heads"], case["dim"]
        s["q"] = _randn(g, b, case["q_len"], h, d).to(dt)
        kv = _randn(g, b, case["kv_len"], 2, n, d).to(dt)                        # one projection makes both
        s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
        s["lens"] = None
        if case["ragged"]:
            lens = torch.randint((case["kv_len"] + 1) // 2, case["kv_len"] + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
            lens[0] = case["kv_len"]
            s["lens"] = lens
        s["scale"] = d ** -0.5
        s["o"] = torch.empty_like(s["q"])
    elif case["op"] == "rotary":
        b, t, a = case["batch"], case["tokens"], case["axes"]
        qkv = _randn(g, b, t, case["heads"] + 2 * case["kv_heads"], case["dim"]).to(dt)
        s["x"] = qkv[:, :, :case["heads"] + case["kv_heads"]]
        s["pairs"] = _axis_pairs(case)
        # turns per position of each pair: base^(-i/n) / 2 pi, in 64 bits
        s["freqs"] = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) / (2 * math.pi) for n in s["pairs"]]).cuda()
        if a == 1:
            first = torch.randint(0, 1000000 if case["far"] else 1000, (b, 1), generator=g, device="cuda", dtype=torch.int32)
            s["positions"] = (first + torch.arange(t, device="cuda", dtype=torch.int32)).unsqueeze(2)
        else:                                                                    # time, row (and column) of each patch
            i = torch.arange(t, device="cuda", dtype=torch.int32)
            at = [i // 1350, i % 1350 // 45, i % 45] if a == 3 else [i // 45, i % 45]
            first = torch.randint(0, 1000, (b, 1, 1), generator=g, device="cuda", dtype=torch.int32)
            s["positions"] = (torch.stack(at, 1) + first).contiguous()
        s["y"] = torch.empty(s["x"].shape, dtype=dt, device="cuda")
    else:
        b, t, c = case["batch"], case["tokens"], case["channels"]
        m = -(-t // case["group"])
        st = TYPES[case["stream"]]
        s["x"] = (2 * _randn(g, b, t, c) + 0.5).to(st)
        s["h"] = _randn(g, b, t, c).to(dt)
        mods = (0.3 * _randn(g, b, m, 3, c)).to(dt)                              # one projection makes the three
        s["gate"], s["scale"], s["shift"] = mods[:, :, 0], mods[:, :, 1], mods[:, :, 2]
        s["weight"] = 1 + 0.1 * _randn(g, c)
        s["post"] = 1 + 0.1 * _randn(g, c) if case["post"] else None
        s["x_out"], s["y"] = torch.empty_like(s["x"]), torch.empty_like(s["h"])
    return s


EPS, ALPHA = 1e-6, 0.7


def _attention_plain(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    b, t, h, d = q.shape
    n = k.shape[2]
    q = q.reshape(b, t, n, h // n, d).permute(0, 2, 3, 1, 4)                     # [b, n, group, t, d]
    p = torch.matmul(q * s["scale"], k.permute(0, 2, 3, 1).unsqueeze(2))
    v = v.permute(0, 2, 1, 3).unsqueeze(2)
    if s["lens"] is not None:
        gone = torch.arange(k.shape[1], device=q.device) >= s["lens"].view(b, 1, 1, 1, 1)
        p = p.masked_fill(gone, -math.inf)
        v = v.masked_fill(gone.transpose(3, 4), 0.0)
    p = (p - p.amax(4, keepdim=True)).exp_()
    o = torch.matmul(p, v) / p.sum(4, keepdim=True)
    if s["lens"] is not None:
        o = o.masked_fill(s["lens"].view(b, 1, 1, 1, 1) == 0, 0.0)
    return o.permute(0, 3, 1, 2, 4).reshape(b, t, h, d).to(s["q"].dtype)


def _rotary_plain(s):
    x, n = s["x"].float(), s["freqs"].numel()
    at = s["positions"].double().repeat_interleave(torch.tensor(s["pairs"], device=x.device), dim=2, output_size=n)
    angle = at * s["freqs"]
    angle = (2 * math.pi * (angle - angle.round())).unsqueeze(2)                 # [b, t, 1, pairs], in 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()
    turned, rest = x[..., :2 * n], x[..., 2 * n:]
    if s["case"]["layout"] == "half":
        u, w = turned[..., :n], turned[..., n:]
        y = torch.cat([u * cos - w * sin, u * sin + w * cos, rest], 3)
    else:
        u, w = turned[..., 0::2], turned[..., 1::2]
        y = torch.cat([torch.stack([u * cos - w * sin, u * sin + w * cos], 4).flatten(3), rest], 3)
    return y.to(s["x"].dtype)


def _unit(x, kind):
    if kind == "layer":
        x = x - x.mean(2, keepdim=True)
    return x * torch.rsqrt(x.square().mean(2, keepdim=True) + EPS)


def _norm_plain(s):
    case = s["case"]
    gate, scale, shift = (s[n].float().repeat_interleave(case["group"], 1)[:, :case["tokens"]] for n in ("gate", "scale", "shift"))
    u = s["h"].float()
    if s["post"] is not None:
        u = _unit(u, case["kind"]) * s["post"]
    r = s["x"].float() + ALPHA * gate * u
    y = _unit(r, case["kind"]) * s["weight"] * (1 + scale) + shift
    return {"x": r.to(s["x"].dtype), "y": y.to(s["h"].dtype)}


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        from paper_2602_00608_b200 import binding
        if op == "attention":
            return binding.op_cross_attention(s["q"], s["k"], s["v"], s["lens"], scale=s["scale"], out=s["o"])
        if op == "rotary":
            return binding.op_rotary(s["x"], s["freqs"], s["positions"], layout=s["case"]["layout"], axis_pairs=s["pairs"], out=s["y"])
        x, y = binding.op_gate_norm(s["x"], s["h"], gate=s["gate"], scale=s["scale"], shift=s["shift"], kind=s["case"]["kind"], eps=EPS,
                                    weight=s["weight"], post_norm=s["post"] is not None, post_weight=s["post"], residual_scale=ALPHA,
                                    mod_tokens=s["case"]["group"], x_out=s["x_out"], y=s["y"])
        return {"x": x, "y": y}
    return _attention_plain(s) if op == "attention" else _rotary_plain(s) if op == "rotary" else _norm_plain(s)


def work(case):
    """Inputs once, outputs once; keys of a ragged batch at the three quarters that they have on average (the first has all)."""
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "attention":
        b, h, n, d = case["batch"], case["heads"], case["kv_heads"], case["dim"]
        keys = case["kv_len"] * (1 + 0.75 * (b - 1)) if case["ragged"] else b * case["kv_len"]
        return {"bytes": size * d * (2.0 * b * case["q_len"] * h + 2.0 * keys * n), "flops": 4.0 * case["q_len"] * keys * h * d}
    if case["op"] == "rotary":
        rows = case["batch"] * case["tokens"]
        values = rows * (case["heads"] + case["kv_heads"])
        return {"bytes": 2.0 * size * values * case["dim"] + 4.0 * rows * case["axes"], "flops": 3.0 * values * case["rotary"]}
    rows, c, st = case["batch"] * case["tokens"], case["channels"], 4 if case["stream"] == "f32" else 2
    mods = 3 * case["batch"] * -(-case["tokens"] // case["group"])
    return {"bytes": c * (rows * 2.0 * (st + size) + mods * size), "flops": rows * c * (20.0 if case["post"] else 12.0)}


def exact(case, seed):
    """From the definitions, in 64 bits, head by head and row by row."""
    s = prepare(case, seed)
    dt = torch.float64
    if case["op"] == "attention":
        q, k, v = (s[n].to(dt) for n in "qkv")
        o = torch.zeros_like(q)
        for b in range(case["batch"]):
            n = case["kv_len"] if s["lens"] is None else int(s["lens"][b])
            for h in range(case["heads"] if n else 0):
                at = h * case["kv_heads"] // case["heads"]
                for t in range(0, case["q_len"], 2048):
                    score = s["scale"] * (q[b, t:t + 2048, h] @ k[b, :n, at].T)
                    o[b, t:t + 2048, h] = torch.exp(score - torch.logsumexp(score, 1, keepdim=True)) @ v[b, :n, at]
        return o
    if case["op"] == "rotary":
        x = s["x"].to(dt)
        y = x.clone()
        n, i = case["rotary"] // 2, 0
        for axis, pairs in enumerate(s["pairs"]):
            for j in range(pairs):
                one, two = (i, i + n) if case["layout"] == "half" else (2 * i, 2 * i + 1)
                turn = torch.polar(torch.ones((), dtype=dt, device="cuda"), 2 * math.pi * torch.remainder(s["positions"][:, :, axis].to(dt) * s["freqs"][i], 1.0))
                z = torch.complex(x[..., one], x[..., two]) * turn.unsqueeze(2)
                y[..., one], y[..., two] = z.real, z.imag
                i += 1
        return y
    mods = {n: s[n].to(dt)[:, torch.arange(case["tokens"], device="cuda") // case["group"]] for n in ("gate", "scale", "shift")}

    def unit(z):
        if case["kind"] == "layer":
            var, mean = torch.var_mean(z, dim=2, correction=0, keepdim=True)
            return (z - mean) / torch.sqrt(var + EPS)
        return z / torch.sqrt(torch.linalg.vector_norm(z, dim=2, keepdim=True) ** 2 / z.shape[2] + EPS)

    u = s["h"].to(dt)
    if case["post"]:
        u = unit(u) * s["post"].to(dt)
    r = torch.addcmul(s["x"].to(dt), mods["gate"], u, value=ALPHA)
    return {"x": r, "y": torch.addcmul(mods["shift"], unit(r) * s["weight"].to(dt), 1 + mods["scale"])}
