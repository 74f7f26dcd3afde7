"""The 8-bit products of a DiT block on the active rows and what feeds them, as timed cases.

Kinds:

  quant   rows of bf16 values to 8-bit codes with one power-of-two scale per 1 x 128 block
          (activations) or 128 x 128 block (weights).
  rms     h += gate * y, then the root-mean-square norm with its weight and the request's
          modulation, as 8-bit rows with scales.
  rope    q | k | v rows: q and k turned by the token's position on several axes, q to its rows,
          k and v to the cache rows of their tokens.
  linear  act(A W^T + bias) of 8-bit rows and weights with block scales, to bf16, fp32 or 8-bit rows.

8-bit values are e4m3 codes times 2^(s - 127), s a byte per block: s - 127 is the smallest power at
which the block's largest magnitude is at most 448.  Row counts are the active rows of the package's
workloads (image, video, audio, packed images) and odd ones; widths are those models' and odd ones.
"""
from __future__ import annotations

import math

import torch

own = False

# model widths: hidden size and head dim of the package's image, video and audio models, and odd ones
WIDTHS = (64, 384, 576, 1024, 1088, 1536, 2048)
MOST_FLOPS = 2 * 32760 * 1536 * 6144


def listed():
    return [
        # one active token behind the attention of a block: latency
        dict(name="rms_one", kind="rms", rows=1, width=1536, requests=1, branch=True),
        # a packed batch of eight image requests, each with its own modulation
        dict(name="rms_packed", kind="rms", rows=8937, width=1536, requests=8, branch=True),
        # the attention output of a video step on its way to the out-projection
        dict(name="quant_video", kind="quant", rows=9828, width=1536, block=1),
        # an MLP weight when a model is loaded (odd width: the last block is half a block)
        dict(name="quant_weight", kind="quant", rows=4352, width=1088, block=128),
        # one row of a short sequence, one axis
        dict(name="rope_one", kind="rope", rows=1, tokens=2048, heads=16, kv_heads=16, dh=64, axes="64", halves=True, far=1),
        # a video step: time, height and width, 30% of the tokens active
        dict(name="rope_video", kind="rope", rows=9828, tokens=32760, heads=12, kv_heads=12, dh=128, axes="44,42,42", halves=False, far=1),
        # an image with shared key heads and far, rescaled positions
        dict(name="rope_image", kind="rope", rows=1664, tokens=4096, heads=24, kv_heads=8, dh=64, axes="32,32", halves=True, far=1000),
        # one active token through the fused projection: the weights are all that is read
        dict(name="linear_one", kind="linear", rows=1, out=4608, inner=1536, act=False, to="bf16"),
        # one image request: the second MLP product
        dict(name="linear_image", kind="linear", rows=1664, out=1536, inner=6144, act=False, to="bf16"),
        # odd sizes: a short sequence, widths that end inside a block, the first MLP product to 8 bits
        dict(name="linear_odd", kind="linear", rows=1021, out=4288, inner=1088, act=True, to="8"),
        # a video step: the first MLP product to 8 bits
        dict(name="linear_video", kind="linear", rows=9828, out=6144, inner=1536, act=True, to="8"),
        # the largest: the second MLP product of a video request's dense warm-up step
        dict(name="linear_dense", kind="linear", rows=32760, out=1536, inner=6144, act=False, to="f32"),
    ]


def draw(rng):
    rows = int(round(math.exp(rng.uniform(0.0, math.log(32760)))))
    kind = rng.choice(("quant", "rms", "rope", "linear", "linear"))
    if kind == "quant":
        return dict(kind=kind, rows=rows, width=16 * rng.randint(4, 384), block=rng.choice((1, 1, 128)))
    if kind == "rms":
        return dict(kind=kind, rows=rows, width=rng.choice(WIDTHS), requests=rng.randint(1, min(rows, 64)), branch=rng.random() < 0.7)
    if kind == "rope":
        dh = rng.choice((16, 64, 128))
        kv = rng.randint(1, 1024 // dh)
        n = rng.randint(1, 3)
        cuts = sorted(2 * rng.randint(1, dh // 2 - 1) for _ in range(n - 1)) if dh > 16 else [2 * (i + 1) for i in range(n - 1)]
        axes = [b - a for a, b in zip([0] + cuts, cuts + [dh]) if b > a]
        return dict(kind=kind, rows=rows, tokens=rows + rng.randint(0, rows), heads=kv * rng.choice((1, 1, 2)), kv_heads=kv, dh=dh,
                    axes=",".join(map(str, axes)), halves=rng.random() < 0.5, far=rng.choice((1, 1000)))
    out, inner = 64 * rng.randint(1, 100), 64 * rng.randint(1, 100)
    rows = max(1, min(rows, MOST_FLOPS // (2 * out * inner)))
    return dict(kind=kind, rows=rows, out=out, inner=inner, act=rng.random() < 0.4, to=rng.choice(("bf16", "f32", "8")))


# ------------------------------------------------------------------ 8-bit blocks, plain

def _blocks(x, block):
    """x [rows][cols] fp32 as [rows / block][block][cols / 128][128], zero-filled."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % block))
    return x.view((r + block - 1) // block, block, (c + 127) // 128, 128)


def _spread(s, r, c, block):
    """The block values s [rows / block][cols / 128] at every place of [r][c]."""
    return s.repeat_interleave(block, 0)[:r].repeat_interleave(128, 1)[:, :c]


def _to_blocks(x, block=1):
    """(codes e4m3 [r][c], powers of two fp32 [blocks]) of x fp32."""
    r, c = x.shape
    top = _blocks(x, block).abs().amax((1, 3))
    mant, ex = torch.frexp(top)                     # top = mant 2^ex, mant in [1/2, 1); 448 = 0.875 * 2^9
    ex = (ex - 9 + (mant > 0.875)).clamp(-126, 127)
    ex = torch.where(top > 0, ex, -126)
    up = torch.ldexp(torch.ones_like(top), -ex)
    return (x * _spread(up, r, c, block)).to(torch.float8_e4m3fn), torch.ldexp(torch.ones_like(top), ex)


def _bytes(s):
    return s.to(torch.float8_e8m0fnu)


def _padded(s):
    """Scales [blocks][cols / 128] as bytes, rows padded to a multiple of four."""
    out = torch.full((s.shape[0], (s.shape[1] + 3) // 4 * 4), 127, dtype=torch.uint8, device=s.device)
    out[:, :s.shape[1]] = _bytes(s).view(torch.uint8)
    return out


def _gelu(z):
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))


# ------------------------------------------------------------------ inputs

def _gen(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 17)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _request_offsets(rows, requests):
    """Requests of different lengths, in order: offsets 0 = o_0 <= ... <= o_B = rows."""
    w = torch.arange(1, requests + 1, dtype=torch.float64)
    o = torch.floor(torch.cumsum(w, 0) / w.sum() * rows).to(torch.int32)
    o[-1] = rows
    return torch.cat([torch.zeros(1, dtype=torch.int32), o])


def prepare(case, seed):
    g = _gen(case, seed)
    rows, s = case["rows"], dict(case)
    s["m"] = torch.tensor([rows], dtype=torch.int32, device="cuda")
    if case["kind"] == "quant":
        s["x"] = (_randn(g, rows, case["width"]) * torch.exp(_randn(g, rows, 1))).to(torch.bfloat16)
        s["q"] = torch.zeros((rows, case["width"]), dtype=torch.float8_e4m3fn, device="cuda")
        nb, nk = -(-rows // case["block"]), -(-case["width"] // 128)
        s["scale"] = torch.full((nb, (nk + 3) // 4 * 4), 127, dtype=torch.uint8, device="cuda")
    elif case["kind"] == "rms":
        w, b = case["width"], case["requests"]
        off = _request_offsets(rows, b)
        s["cu_q"] = off.cuda()
        s["of_row"] = torch.repeat_interleave(torch.arange(b), (off[1:] - off[:-1]).long()).cuda()
        s["h"] = _randn(g, rows, w) * (1.0 + 3.0 * torch.rand((rows, 1), generator=g, device="cuda"))
        s["y"] = _randn(g, rows, w).to(torch.bfloat16) if case["branch"] else None
        s["mod"] = 0.3 * _randn(g, b, 3 * w)        # shift | scale | gate
        s["weight"] = 1.0 + 0.1 * _randn(g, w)
        s["q"] = torch.zeros((rows, w), dtype=torch.float8_e4m3fn, device="cuda")
        s["scale"] = torch.full((rows, (-(-w // 128) + 3) // 4 * 4), 127, dtype=torch.uint8, device="cuda")
    elif case["kind"] == "rope":
        hq, hk, dh, t = case["heads"], case["kv_heads"], case["dh"], case["tokens"]
        s["dims"] = [int(a) for a in case["axes"].split(",")]
        n = len(s["dims"])
        s["theta"] = [10000.0] * n
        s["step"] = [1.0 if case["far"] == 1 else 0.25] * n
        # the grid of the tokens: each axis after the first takes about the n-th root of them
        side = max(1, int(round(t ** (1.0 / n))))
        tok = torch.arange(t, device="cuda")
        axes = [torch.div(tok, side ** (n - 1 - a), rounding_mode="floor") % (t if a == 0 else side) for a in range(n)]
        s["coord"] = (torch.stack(axes, 1) * case["far"]).to(torch.int32).contiguous()
        s["idx"] = torch.randperm(t, generator=g, device="cuda")[:rows].sort().values.to(torch.int32)
        s["qkv"] = _randn(g, rows, (hq + 2 * hk) * dh).to(torch.bfloat16)
        s["k"] = _randn(g, t, hk * dh).to(torch.bfloat16)
        s["v"] = _randn(g, t, hk * dh).to(torch.bfloat16)
        s["q"] = torch.zeros((rows, hq * dh), dtype=torch.bfloat16, device="cuda")
    else:
        n, k = case["out"], case["inner"]
        s["a"], sa = _to_blocks(_randn(g, rows, k) * torch.exp(0.5 * _randn(g, rows, 1)))
        s["w"], sw = _to_blocks(0.02 * _randn(g, n, k), 128)
        s["a_scale"], s["w_scale"] = _padded(sa), _padded(sw)
        s["bias"] = 0.02 * _randn(g, n)
        if case["to"] == "8":
            s["y"] = torch.zeros((rows, n), dtype=torch.float8_e4m3fn, device="cuda")
            s["y_scale"] = torch.full((rows, (-(-n // 128) + 3) // 4 * 4), 127, dtype=torch.uint8, device="cuda")
        else:
            s["y"] = torch.zeros((rows, n), dtype=torch.float32 if case["to"] == "f32" else torch.bfloat16, device="cuda")
            s["y_scale"] = None
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return {"quant": _quant, "rms": _rms, "rope": _rope, "linear": _linear}[s["kind"]](s)


def _quant(s):
    if own:
        from paper_2607_12121_amd import flashdiff as fdl
        fdl.fd_quant_blocks(s["x"], s["block"], s["q"], s["scale"])
        q, scale = s["q"], s["scale"][:, :-(-s["width"] // 128)].view(torch.float8_e8m0fnu)
    else:
        q, scale = _to_blocks(s["x"].float(), s["block"])
        scale = _bytes(scale)
    return {"q": q, "scale": scale}


def _rms(s):
    w = s["width"]
    shift, scale, gate = s["mod"][:, :w], s["mod"][:, w:2 * w], s["mod"][:, 2 * w:]
    if own:
        from paper_2607_12121_amd import flashdiff as fdl
        fdl.fd_rms_quant(s["h"], s["q"], s["scale"], s["cu_q"], s["m"], y=s["y"], gate=gate, weight=s["weight"], shift=shift,
                         mod_scale=scale, eps=1e-6)
        q, sc = s["q"], s["scale"][:, :-(-w // 128)].view(torch.float8_e8m0fnu)
    else:
        b, h = s["of_row"], s["h"]
        if s["y"] is not None:
            h += gate[b] * s["y"].float()
        a = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6) * s["weight"] * (1.0 + scale[b]) + shift[b]
        q, sc = _to_blocks(a)
        sc = _bytes(sc)
    return {"h": s["h"], "q": q, "scale": sc}


def _turned(x, cos, sin, dims, halves):
    """x [rows][heads][dh] fp32, cos and sin [rows][1][pairs]."""
    out, at, pair = [], 0, 0
    for d in dims:
        p, c, n = x[..., at:at + d], cos[..., pair:pair + d // 2], sin[..., pair:pair + d // 2]
        u, v = (p[..., :d // 2], p[..., d // 2:]) if halves else (p[..., 0::2], p[..., 1::2])
        r = (u * c - v * n, u * n + v * c)
        out.append(torch.cat(r, -1) if halves else torch.stack(r, -1).flatten(-2))
        at, pair = at + d, pair + d // 2
    return torch.cat(out + [x[..., at:]], -1)


def _angles(s):
    pos = s["coord"][s["idx"].long()].double()
    freq = [st * th ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
            for d, th, st in zip(s["dims"], s["theta"], s["step"])]
    return torch.cat([pos[:, a:a + 1] * f for a, f in enumerate(freq)], 1)[:, None]


def _rope(s):
    hq, hk, dh = s["heads"], s["kv_heads"], s["dh"]
    if own:
        from paper_2607_12121_amd import flashdiff as fdl
        fdl.fd_rope_axes(s["qkv"], s["coord"], s["idx"], s["m"], s["q"], s["k"], s["v"], heads=hq, kv_heads=hk, head_dim=dh,
                         dims=s["dims"], theta=s["theta"], step=s["step"], halves=s["halves"])
        q = s["q"]
    else:
        ang, rows = _angles(s), s["idx"].long()
        cos, sin = torch.cos(ang).float(), torch.sin(ang).float()
        x = s["qkv"].float().view(s["rows"], hq + 2 * hk, dh)
        qk = _turned(x[:, :hq + hk], cos, sin, s["dims"], s["halves"]).to(torch.bfloat16)
        q = qk[:, :hq].reshape(s["rows"], hq * dh)
        s["k"][rows] = qk[:, hq:].reshape(s["rows"], hk * dh)
        s["v"][rows] = s["qkv"][:, (hq + hk) * dh:]
    return {"q": q, "k": s["k"], "v": s["v"]}


def _linear(s):
    n, k = s["out"], s["inner"]
    if own:
        from paper_2607_12121_amd import flashdiff as fdl
        fdl.fd_scaled_linear(s["a"], s["a_scale"], s["w"], s["w_scale"], s["y"], s["y_scale"], bias=s["bias"], gelu=s["act"], m=s["m"])
        if s["to"] != "8":
            return {"y": s["y"]}
        return {"y": s["y"], "scale": s["y_scale"][:, :-(-n // 128)].view(torch.float8_e8m0fnu)}
    nk = -(-k // 128)
    a = s["a"].float() * _spread(s["a_scale"][:, :nk].view(torch.float8_e8m0fnu).float(), s["rows"], k, 1)
    w = s["w"].float() * _spread(s["w_scale"][:, :nk].view(torch.float8_e8m0fnu).float(), n, k, 128)
    y = a @ w.t() + s["bias"]
    if s["act"]:
        y = _gelu(y)
    if s["to"] == "8":
        y, scale = _to_blocks(y)
        return {"y": y, "scale": _bytes(scale)}
    return {"y": y.to(s["y"].dtype)}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    r = case["rows"]
    if case["kind"] == "quant":
        n, blocks = r * case["width"], -(-r // case["block"]) * -(-case["width"] // 128)
        return {"bytes": 3 * n + blocks, "flops": 3 * n}
    if case["kind"] == "rms":
        n = r * case["width"]
        return {"bytes": n * (4 + 1 + (2 + 4 if case["branch"] else 0)) + r * -(-case["width"] // 128)
                + 4 * case["width"] * (1 + case["requests"] * (3 if case["branch"] else 2)), "flops": 9 * n}
    if case["kind"] == "rope":
        hq, hk, dh, axes = case["heads"], case["kv_heads"], case["dh"], case["axes"].count(",") + 1
        return {"bytes": r * (4 * (hq + 2 * hk) * dh + 4 * axes + 4), "flops": 3 * r * (hq + hk) * dh}
    n, k = case["out"], case["inner"]
    size = {"bf16": 2, "f32": 4, "8": 1}[case["to"]]
    blocks = (r + -(-n // 128)) * -(-k // 128) + (r * -(-n // 128) if case["to"] == "8" else 0)
    return {"bytes": r * k + n * k + r * n * size + blocks + 4 * n, "flops": 2 * r * n * k}


# ------------------------------------------------------------------ the definitions in 64 bits

def _codes64(x, group):
    """(what the codes stand for before the scale, the scale) of x fp64, blocks of `group` x 128: the
    least power of two with amax / power <= 448, then the nearest value of 3 mantissa bits, ties to even."""
    r, c = x.shape
    pad = torch.zeros((-(-r // group) * group, -(-c // 128) * 128), dtype=torch.float64, device=x.device)
    pad[:r, :c] = x
    top = pad.reshape(pad.shape[0] // group, group, -1, 128).abs().transpose(1, 2).flatten(2).max(2).values
    power = torch.ceil(torch.log2(top / 448.0)).nan_to_num(neginf=-126.0).clamp(-126, 127)
    power = torch.where(top > 448.0 * torch.exp2(power), power + 1, power)
    power = torch.where((top <= 448.0 * torch.exp2(power - 1)) & (power > -126), power - 1, power)
    scale = torch.exp2(power)
    v = x / scale.repeat_interleave(group, 0)[:r].repeat_interleave(128, 1)[:, :c]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step, scale


def exact(case, seed):
    s = prepare(case, seed)
    r = case["rows"]
    if case["kind"] == "quant":
        q, scale = _codes64(s["x"].double(), case["block"])
        return {"q": q, "scale": scale}
    if case["kind"] == "rms":
        h, mod, w = s["h"].double(), s["mod"].double(), case["width"]
        m = torch.cat([mod[i:i + 1].expand(int(n), -1) for i, n in enumerate((s["cu_q"][1:] - s["cu_q"][:-1]).tolist())])
        if case["branch"]:
            h = h + m[:, 2 * w:] * s["y"].double()
        norm = h / (h.pow(2).sum(1, keepdim=True) / w + 1e-6).sqrt()
        q, scale = _codes64(norm * s["weight"].double() * (1 + m[:, w:2 * w]) + m[:, :w], 1)
        return {"h": h, "q": q, "scale": scale}
    if case["kind"] == "rope":
        hq, hk, dh = case["heads"], case["kv_heads"], case["dh"]
        tok = s["idx"].long()
        x = s["qkv"].double().view(r, hq + 2 * hk, dh)
        turned = x.clone()
        at = 0
        for a, d in enumerate(s["dims"]):
            for j in range(d // 2):
                ang = s["coord"][tok, a].double() * (s["step"][a] * s["theta"][a] ** (-2.0 * j / d))
                u, v = (at + j, at + j + d // 2) if case["halves"] else (at + 2 * j, at + 2 * j + 1)
                z = torch.polar(torch.ones_like(ang), ang)[:, None] * torch.complex(x[:, :hq + hk, u], x[:, :hq + hk, v])
                turned[:, :hq + hk, u], turned[:, :hq + hk, v] = z.real, z.imag
            at += d
        k, v = s["k"].double(), s["v"].double()
        k[tok] = turned[:, hq:hq + hk].reshape(r, -1)
        v[tok] = x[:, hq + hk:].reshape(r, -1)
        return {"q": turned[:, :hq].reshape(r, -1), "k": k, "v": v}
    n, k = case["out"], case["inner"]
    y = s["bias"].double().expand(r, n).clone()
    for kb in range(-(-k // 128)):
        c = slice(128 * kb, min(k, 128 * kb + 128))
        p = s["a"][:, c].double() @ s["w"][:, c].double().t()
        p *= torch.exp2(s["a_scale"][:, kb].double() - 127)[:, None]
        y += p * torch.exp2(s["w_scale"][:, kb].double() - 127).repeat_interleave(128)[:n]
    if case["act"]:
        y = y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    if case["to"] == "8":
        q, scale = _codes64(y, 1)
        return {"y": q, "scale": scale}
    return {"y": y}
