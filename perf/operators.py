"""Rotary positions, norms of queries and keys with the rotation, and differential attention, as cases that can be timed and compared.

These are what a denoising transformer runs between its fused q/k/v projection and its output projection.  A pass is one call of one
of the three operators on tensors that the program has in hand.  Every case is a dict of plain values:

kind "rope"       x_a' = A (x_a cos t - x_b sin t), x_b' = A (x_b cos t + x_a sin t) for every pair (a, b) of a head, t = position * frequency
kind "norm_rope"  an RMS norm or LayerNorm over each head of q and k, then the same rotation
kind "diff"       (softmax(q1 k1' / sqrt d) - lambda softmax(q2 k2' / sqrt d)) v, then an RMS norm over each head

listed()   sizes of the image, video and text layers of the configurations in tests/configs.py, single tokens, odd sizes
draw(rng)  other sizes, layouts, scalings, masks and types of the same ranges
own        False: the plain form in elementary torch operations; True: the library's kernels
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LAYOUTS = ("half", "interleaved")
SCALINGS = ("plain", "linear", "base", "parts")
ORIGINAL_LEN, SLOW_TURNS, FAST_TURNS = 4096.0, 1.0, 32.0


def _rows(kind, dtype, batch, l, heads, kv_heads, d, axes, layout="half", scaling="plain", factor=1.0, first=0, packed=False, norm="rms", **more):
    """axes: how many elements of a head each axis of positions rotates ("16,24,24"); first: the first position; packed: q and k are columns
    of one q/k/v buffer, as the fused projection leaves them."""
    c = dict(kind=kind, dtype=dtype, batch=batch, l=l, heads=heads, kv_heads=kv_heads, d=d, axes=axes, layout=layout, scaling=scaling, factor=factor,
             first=first, packed=packed, base=10000.0)
    if kind == "norm_rope":
        c["norm"] = norm
    c.update(more)
    return c


def _diff(dtype, batch, l, lk, heads, kv_heads, d, ragged=False, causal=False, packed=False):
    """d: width of one map's head (the values are 2 d wide); ragged: every sample has its own number of keys."""
    return dict(kind="diff", dtype=dtype, batch=batch, l=l, lk=lk, heads=heads, kv_heads=kv_heads, d=d, ragged=ragged, causal=causal, packed=packed)


def listed():
    cases = {
        # one new token of two sequences: the smallest call, nothing but latency
        "rope_token": _rows("rope", "bf16", 2, 1, 5, 5, 64, "64", layout="interleaved", first=1000),
        # 16 frames of 32 x 32 positions, a level-1 layer of a video model: frame, row and column each turn a part of the head
        "rope_video": _rows("rope", "bf16", 1, 16384, 10, 10, 64, "16,24,24"),
        # long sequence far behind the trained length, part of the head turned, frequencies scaled by parts, shared key heads, odd length
        "rope_far_f32": _rows("rope", "f32", 2, 5003, 8, 2, 80, "48", layout="interleaved", scaling="parts", factor=8.0, first=200000),
        # text tokens: 77 rows of two samples
        "norm_rope_text": _rows("norm_rope", "bf16", 2, 77, 10, 10, 64, "64", packed=True),
        # level 0 of the 768px model (96 x 96 positions, 320 channels): both halves of 5 differential heads, columns of the projection's output
        "norm_rope_768px": _rows("norm_rope", "bf16", 2, 9216, 10, 10, 32, "16,16", packed=True),
        # fp32, LayerNorm with offsets, wide heads, interpolated positions, odd length
        "norm_rope_f32": _rows("norm_rope", "f32", 1, 2311, 6, 3, 128, "64,64", layout="interleaved", scaling="linear", factor=4.0, norm="layer"),
        # one token of two sequences against thousands of keys, eight query heads to a key head: what generation step by step asks for
        "diff_token": _diff("bf16", 2, 1, 8190, 16, 2, 64, ragged=True),
        # image tokens against the text: few keys, padded to the longest prompt
        "diff_text": _diff("bf16", 2, 9216, 77, 5, 5, 32, ragged=True),
        # self-attention of level 0 of the 768px model: the largest case
        "diff_768px": _diff("bf16", 2, 9216, 9216, 5, 5, 32, packed=True),
        # self-attention of level 1 of the 768px model (48 x 48 positions, 640 channels)
        "diff_mid": _diff("bf16", 2, 2304, 2304, 5, 5, 64, packed=True),
        # a chunk of new frames against the frames so far, causal, wide heads that share keys, odd sizes
        "diff_causal_wide": _diff("bf16", 1, 1511, 6007, 8, 2, 128, causal=True),
        # fp32, an odd length, samples of different lengths
        "diff_f32": _diff("f32", 2, 577, 577, 4, 4, 64, ragged=True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _between(rng, low, high):
    """A whole number between low and high, spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(("rope", "norm_rope", "diff", "diff"))
    kv = rng.choice((1, 1, 2, 3, 4, 5, 8))
    heads = kv * rng.choice((1, 1, 2, 4))
    if kind == "diff":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        d = rng.choice((16, 32, 32, 40, 64, 64, 80, 96, 128))
        batch = rng.choice((1, 1, 2, 3))
        l = rng.choice((1, rng.randint(2, 12), _between(rng, 13, 9216), _between(rng, 13, 9216)))
        lk = _between(rng, 1, 65536 if l <= 12 else 9216)
        if rng.random() < 0.4:
            lk = l
        # at most the work of the largest listed case, fp32 (a sixteenth of the matrix rate) a sixteenth of it
        most = 2 * 9216 * 9216 * 5 * 32 // (16 if dtype == "f32" else 1)
        while batch * l * lk * heads * max(d, 32) > most:
            l, lk = (l + 1) // 2, (lk + 1) // 2
        return _diff(dtype, batch, l, lk, heads, kv, d, ragged=rng.random() < 0.4, causal=rng.random() < 0.4, packed=l == lk and rng.random() < 0.5)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    d = rng.choice((32, 40, 48, 64, 64, 72, 80, 96, 128))
    n = rng.choice((1, 1, 2, 3))
    turned = d if rng.random() < 0.6 else d // 2
    part = turned // n // 4 * 4
    dims = [part] * (n - 1) + [turned - part * (n - 1)]
    batch, l = rng.choice((1, 2, 3)), _between(rng, 1, 16384)
    while batch * l * (heads + kv) * d * (2 if dtype == "bf16" else 4) > 16384 * 20 * 64 * 2:
        l = (l + 1) // 2
    scaling = rng.choice(SCALINGS)
    more = dict(layout=rng.choice(LAYOUTS), scaling=scaling, factor=1.0 if scaling == "plain" else rng.choice((2.0, 4.0, 10.0)),
                first=_between(rng, 1, 1000000), packed=rng.random() < 0.5)
    if kind == "norm_rope":
        more["norm"] = rng.choice(("rms", "rms", "layer"))
    return _rows(kind, dtype, batch, l, heads, kv, d, ",".join(map(str, dims)), **more)


def _dims(case):
    return [int(n) for n in case["axes"].split(",")]


def _grid(case):
    """Positions [axes][l]: a running number on one axis; rows and columns of a grid (and frames of one) on two and three, as an image's tokens are numbered."""
    n, l, first = len(_dims(case)), case["l"], case["first"]
    i = torch.arange(l, device=DEVICE)
    if n == 1:
        axes = [i]
    else:
        w = max(1, math.isqrt(l if n == 2 else max(1, l // 16)))
        axes = [i // w, i % w] if n == 2 else [i // (w * w), i // w % w, i % w]
    return (torch.stack(axes) + first).to(torch.int32).contiguous()


def _frequencies(case):
    """(frequencies of the pairs in radians per position, axis of each, amplitude), in 64 bits."""
    freq, axis, s = [], [], case["factor"]
    for a, dim in enumerate(_dims(case)):
        base = case["base"]
        if case["scaling"] == "base" and dim > 2:
            base *= s ** (dim / (dim - 2))
        for i in range(dim // 2):
            f = base ** (-2 * i / dim)
            if case["scaling"] == "linear":
                f /= s
            if case["scaling"] == "parts":
                turns = ORIGINAL_LEN * f / (2 * math.pi)
                keep = min(1.0, max(0.0, (turns - SLOW_TURNS) / (FAST_TURNS - SLOW_TURNS)))
                f = f / s * (1 - keep) + f * keep
            freq.append(f)
            axis.append(a)
    return freq, axis, 0.1 * math.log(s) + 1 if case["scaling"] == "parts" else 1.0


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, mean=0.0, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, device=DEVICE, generator=g) * std + mean).to(dtype)

    b, l, h, kv, d = (case[n] for n in ("batch", "l", "heads", "kv_heads", "d"))
    s = dict(case=case)
    if case["kind"] == "diff":
        lk, w = case["lk"], 2 * d
        if case["packed"]:
            qkv = normal(b, l, (h + 2 * kv) * w, dtype=t)
            s["q"], s["k"], s["v"] = qkv[..., :h * w], qkv[..., h * w:(h + kv) * w], qkv[..., (h + kv) * w:]
        else:
            s["q"], s["k"], s["v"] = normal(b, l, h * w, dtype=t), normal(b, lk, kv * w, dtype=t), normal(b, lk, kv * w, dtype=t)
        s["lens"] = None
        if case["ragged"]:
            s["lens"] = torch.randint((lk + 1) // 2, lk + 1, (b,), device=DEVICE, generator=g).to(torch.int32)
        s["lambda"] = torch.rand(h, device=DEVICE, generator=g) * 0.6 + 0.2
        s["gain"] = normal(w, mean=1.0, std=0.1)
        s["eps"], s["scale"] = 1e-5, 0.8
        if own:
            from paper_2406_06911_amd import binding as B
            s["out"] = torch.empty(b, l, h * w, device=DEVICE, dtype=t)
            n = B.lib.ad_diff_attention_workspace_bytes(_type(case), b, l, lk, h, kv, d)
            s["work"] = torch.empty(max(n, 16), device=DEVICE, dtype=torch.uint8)
        return s
    std, mean = (1.0, 0.0) if case["kind"] == "rope" else (1.7, 0.2)
    if case["packed"]:
        qkv = normal(b, l, (h + 2 * kv) * d, mean=mean, std=std, dtype=t)
        s["q"], s["k"] = qkv[..., :h * d], qkv[..., h * d:(h + kv) * d]
    else:
        s["q"], s["k"] = normal(b, l, h * d, mean=mean, std=std, dtype=t), normal(b, l, kv * d, mean=mean, std=std, dtype=t)
    if case["kind"] == "norm_rope":
        s["q_gain"], s["k_gain"] = normal(d, mean=1.0, std=0.1), normal(d, mean=1.0, std=0.1)
        s["q_offset"], s["k_offset"] = (normal(d, std=0.1), normal(d, std=0.1)) if case["norm"] == "layer" else (None, None)
        s["eps"] = 1e-6
    s["positions"] = _grid(case)
    freq, axis, amplitude = _frequencies(case)
    if own:
        from paper_2406_06911_amd import binding as B
        s["rope"] = B.RopeCfg.make(_dims(case), layout=LAYOUTS.index(case["layout"]), base=case["base"], scaling=SCALINGS.index(case["scaling"]), factor=case["factor"],
                                   original_len=ORIGINAL_LEN, slow_turns=SLOW_TURNS, fast_turns=FAST_TURNS)
        s["table"] = torch.from_numpy(B.rope_table(s["rope"])).to(DEVICE)
        s["q_out"], s["k_out"] = torch.empty(b, l, h * d, device=DEVICE, dtype=t), torch.empty(b, l, kv * d, device=DEVICE, dtype=t)
    else:
        s["freq"], s["axis"] = torch.tensor(freq, device=DEVICE, dtype=torch.float64), torch.tensor(axis, device=DEVICE)
        s["amplitude"] = amplitude
    return s


def _type(case):
    return 1 if case["dtype"] == "bf16" else 0


# ---- the plain form ------------------------------------------------------------------------------------------------------------

def _turn(x, s):
    """x [b][l][heads][d] in 32 bits, its first elements rotated; the angles are formed in 64 bits, far positions need them."""
    case = s["case"]
    angle = s["positions"][s["axis"]].double().t() * s["freq"]                       # [l][pairs]
    cos, sin = ((f(angle) * s["amplitude"]).float()[None, :, None] for f in (torch.cos, torch.sin))
    n = 2 * s["freq"].numel()
    turned, rest = x[..., :n], x[..., n:]
    if case["layout"] == "half":
        a, b = turned[..., :n // 2], turned[..., n // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = turned[..., 0::2], turned[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _norm(x, gain, offset, s):
    if s["case"]["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * gain
    return y if offset is None else y + offset


def _plain_rows(s, name):
    case = s["case"]
    x = s[name].float().unflatten(-1, (-1, case["d"]))
    if case["kind"] == "norm_rope":
        x = _norm(x, s[name + "_gain"], s[name + "_offset"], s)
    return _turn(x, s).flatten(-2).to(TYPES[case["dtype"]])


def _plain_diff(s):
    case = s["case"]
    b, l, lk, h, kv, d = (case[n] for n in ("batch", "l", "lk", "heads", "kv_heads", "d"))
    group = h // kv
    q = s["q"].float().reshape(b, l, h, 2, d).permute(3, 0, 2, 1, 4).contiguous()                            # [map][b][h][l][d]
    k = s["k"].float().reshape(b, lk, kv, 2, d).permute(3, 0, 2, 4, 1).repeat_interleave(group, 2).contiguous()  # [map][b][h][d][lk]
    v = s["v"].float().reshape(b, lk, kv, 2 * d).permute(0, 2, 1, 3).repeat_interleave(group, 1).contiguous()
    lens = s["lens"] if s["lens"] is not None else torch.full((b,), lk, device=DEVICE)
    j = torch.arange(lk, device=DEVICE)
    seen = j[None, None] < lens[:, None, None]                                                               # [b][1 or l][lk]
    if case["causal"]:
        seen = seen & (j[None, None] <= torch.arange(l, device=DEVICE)[None, :, None] + (lens[:, None, None] - l))
    seen = seen[:, None]

    def weights(m):
        score = torch.matmul(q[m], k[m]) * d ** -0.5
        score = torch.where(seen, score, -math.inf)
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
        total = e.sum(-1, keepdim=True)
        return e / torch.where(total == 0, 1.0, total)                                                       # a row that sees nothing: zeros

    o = torch.matmul(weights(0) - s["lambda"][None, :, None, None] * weights(1), v)
    o = o / torch.sqrt((o * o).mean(-1, keepdim=True) + s["eps"]) * (s["gain"] * s["scale"])
    return o.permute(0, 2, 1, 3).reshape(b, l, h * 2 * d).to(TYPES[case["dtype"]])


# ---- the library's calls ---------------------------------------------------------------------------------------------------------

def _at(t):
    return None if t is None else t.data_ptr()


def _own_rows(s):
    from paper_2406_06911_amd import binding as B
    case, q, k = s["case"], s["q"], s["k"]
    stream = torch.cuda.current_stream().cuda_stream
    shape = (case["batch"], case["l"], case["heads"], case["kv_heads"], case["d"], q.stride(1), k.stride(1))
    qo, ko = s["q_out"], s["k_out"]
    to = (_at(qo), _at(ko), qo.stride(1), ko.stride(1), stream)
    if case["kind"] == "rope":
        B.check(B.lib.ad_rope_forward(_type(case), s["rope"], _at(s["table"]), _at(s["positions"]), 0, _at(q), _at(k), *shape, *to))
    else:
        B.check(B.lib.ad_qk_norm_rope_forward(_type(case), B.AD_NORM_LAYER if case["norm"] == "layer" else B.AD_NORM_RMS, s["rope"], _at(s["table"]),
                                              _at(s["positions"]), 0, _at(q), _at(k), _at(s["q_gain"]), _at(s["k_gain"]), _at(s["q_offset"]), _at(s["k_offset"]),
                                              s["eps"], *shape, *to))
    return {"q": qo, "k": ko}


def _own_diff(s):
    from paper_2406_06911_amd import binding as B
    case, q, k, v, out, work = s["case"], s["q"], s["k"], s["v"], s["out"], s["work"]
    B.check(B.lib.ad_diff_attention_forward(_type(case), _at(q), _at(k), _at(v), case["batch"], case["l"], case["lk"], case["heads"], case["kv_heads"], case["d"],
                                            q.stride(1), k.stride(1), v.stride(1), out.stride(1), _at(s["lens"]), int(case["causal"]), _at(s["lambda"]),
                                            _at(s["gain"]), s["eps"], s["scale"], _at(out), _at(work), work.numel(), torch.cuda.current_stream().cuda_stream))
    return {"out": out}


def run(s):
    if own:
        return _own_diff(s) if s["case"]["kind"] == "diff" else _own_rows(s)
    if s["case"]["kind"] == "diff":
        return {"out": _plain_diff(s)}
    return {"q": _plain_rows(s, "q"), "k": _plain_rows(s, "k")}


def _visible(case):
    """(query, key) pairs of one head, with every sample at its full length."""
    b, l, lk = case["batch"], case["l"], case["lk"]
    if not case["causal"]:
        return b * l * lk
    first = max(0, l - lk)                                                             # rows in front of it see nothing
    n = l - first
    return b * (n * (lk - l + first + 1) + n * (n - 1) // 2)


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    b, l, h, kv, d = (case[n] for n in ("batch", "l", "heads", "kv_heads", "d"))
    if case["kind"] == "diff":
        # two products with k and, the maps joined, one with v: 8 d operations for each pair of a query and a key it sees
        return {"bytes": 2 * d * es * b * (2 * l * h + 2 * case["lk"] * kv), "flops": 8 * d * h * _visible(case)}
    elements = b * l * (h + kv) * d
    turned = sum(_dims(case))
    return {"bytes": 2 * es * elements + 4 * l * len(_dims(case)), "flops": elements // d * (3 * turned + (4 * d if case["kind"] == "norm_rope" else 0))}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------------

def _exact_rows(s, name):
    case, n = s["case"], sum(_dims(s["case"]))
    x = s[name].double()
    x = x.reshape(*x.shape[:2], -1, case["d"])
    if case["kind"] == "norm_rope":
        mean = x.mean(-1, keepdim=True) if case["norm"] == "layer" else torch.zeros_like(x[..., :1])
        x = (x - mean) * (((x - mean) ** 2).mean(-1, keepdim=True) + s["eps"]).rsqrt()
        x = x * s[name + "_gain"].double()
        if s[name + "_offset"] is not None:
            x = x + s[name + "_offset"].double()
    freq, axis, amplitude = _frequencies(case)
    where = s["positions"].double().cpu()
    angle = torch.stack([where[a] * f for a, f in zip(axis, freq)], -1).to(DEVICE)     # [l][pairs]
    spin = torch.polar(torch.full_like(angle, amplitude), angle)[None, :, None]
    if case["layout"] == "half":
        z = torch.complex(x[..., :n // 2], x[..., n // 2:n]) * spin
        y = torch.cat([z.real, z.imag], -1)
    else:
        y = torch.view_as_real(torch.view_as_complex(x[..., :n].reshape(*x.shape[:-1], n // 2, 2).contiguous()) * spin).flatten(-2)
    return torch.cat([y, x[..., n:]], -1).flatten(-2)


def _exact_diff(s):
    case = s["case"]
    b, l, lk, h, kv, d = (case[n] for n in ("batch", "l", "lk", "heads", "kv_heads", "d"))
    out = torch.zeros(b, l, h * 2 * d, device=DEVICE, dtype=torch.float64)
    for i in range(b):
        n = lk if s["lens"] is None else int(s["lens"][i])
        start = max(0, l - n) if case["causal"] else 0                                   # rows in front of it see nothing
        if n == 0 or start >= l:
            continue
        for head in range(h):
            at = head // (h // kv) * 2 * d
            key, value = s["k"][i, :n, at:at + 2 * d].double(), s["v"][i, :n, at:at + 2 * d].double()
            query = s["q"][i, start:, head * 2 * d:(head + 1) * 2 * d].double()
            maps = []
            for m in (0, d):
                score = query[:, m:m + d] @ key[:, m:m + d].t() / math.sqrt(d)
                if case["causal"]:
                    hidden = torch.ones_like(score, dtype=torch.bool).triu(n - l + start + 1)
                    score = score.masked_fill(hidden, -math.inf)
                maps.append(torch.exp(score - torch.logsumexp(score, -1, keepdim=True)))
            o = maps[0] @ value - float(s["lambda"][head]) * (maps[1] @ value)
            o = o * ((o ** 2).mean(-1, keepdim=True) + s["eps"]).rsqrt() * s["gain"].double() * s["scale"]
            out[i, start:, head * 2 * d:(head + 1) * 2 * d] = o
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "diff":
        return {"out": _exact_diff(s)}
    return {"q": _exact_rows(s, "q"), "k": _exact_rows(s, "k")}
