"""Rotary positions and the norms of queries and keys in front of them, against the formulas in 64 bits.

Tolerances, from the roundings.  With u = 2^-24: the phase is cut at 2^-32 turn and converted to fp32 (2^-26 turn at most), together 9.5e-8 rad; sine and
cosine of the hardware are off by at most 1.3e-7 and multiplied by the amplitude (u); a rotated element is two products and a sum (3 u of each term).  So it is
off by at most (|x_a| + |x_b|) A (2.3e-7 + 4 u) = 4.7e-7 A (|x_a| + |x_b|), and by half a step of its own type, finfo.eps / 2.  A norm over d <= 128 elements:
the mean of the squares is off by at most (16 + 6 + 2) u of itself (a lane's chain, the lanes' tree, 1 / d), its root by half of that, the hardware's root by 2 u,
the two products by 2 u: 16 u.  A mean that is taken off is off by 24 u of mean |x|.  All of these are doubled by nothing: they are bounds, not estimates."""
import math

import numpy as np
import pytest
import torch

import synthetic_inputs as SI
from gpu_util import DEV, dev_f32, p, quantize, stream_ptr, tdtype
from paper_2406_06911_amd import binding as B

pytestmark = pytest.mark.gpu
lib = B.lib
DT = [B.AD_F32, B.AD_BF16]
U = 2.0 ** -24


def freqs(cfg):
    f, axis = [], []
    for a in range(cfg.n_axes):
        dim, base = cfg.axis_dims[a], cfg.base
        if cfg.scaling == B.AD_ROPE_BASE and dim > 2:
            base = base * cfg.factor ** (dim / (dim - 2))
        for i in range(dim // 2):
            v = base ** (-2.0 * i / dim)
            if cfg.scaling == B.AD_ROPE_LINEAR:
                v /= cfg.factor
            if cfg.scaling == B.AD_ROPE_PARTS:
                t = min(1.0, max(0.0, (cfg.original_len * v / (2 * math.pi) - cfg.slow_turns) / (cfg.fast_turns - cfg.slow_turns)))
                v = v / cfg.factor * (1 - t) + v * t
            f.append(v)
            axis.append(a)
    amp = cfg.amplitude or (0.1 * math.log(cfg.factor) + 1 if cfg.scaling == B.AD_ROPE_PARTS else 1.0)
    return np.array(f), np.array(axis), amp


def reference(x, cfg, pos, norm=None, gain=None, offset=None, eps=0.0):
    """x [b][l][heads][d] float64, pos [b][axes][l]; returns the result and the bound on what the kernel's arithmetic may be off by."""
    err = np.zeros_like(x)
    if norm is not None:
        mean = x.mean(-1, keepdims=True) if norm == B.AD_NORM_LAYER else 0.0
        r = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
        g = 1.0 if gain is None else gain.astype(np.float64)
        y = (x - mean) * r * g
        err = 16 * U * np.abs(y)
        if norm == B.AD_NORM_LAYER:
            err = err + 24 * U * np.abs(x).mean(-1, keepdims=True) * r * (np.abs(g) + np.abs(y)) + U * np.abs(y)
        x = y if offset is None else y + offset.astype(np.float64)
        err = err + U * np.abs(x)
    if cfg is None:
        return x, err
    f, axis, amp = freqs(cfg)
    n = 2 * len(f)
    angle = pos[:, axis, :].astype(np.float64).transpose(0, 2, 1) * f             # [b][l][pairs]
    co, si = (amp * np.cos(angle))[:, :, None], (amp * np.sin(angle))[:, :, None]
    ia, ib = (np.arange(n // 2), np.arange(n // 2) + n // 2) if cfg.layout == B.AD_ROPE_HALF else (np.arange(0, n, 2), np.arange(1, n, 2))
    out, eo = x.copy(), err.copy()
    xa, xb, ea, eb = x[..., ia], x[..., ib], err[..., ia], err[..., ib]
    out[..., ia], out[..., ib] = xa * co - xb * si, xb * co + xa * si
    # positions up to 2^31: the 64-bit angle of this reference is itself off by 2^-53 of the angle, twice (frequency and product)
    far = 2.0 ** -52 * np.abs(angle)[:, :, None]
    both = (4.7e-7 + far) * amp * (np.abs(xa) + np.abs(xb)) + amp * (ea + eb)
    eo[..., ia], eo[..., ib] = both, both
    return out, eo


def check(got, ref, err, dtype):
    half_step = torch.finfo(tdtype(dtype)).eps / 2
    bound = err + half_step * (np.abs(ref) + err) + 1e-37
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], ref[bad][:3], bound[bad][:3])


def run(dtype, cfg, b, l, heads, kv, d, norm=None, pos=None, per_sample=False, pad=(0, 0), shift=0, in_place=False, gains=True, eps=1e-6, seed=0, scale=1.0, stream=None):
    """pad: elements behind the heads of a row of q and k; shift: elements in front of the first one."""
    n_axes = cfg.n_axes if cfg is not None else 1
    if pos is None:
        pos = np.stack([(np.arange(n_axes * l).reshape(n_axes, l) * (7 + s) + 3 * s) % 1237 for s in range(b)])
        if not per_sample:
            pos = np.repeat(pos[:1], b, 0)
    pos = pos.astype(np.int32)
    dpos = torch.from_numpy(np.ascontiguousarray(pos if per_sample else pos[0])).to(DEV)
    table = torch.from_numpy(B.rope_table(cfg)).to(DEV) if cfg is not None else None
    host, src, out, gain, offset = [], [], [], [], []
    for t, (h, extra) in enumerate(((heads, pad[0]), (kv, pad[1]))):
        x = quantize(SI.make_array((b, l, max(h, 1), d), 300 + seed + t) * scale + (0.2 if norm is not None else 0.0), dtype)
        host.append(x.astype(np.float64))
        ld = h * d + extra
        flat = torch.full((b * l * ld + shift + 64,), 77.0, device=DEV, dtype=tdtype(dtype))
        if h:
            flat[shift:shift + b * l * ld].view(b, l, ld)[..., :h * d] = torch.from_numpy(x).to(DEV).to(tdtype(dtype)).reshape(b, l, h * d)
        src.append(flat)
        out.append(flat if in_place else torch.full_like(flat, 55.0))
        gain.append(np.float32(1 + SI.make_array((d,), 320 + t, 0.2)) if norm is not None and gains else None)
        offset.append(SI.make_array((d,), 330 + t, 0.2).astype(np.float32) if norm == B.AD_NORM_LAYER and gains else None)
    at = [x.data_ptr() + shift * x.element_size() for x in src]
    to = [x.data_ptr() + shift * x.element_size() for x in out]
    ld = [heads * d + pad[0], kv * d + pad[1]]
    dg = [dev_f32(x) if x is not None else None for x in gain + offset]
    torch.cuda.synchronize()
    s = stream_ptr(stream)
    if norm is None:
        B.check(lib.ad_rope_forward(dtype, cfg, p(table), p(dpos), int(per_sample), at[0], at[1] if kv else None, b, l, heads, kv, d, ld[0], ld[1], to[0], to[1] if kv else None, ld[0], ld[1], s))
    else:
        B.check(lib.ad_qk_norm_rope_forward(dtype, norm, cfg, p(table), p(dpos), int(per_sample), at[0], at[1] if kv else None, p(dg[0]), p(dg[1]), p(dg[2]), p(dg[3]), eps,
                                            b, l, heads, kv, d, ld[0], ld[1], to[0], to[1] if kv else None, ld[0], ld[1], s))
    torch.cuda.synchronize()
    for t, h in enumerate((heads, kv)):
        if not h:
            continue
        rest = 77.0 if in_place else 55.0                                # what is in front, behind and between the heads stays as it was
        flat = out[t].float()
        body = flat[shift:shift + b * l * ld[t]].view(b, l, ld[t])
        assert (flat[:shift] == rest).all() and (flat[shift + b * l * ld[t]:] == rest).all() and (body[..., h * d:] == rest).all()
        got = body[..., :h * d].reshape(b, l, h, d).double().cpu().numpy()
        ref, err = reference(host[t], cfg, pos, norm, gain[t], offset[t], eps)
        check(got, ref, err, dtype)
    return out


HALF, INTER = B.AD_ROPE_HALF, B.AD_ROPE_INTERLEAVED
# batch, l, heads, kv heads, d, axes: every width of access (pairs and heads that are multiples of 8, 4, 2 and of nothing), whole and partial heads,
# one to three axes, one token, odd lengths, heads that are not a multiple of what a lane keeps in flight
SHAPES = [(1, 1, 1, 0, 64, [64]), (2, 1, 5, 5, 64, [64]), (2, 77, 10, 10, 64, [64]), (1, 33, 3, 1, 128, [128]), (2, 19, 8, 2, 80, [48]), (1, 45, 5, 5, 32, [16, 16]),
          (1, 64, 10, 10, 64, [16, 24, 24]), (3, 7, 4, 1, 72, [36]), (1, 13, 7, 7, 40, [20]), (1, 9, 2, 1, 7, [2]), (2, 5, 3, 3, 33, [30]), (1, 21, 12, 4, 96, [32, 32, 32]),
          (1, 3, 2, 2, 2, [2]), (1, 5, 1, 1, 1, []), (1, 4099, 1, 1, 8, [4]), (1, 600, 40, 40, 128, [60, 66]), (2, 11, 2, 2, 128, [2, 2, 2])]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("layout", [HALF, INTER], ids=["half", "interleaved"])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[5]], ids=str)
def test_rope(dtype, layout, shape):
    b, l, heads, kv, d, axes = shape
    run(dtype, B.RopeCfg.make(axes, layout=layout), b, l, heads, kv, d, per_sample=b > 1)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("norm", [B.AD_NORM_RMS, B.AD_NORM_LAYER], ids=["rms", "layer"])
@pytest.mark.parametrize("layout", [HALF, INTER], ids=["half", "interleaved"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_qk_norm_rope(dtype, norm, layout, shape):
    b, l, heads, kv, d, axes = shape
    run(dtype, B.RopeCfg.make(axes, layout=layout) if axes else None, b, l, heads, kv, d, norm=norm)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("norm", [None, B.AD_NORM_RMS, B.AD_NORM_LAYER], ids=["none", "rms", "layer"])
@pytest.mark.parametrize("pad,shift,in_place", [((320, 576), 0, False), ((8, 8), 0, True), ((3, 5), 0, False), ((4, 4), 4, False), ((2, 2), 2, True), ((0, 0), 1, False)], ids=str)
def test_rows_strides_and_alignment(dtype, norm, pad, shift, in_place):
    run(dtype, B.RopeCfg.make([24, 40], layout=INTER), 2, 21, 5, 3, 64, norm=norm, pad=pad, shift=shift, in_place=in_place, gains=shift != 2)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("scaling,factor", [(B.AD_ROPE_LINEAR, 4.0), (B.AD_ROPE_BASE, 8.0), (B.AD_ROPE_PARTS, 8.0), (B.AD_ROPE_PARTS, 1.0)])
def test_scaled_frequencies(dtype, scaling, factor):
    cfg = B.RopeCfg.make([64, 2], scaling=scaling, factor=factor, original_len=4096.0, slow_turns=1.0, fast_turns=32.0)
    pos = np.stack([np.stack([np.arange(50) * 999, np.arange(50) - 25])])
    run(dtype, cfg, 1, 50, 3, 3, 80, pos=pos)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("layout", [HALF, INTER], ids=["half", "interleaved"])
def test_far_and_negative_positions(dtype, layout):
    pos = np.array([[[0, -1, 1, 2 ** 31 - 1, -2 ** 31, 1000003, -1000003, 2 ** 24 + 1, -2 ** 24 - 1]]], np.int64)
    run(dtype, B.RopeCfg.make([64], layout=layout, base=1000000.0, amplitude=0.75), 1, 9, 2, 2, 64, pos=pos)


@pytest.mark.parametrize("dtype", DT)
def test_turning_back_gives_what_was_there(dtype):
    """Negative positions turn the other way: two passes are the identity up to the roundings of both."""
    cfg, d, l = B.RopeCfg.make([48]), 64, 37
    x = torch.randn(1, l, d, device=DEV, generator=torch.Generator(DEV).manual_seed(3)).to(tdtype(dtype))
    table = torch.from_numpy(B.rope_table(cfg)).to(DEV)
    pos = torch.arange(l, device=DEV, dtype=torch.int32) * 1001
    there, back = torch.empty_like(x), torch.empty_like(x)
    neg = -pos
    B.check(lib.ad_rope_forward(dtype, cfg, p(table), p(pos), 0, p(x), None, 1, l, 1, 0, d, d, 0, p(there), None, d, 0, stream_ptr()))
    B.check(lib.ad_rope_forward(dtype, cfg, p(table), p(neg), 0, p(there), None, 1, l, 1, 0, d, d, 0, p(back), None, d, 0, stream_ptr()))
    torch.cuda.synchronize()
    half = torch.finfo(tdtype(dtype)).eps / 2
    # each pass is off by half a step of an element of size |(x_a, x_b)| and by 4.7e-7 of |x_a| + |x_b|
    size = torch.sqrt(x.double()[..., :24] ** 2 + x.double()[..., 24:48] ** 2)
    diff = (back.double() - x.double()).abs()
    bound = (2.0 * half + 2 * 4.7e-7) * 1.5 * size * 1.01
    assert (diff[..., :24] <= bound).all() and (diff[..., 24:48] <= bound).all()
    assert (diff[..., 48:] == 0).all()


@pytest.mark.parametrize("norm", [B.AD_NORM_RMS, B.AD_NORM_LAYER], ids=["rms", "layer"])
def test_norm_of_constant_and_zero_heads(norm):
    """A head of zeros stays zero, a constant one has no variance: nothing is divided by zero."""
    d, cfg = 64, None
    x = torch.zeros(1, 3, d, device=DEV)
    x[0, 1] = 5.0
    x[0, 2] = torch.arange(d, device=DEV).float()
    out = torch.full_like(x, float("nan"))
    B.check(lib.ad_qk_norm_rope_forward(B.AD_F32, norm, cfg, None, None, 0, p(x), None, None, None, None, None, 1e-6, 1, 3, 1, 0, d, d, 0, p(out), None, d, 0, stream_ptr()))
    torch.cuda.synchronize()
    ref, err = reference(x.double().cpu().numpy()[:, :, None], None, None, norm, eps=1e-6)
    check(out.double().cpu().numpy()[:, :, None], ref, err + (24 * U * 5 * 1e3 if norm == B.AD_NORM_LAYER else 0), B.AD_F32)


def test_nan_and_infinity_stay_in_their_head():
    d, cfg = 64, B.RopeCfg.make([64])
    table = torch.from_numpy(B.rope_table(cfg)).to(DEV)
    x = torch.randn(1, 4, 3 * d, device=DEV)
    clean = x.clone()
    x[0, 1, 7], x[0, 2, d + 1] = float("nan"), float("inf")
    pos = torch.arange(4, device=DEV, dtype=torch.int32)
    outs = []
    for t in (x, clean):
        o = torch.empty_like(t)
        B.check(lib.ad_qk_norm_rope_forward(B.AD_F32, B.AD_NORM_RMS, cfg, p(table), p(pos), 0, p(t), None, None, None, None, None, 1e-6, 1, 4, 3, 0, d, 3 * d, 0, p(o), None, 3 * d, 0, stream_ptr()))
        outs.append(o)
    torch.cuda.synchronize()
    same = (outs[0] == outs[1]).view(4, 3, d).all(-1).cpu()
    want = torch.ones(4, 3, dtype=torch.bool)
    want[1, 0] = want[2, 1] = False
    assert (same == want).all()


def test_captured_and_replayed_on_another_stream():
    cfg, d, l, h = B.RopeCfg.make([32, 32]), 64, 130, 6
    table = torch.from_numpy(B.rope_table(cfg)).to(DEV)
    pos = torch.stack([torch.arange(l) // 12, torch.arange(l) % 12]).to(torch.int32).to(DEV)
    q, k = (torch.randn(1, l, h * d, device=DEV).bfloat16() for _ in range(2))
    gain = 1 + 0.1 * torch.randn(d, device=DEV)
    qo, ko, qe, ke = (torch.empty_like(q) for _ in range(4))

    def call(a, b, s):
        B.check(lib.ad_qk_norm_rope_forward(B.AD_BF16, B.AD_NORM_RMS, cfg, p(table), p(pos), 0, p(q), p(k), p(gain), p(gain), None, None, 1e-6, 1, l, h, h, d, h * d, h * d, p(a), p(b),
                                            h * d, h * d, stream_ptr(s)))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(qo, ko, side)
    for n in range(3):
        q.copy_(torch.randn(1, l, h * d, device=DEV))
        pos.add_(17)
        call(qe, ke, None)
        torch.cuda.synchronize()
        qo.fill_(9); ko.fill_(9)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qo, qe) and torch.equal(ko, ke)
