"""Differential attention against the formula in 64 bits.

Tolerances, element by element, from the roundings (u = 2^-24).  A score is a sum of d products held in fp32: off by at most (d + 4) u sum |q||k| / sqrt d, d the
term that covers every order of summation; the exponential's argument is that score times log2 e less a reference, off by 3 u of their sizes more, and the
exponential by 2 u.  With e the largest of these over a row's keys, a map's weights are off by a factor within 1 +- 2 e (numerator and denominator), its sums by the number of
terms that follow each other in one register, at most 16 + lk / 16 times u.  bf16 rounds each weight, once: finfo(bf16).eps / 2 of itself, 2^-8, and a
sum of such weights is off by as much of itself at most, which moves the quotient by 2^-8 of the row.  So a map's row is off by
(2 e + (lk / 16 + 24) u [+ 2^-8]) sum p |v| [+ 2^-8 |sum p v|], the difference by the first map's plus |lambda| times the second's, and the result by half a step of its type more.
The norm divides by the row's root mean square: the relative error of that root is at most the norm of the row's errors over the norm of the row."""
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


def reference(dtype, q, k, v, lam, lens, causal, gain, eps, scale):
    """q [b][l][h][2][d], k [b][lk][kv][2][d], v [b][lk][kv][2d] in float64; returns (out [b][l][h][2d], bound)."""
    b, l, h, _, d = q.shape
    lk, kv = k.shape[1], k.shape[2]
    out, bound = np.zeros((b, l, h, 2 * d)), np.zeros((b, l, h, 2 * d))
    half = torch.finfo(tdtype(dtype)).eps / 2
    for i in range(b):
        n = lk if lens is None else min(max(int(lens[i]), 0), lk)
        for head in range(h):
            g = head // (h // kv)
            o, err = np.zeros((l, 2 * d)), np.zeros((l, 2 * d))
            for m, factor in ((0, 1.0), (1, -float(lam[head]))):
                if n == 0:
                    continue
                s = q[i, :, head, m] @ k[i, :n, g, m].T / np.sqrt(d)
                size = np.abs(q[i, :, head, m]) @ np.abs(k[i, :n, g, m]).T / np.sqrt(d)
                seen = np.ones((l, n), bool)
                if causal:
                    seen = np.arange(n)[None] <= np.arange(l)[:, None] + (n - l)
                s = np.where(seen, s, -np.inf)
                top = s.max(-1, keepdims=True)
                top = np.where(np.isfinite(top), top, 0.0)
                w = np.exp(s - top)
                total = w.sum(-1, keepdims=True)
                w = w / np.where(total == 0, 1.0, total)
                # an argument far below the reference belongs to a weight that hardly counts: its error is weighted with it
                e = ((d + 4) * U * size + 3 * U * (np.abs(np.where(seen, s, 0.0)) + np.abs(top)) * 1.5 + 2 * U) * seen
                rel = e + (w * e).sum(-1, keepdims=True)
                vv = np.abs(v[i, :n, g])
                o += factor * (w @ v[i, :n, g])
                if dtype == B.AD_BF16:
                    err += abs(factor) * 2.0 ** -8 * np.abs(w @ v[i, :n, g])
                err += abs(factor) * ((w * (rel + (lk / 16 + 24) * U + (2.0 ** -8 if dtype == B.AD_BF16 else 0.0))) @ vv)
            err += 6 * U * np.abs(o)
            if gain is not None:
                r = 1.0 / np.sqrt((o * o).mean(-1, keepdims=True) + eps)
                gs = gain.astype(np.float64) * scale
                off = np.linalg.norm(err, axis=-1, keepdims=True) / np.maximum(np.linalg.norm(o, axis=-1, keepdims=True), 1e-300)
                off = np.minimum(off, 1.0) * (r * r * (o * o).mean(-1, keepdims=True))   # eps in the root holds it still
                # a row whose own error is a part x of it moves the root by a factor 1 / (1 - x) at most
                err = np.abs(gs) * r * (err + np.abs(o) * (off + 16 * U)) / np.maximum(1.0 - off, 0.25)
                o = o * r * gs
            else:
                o, err = o * scale, err * abs(scale)
            out[i, :, head], bound[i, :, head] = o, err + half * (np.abs(o) + err) + 1e-37
    return out, bound


class Case:
    def __init__(self, dtype, b, l, lk, heads, kv, d, lens=None, causal=False, norm=True, seed=0, qscale=1.0, pad=0, packed=False, lam=None):
        self.dtype, self.shape = dtype, (b, l, lk, heads, kv, d)
        self.causal, self.eps, self.scale = causal, 1e-5, 0.8
        t, w = tdtype(dtype), 2 * d
        make = lambda s, n, f=1.0: quantize(SI.make_array(s, 700 + seed + n) * f, dtype)
        self.hq, self.hk, self.hv = make((b, l, heads * w), 0, qscale), make((b, lk, kv * w), 1), make((b, lk, kv * w), 2)
        if packed:
            assert l == lk
            buf = torch.full((b, l, (heads + 2 * kv) * w + pad), 3.0, device=DEV, dtype=t)
            self.q, self.k, self.v = buf[..., :heads * w], buf[..., heads * w:(heads + kv) * w], buf[..., (heads + kv) * w:(heads + 2 * kv) * w]
        else:
            self.q, self.k, self.v = (torch.full((b, n, c * w + pad), float("nan"), device=DEV, dtype=t)[..., :c * w] for n, c in ((l, heads), (lk, kv), (lk, kv)))
        for to, x in ((self.q, self.hq), (self.k, self.hk), (self.v, self.hv)):
            to.copy_(torch.from_numpy(x))
        self.out_all = torch.full((b * l + 2, heads * w + pad), 55.0, device=DEV, dtype=t)
        self.out = self.out_all[1:-1].view(b, l, -1)[..., :heads * w]
        self.lens = None if lens is None else torch.tensor(lens, device=DEV, dtype=torch.int32)
        self.hlens = lens
        self.hlam = np.float32(np.linspace(0.2, 0.8, heads)) if lam is None else np.float32(lam)
        self.lam = dev_f32(self.hlam)
        self.hgain = np.float32(1 + 0.2 * SI.make_array((w,), 710 + seed)) if norm else None
        self.gain = dev_f32(self.hgain) if norm else None
        n = lib.ad_diff_attention_workspace_bytes(dtype, b, l, lk, heads, kv, d)
        self.work = torch.full((n // 4 + 4,), float("nan"), device=DEV)       # what a workspace holds before a call does not matter
        self.work_bytes = n

    def call(self, out=None, work=True, stream=None):
        b, l, lk, heads, kv, d = self.shape
        out = self.out if out is None else out
        B.check(lib.ad_diff_attention_forward(self.dtype, p(self.q), p(self.k), p(self.v), b, l, lk, heads, kv, d, self.q.stride(1), self.k.stride(1), self.v.stride(1), out.stride(1),
                                              p(self.lens), int(self.causal), p(self.lam), p(self.gain), self.eps, self.scale, p(out), p(self.work) if work else None,
                                              self.work_bytes if work else 0, stream_ptr(stream)))
        return out

    def reference(self):
        b, l, lk, heads, kv, d = self.shape
        f = lambda x, n, c: x.astype(np.float64).reshape(b, n, c, -1)
        return reference(self.dtype, f(self.hq, l, heads).reshape(b, l, heads, 2, d), f(self.hk, lk, kv).reshape(b, lk, kv, 2, d), f(self.hv, lk, kv), self.hlam, self.hlens, self.causal,
                         self.hgain, self.eps, self.scale)

    def check(self, work=True):
        torch.cuda.synchronize()
        self.call(work=work)
        torch.cuda.synchronize()
        b, l, lk, heads, kv, d = self.shape
        ref, bound = self.reference()
        got = self.out.double().cpu().numpy().reshape(ref.shape)
        bad = ~(np.abs(got - ref) <= bound)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], ref[bad][:3], bound[bad][:3])
        frame = self.out_all.clone()
        frame[1:-1].view(b, l, -1)[..., :heads * 2 * d] = 55.0
        assert (frame == 55.0).all()                                          # in front of, behind and between the rows nothing is written
        return got, ref


# batch, l, lk, heads, kv heads, d.  Lengths of one, tiles' borders and one beside them, heads that share keys, every width of head
SHAPES = [(1, 1, 1, 1, 1, 64), (2, 1, 5, 3, 3, 32), (1, 2, 64, 4, 2, 64), (2, 17, 33, 2, 1, 16), (1, 32, 32, 1, 1, 64), (1, 31, 63, 2, 2, 64), (1, 33, 65, 2, 2, 32), (1, 65, 77, 5, 5, 32),
          (2, 64, 128, 2, 2, 64), (1, 127, 129, 1, 1, 128), (1, 129, 127, 2, 2, 64), (1, 130, 300, 2, 1, 128), (2, 200, 200, 3, 3, 64), (1, 257, 511, 1, 1, 32), (3, 9, 100, 6, 2, 40),
          (1, 50, 90, 2, 2, 96), (1, 70, 70, 1, 1, 80), (1, 21, 48, 2, 1, 8), (1, 40, 66, 4, 4, 72), (1, 16, 31, 3, 1, 112), (1, 300, 1, 2, 2, 64), (1, 640, 640, 1, 1, 64), (1, 576, 577, 2, 2, 32)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(dtype, shape):
    Case(dtype, *shape).check()


@pytest.mark.parametrize("shape", [(1, 20, 40, 2, 1, 4), (2, 7, 19, 1, 1, 12), (1, 33, 34, 2, 2, 20), (1, 18, 50, 1, 1, 100), (1, 12, 70, 1, 1, 124)], ids=str)
def test_fp32_head_widths_of_four(shape):
    Case(B.AD_F32, *shape).check()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("shape", [(1, 1, 1500, 1, 1, 64), (2, 1, 4097, 16, 2, 64), (1, 3, 2049, 4, 4, 32), (1, 5, 3000, 8, 1, 128), (1, 40, 1025, 2, 2, 64), (2, 1, 600, 2, 1, 40), (1, 100, 2000, 1, 1, 96)], ids=str)
@pytest.mark.parametrize("work", [True, False], ids=["shared out", "no workspace"])
def test_few_rows_and_many_keys(dtype, shape, work):
    c = Case(dtype, *shape)
    assert c.work_bytes > 0
    c.check(work)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("shape", [(1, 64, 64, 2, 2, 64), (1, 100, 37, 2, 2, 32), (1, 37, 100, 4, 1, 64), (2, 1, 700, 4, 2, 64), (1, 200, 333, 2, 1, 128), (1, 129, 2, 1, 1, 64), (1, 300, 300, 3, 3, 32),
                                   (1, 6, 3000, 2, 1, 64)], ids=str)
@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
def test_causal(dtype, shape, norm):
    c = Case(dtype, *shape, causal=True, norm=norm)
    got, ref = c.check()
    b, l, lk = shape[:3]
    if l > lk:
        assert (got[:, :l - lk] == 0).all()                                   # rows in front of the first key see nothing


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("l,lk,lens,d", [(33, 130, [0, 1, 129, 130], 64), (1, 900, [0, 900, 257, 16], 64), (70, 70, [70, 64, 0, 33], 32), (2, 5000, [1, 0, 4999, 300], 128), (100, 77, [77, 500, -3, 12], 32)])
def test_lengths_and_what_lies_behind_them(dtype, causal, l, lk, lens, d):
    """Keys and values behind a sample's length are NaN and infinity; lengths outside 0 .. lk are held to it."""
    c = Case(dtype, len(lens), l, lk, 4, 2, d, lens=lens, causal=causal)
    for i, n in enumerate(lens):
        n = min(max(n, 0), lk)
        c.k[i, n:] = float("nan")
        c.v[i, n:] = float("nan")
        c.v[i, n:, ::3] = float("inf")
        c.k[i, n:, ::5] = -float("inf")
    got, _ = c.check()
    for i, n in enumerate(lens):
        if n <= 0:
            assert (got[i] == 0).all()
    c.check(work=False)


# enough rows for tiles of 128 and of 64, every class of head width, keys that end inside a tile and beside one, a key more than lies in LDS at once
@pytest.mark.parametrize("d", [16, 32, 48, 64, 80, 96, 128])
@pytest.mark.parametrize("l,lk,causal", [(3900, 130, False), (3900, 320, True), (2000, 193, False), (2000, 64, True), (3900, 97, False), (3900, 96, False), (6700, 130, False)])
def test_tiles_of_many_rows(d, l, lk, causal):
    Case(B.AD_BF16, 1, l, lk, 5, 5, d, causal=causal, lens=[lk - 1] if lk == 193 else None).check()


@pytest.mark.parametrize("d", [32, 64, 128])
def test_many_rows_that_share_keys(d):
    """Rows of one tile are queries and heads: 3 queries x 3 heads, tiles that end inside a query."""
    Case(B.AD_BF16, 2, 1001, 200, 9, 3, d, causal=True, lens=[200, 77]).check()


@pytest.mark.parametrize("d,nan_at", [(32, 40), (64, 70), (32, 130), (128, 130)])
def test_what_lies_behind_the_keys_of_a_tensor(d, nan_at):
    """k and v are the front part of larger buffers whose next rows are NaN: nothing behind the last key is used."""
    c = Case(B.AD_BF16, 1, 200, nan_at, 2, 2, d)
    for name in ("k", "v"):
        whole = torch.full((1, nan_at + 200, 4 * d), float("nan"), device=DEV, dtype=torch.bfloat16)
        whole[:, :nan_at] = getattr(c, name)
        setattr(c, name, whole[:, :nan_at])
    c.check()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("pad,packed", [(0, True), (64, True), (8, False), (200, False)])
def test_strides(dtype, pad, packed):
    Case(dtype, 2, 90, 90 if packed else 140, 4, 2 if not packed else 4, 64, pad=pad, packed=packed).check()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("lam", [[0.0, 0.0], [1.0, -0.5], [3.0, 0.1]], ids=str)
@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
def test_lambda(dtype, lam, norm):
    Case(dtype, 1, 40, 200, 2, 2, 64, lam=lam, norm=norm).check()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("shape", [(1, 40, 700, 2, 1, 64), (1, 1, 3000, 2, 1, 32), (1, 130, 300, 1, 1, 128)], ids=str)
@pytest.mark.parametrize("ramp", [40.0, -40.0, 400.0], ids=str)
def test_maximum_that_rises_and_falls_along_the_keys(dtype, shape, ramp):
    """Scores that grow or shrink by hundreds along the keys, in opposite directions in the two maps."""
    c = Case(dtype, *shape, norm=False)
    b, l, lk, h, kv, d = shape
    slope = torch.linspace(-1, 1, lk, device=DEV)
    q, k = c.q.view(b, l, h, 2, d), c.k.view(b, lk, kv, 2, d)
    for m, sign in ((0, 1.0), (1, -1.0)):
        q[:, :, :, m, 0] = d ** 0.5
        k[:, :, :, m, 0] = sign * ramp * slope[None, :, None]
    c.hq, c.hk = c.q.float().cpu().numpy(), c.k.float().cpu().numpy()
    c.check()


@pytest.mark.parametrize("dtype", DT)
def test_sharp_weights(dtype):
    Case(dtype, 1, 100, 400, 2, 2, 64, qscale=8.0).check()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("l,lk", [(40, 300), (1, 3000)])
def test_scores_of_the_lowest_values(dtype, l, lk):
    """Rows of keys at the type's lowest finite values: scores of minus infinity have no weight, and a row of nothing else is zero."""
    c = Case(dtype, 1, l, lk, 1, 1, 64, norm=False)
    low = torch.finfo(tdtype(dtype)).min
    c.q.abs_()
    c.q.add_(1.0)
    c.k[:, ::2] = low
    c.hq, c.hk = c.q.float().cpu().numpy(), c.k.float().cpu().numpy()
    torch.cuda.synchronize()
    c.call()
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        ref = Case.__new__(Case)
        ref.__dict__ = dict(c.__dict__, shape=(1, l, (lk) // 2, 1, 1, 64), hk=c.hk[:, 1::2], hv=c.hv[:, 1::2])
        want, bound = ref.reference()
    got = c.out.double().cpu().numpy().reshape(want.shape)
    assert (np.abs(got - want) <= bound + (lk / 16) * U * np.abs(c.hv).max()).all()
    c.k.fill_(low)
    c.call()
    torch.cuda.synchronize()
    assert (c.out == 0).all()


@pytest.mark.parametrize("dtype", DT)
def test_a_bad_query_stays_in_its_row(dtype):
    c = Case(dtype, 1, 50, 90, 4, 2, 64)
    clean = c.call().clone()
    c.q[0, 7, 3] = float("nan")
    c.q[0, 20, 128 + 5] = float("inf")
    dirty = c.call().clone()
    torch.cuda.synchronize()
    same = (clean == dirty).view(50, 4, 128).all(-1).cpu()
    want = torch.ones(50, 4, dtype=torch.bool)
    want[7, 0] = want[20, 1] = False
    assert (same == want).all()


@pytest.mark.parametrize("dtype", DT)
def test_more_than_four_gigabytes_of_keys(dtype):
    """Rows of the cache far apart: offsets of the last keys pass 32 bits."""
    ld, lk = (65536, 40000) if dtype == B.AD_BF16 else (32768, 40000)
    c = Case(dtype, 1, 3, lk, 2, 1, 32)
    big = torch.empty(lk, ld, device=DEV, dtype=tdtype(dtype))
    for name, at in (("k", 0), ("v", ld - 64)):
        view = big[:, at:at + 64].unsqueeze(0)
        view.copy_(getattr(c, name))
        setattr(c, name, view)
    c.check()
    c.check(work=False)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("shape", [(2, 1, 3000, 8, 2, 64), (1, 300, 500, 2, 2, 32)], ids=str)
def test_captured_replayed_and_beside_another_call(dtype, shape):
    a, b = Case(dtype, *shape), Case(dtype, *shape, seed=40)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.call(stream=side)
    for n in range(3):
        a.q.copy_(torch.randn_like(a.q))
        eager = a.call(out=torch.empty_like(a.out)).clone()
        alone = b.call(out=torch.empty_like(b.out)).clone()
        torch.cuda.synchronize()
        a.out.fill_(9)
        b.out.fill_(9)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        b.call(stream=other)
        torch.cuda.synchronize()
        assert torch.equal(a.out, eager) and torch.equal(b.out, alone)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("causal", [False, True])
def test_projection_norm_rotation_and_attention_together(dtype, causal):
    """As a transformer runs them: the fused q/k/v projection, norm and rotation of q and k in place over a 9 x 11 grid, the attention on what they left."""
    b, h, kv, d, c, grid = 2, 4, 4, 32, 256, (9, 11)
    l, t, w = grid[0] * grid[1], tdtype(dtype), 64
    x = torch.from_numpy(quantize(SI.make_array((b, l, c), 760), dtype)).to(DEV).to(t)
    weight = quantize(SI.make_array((3 * c, c), 761, 0.08), dtype)
    packed = torch.from_numpy(B.pack_conv_weight(dtype, weight)).to(DEV)
    q, k, v, out = (torch.full((b, l, c), float("nan"), device=DEV, dtype=t) for _ in range(4))
    B.check(lib.ad_conv_forward(dtype, p(x), None, c, 0, b, l, 1, 0, 1, 1, p(packed), 3 * c, None, None, None, p(q), p(k), p(v), B.OUT_QKV, 0, None, 0, stream_ptr()))
    raw = [z.clone() for z in (q, k)]
    cfg = B.RopeCfg.make([16, 16])
    table = torch.from_numpy(B.rope_table(cfg)).to(DEV)
    pos = torch.stack([torch.arange(l) // grid[1], torch.arange(l) % grid[1]]).to(torch.int32).to(DEV)
    hg = [np.float32(1 + 0.1 * SI.make_array((d,), 762 + n)) for n in range(2)]
    gains = [dev_f32(g) for g in hg]
    B.check(lib.ad_qk_norm_rope_forward(dtype, B.AD_NORM_RMS, cfg, p(table), p(pos), 0, p(q), p(k), p(gains[0]), p(gains[1]), None, None, 1e-6, b, l, 2 * h, 2 * kv, d, c, c, p(q), p(k), c, c,
                                        stream_ptr()))
    lam, sub = np.float32([0.3] * h), np.float32(1 + 0.1 * SI.make_array((w,), 764))
    dl, ds = dev_f32(lam), dev_f32(sub)
    B.check(lib.ad_diff_attention_forward(dtype, p(q), p(k), p(v), b, l, l, h, kv, d, c, c, c, c, None, int(causal), p(dl), p(ds), 1e-5, 0.5, p(out), None, 0, stream_ptr()))
    torch.cuda.synchronize()
    import test_gpu_rope as R
    f64 = lambda z: z.double().cpu().numpy()
    # each operator is held to its own bound on what the one before it left
    where = np.repeat(pos.cpu().numpy()[None], b, 0)
    for before, after, g in zip(raw, (q, k), hg):
        ref, err = R.reference(f64(before).reshape(b, l, -1, d), cfg, where, B.AD_NORM_RMS, g, None, 1e-6)
        R.check(f64(after).reshape(ref.shape), ref, err, dtype)
    ref, bound = reference(dtype, f64(q).reshape(b, l, h, 2, d), f64(k).reshape(b, l, kv, 2, d), f64(v).reshape(b, l, kv, w), lam, None, causal, sub, 1e-5, 0.5)
    assert (np.abs(f64(out).reshape(ref.shape) - ref) <= bound).all()
    # and the projection to its single rounding
    proj = f64(x) @ weight.astype(np.float64).T
    assert np.abs(f64(raw[0]) - proj[..., :c]).max() <= (2.0 ** -8 if dtype == B.AD_BF16 else 1e-5) * np.abs(proj).max()
