"""Rotary positions, norms of queries and keys, differential attention: what the host does, and what it refuses (no GPU needed)."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest

from paper_2406_06911_amd import binding as B

L = B.lib
FAKE = 1 << 20                                     # an aligned address that is never used: every call below is refused first


def decoded(cfg):
    """Frequencies in turns a position, modulo one turn."""
    return B.rope_table(cfg).view(np.uint64).astype(object)


def test_table_holds_fractions_of_a_turn():
    cfg = B.RopeCfg.make([8, 4], base=500.0)
    got = [Fraction(int(t), 2 ** 64) for t in decoded(cfg)]
    want = [500.0 ** (-2 * i / 8) for i in range(4)] + [500.0 ** (-2 * i / 4) for i in range(2)]
    assert len(got) == 6
    for g, w in zip(got, want):
        assert abs(float(g) * 2 * math.pi - w) <= 4 * 2.0 ** -53 * w      # pow, the division by 2 pi, the conversion back


@pytest.mark.parametrize("position", [1, -1, 12345, 2 ** 31 - 1, -2 ** 31])
def test_phase_of_far_positions(position):
    """The kernel's whole-number phase, restated, against exact rational arithmetic with 2 pi to 40 digits."""
    two_pi = Fraction(62831853071795864769252867665590057683943, 10 ** 40)
    cfg = B.RopeCfg.make([64], base=10000.0)
    for i, t in enumerate(decoded(cfg)):
        phase = (((position % 2 ** 64) * int(t)) % 2 ** 64) >> 32
        f = Fraction(math.pow(10000.0, -2.0 * i / 64))
        exact = (position * f / two_pi) % 1
        off = abs(Fraction(phase, 2 ** 32) - exact)
        # 2^-32 for the cut, the long double's 2^-64 and the table's half step times the position
        assert min(off, 1 - off) <= Fraction(1, 2 ** 32) + abs(position) * Fraction(3, 2 ** 64)


def test_scalings_of_the_frequencies():
    n = 16
    plain = [10000.0 ** (-2 * i / n) for i in range(n // 2)]
    radians = lambda cfg: [float(Fraction(int(t), 2 ** 64)) * 2 * math.pi for t in decoded(cfg)]
    np.testing.assert_allclose(radians(B.RopeCfg.make([n], scaling=B.AD_ROPE_LINEAR, factor=4.0)), [f / 4 for f in plain], rtol=1e-14)
    raised = 10000.0 * 4.0 ** (n / (n - 2))
    np.testing.assert_allclose(radians(B.RopeCfg.make([n], scaling=B.AD_ROPE_BASE, factor=4.0)), [raised ** (-2 * i / n) for i in range(n // 2)], rtol=1e-13)
    parts = radians(B.RopeCfg.make([n], scaling=B.AD_ROPE_PARTS, factor=4.0, original_len=100.0, slow_turns=1.0, fast_turns=4.0))
    for f, g in zip(plain, parts):
        turns = 100.0 * f / (2 * math.pi)
        want = f if turns > 4 else f / 4 if turns < 1 else f / 4 * (1 - (turns - 1) / 3) + f * (turns - 1) / 3
        assert abs(g - want) <= 1e-14 * want
    # the lowest frequency of a raised base is the interpolated one: base'^(-(n-2)/n) = base^(-(n-2)/n) / factor
    assert abs(radians(B.RopeCfg.make([n], scaling=B.AD_ROPE_BASE, factor=4.0))[-1] - plain[-1] / 4) <= 1e-13 * plain[-1]


@pytest.mark.parametrize("change", [
    dict(layout=2), dict(n_axes=0), dict(n_axes=4), dict(axis_dims=(C.c_int * 3)(3, 0, 0)), dict(axis_dims=(C.c_int * 3)(0, 0, 0)), dict(axis_dims=(C.c_int * 3)(130, 0, 0)),
    dict(n_axes=2, axis_dims=(C.c_int * 3)(64, 66, 0)), dict(axis_dims=(C.c_int * 3)(-2, 0, 0)), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(amplitude=-1.0),
    dict(amplitude=float("inf")), dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=2, factor=float("nan")), dict(scaling=3, factor=2.0, original_len=0.0),
    dict(scaling=3, factor=2.0, original_len=10.0, slow_turns=4.0, fast_turns=4.0), dict(scaling=3, factor=2.0, original_len=10.0, slow_turns=-1.0)], ids=str)
def test_bad_rotary_configurations_are_refused(change):
    cfg = B.RopeCfg.make([64])
    for name, value in change.items():
        setattr(cfg, name, value)
    n = C.c_size_t()
    assert L.ad_rope_table(C.byref(cfg), None, C.byref(n)) == B.AD_ERR_INVALID
    assert L.ad_rope_forward(B.AD_F32, cfg, FAKE, FAKE, 0, FAKE, None, 1, 4, 1, 0, 64, 64, 0, FAKE, None, 64, 0, None) == B.AD_ERR_INVALID
    assert L.ad_rope_table(None, None, C.byref(n)) == B.AD_ERR_INVALID


GOOD_ROPE = dict(dtype=B.AD_BF16, cfg=B.RopeCfg.make([64]), table=FAKE, positions=FAKE, per=0, q=FAKE, k=FAKE, b=2, l=4, heads=5, kv=5, d=64, ldq=320, ldk=320, qo=2 * FAKE, ko=3 * FAKE,
                 ldqo=320, ldko=320)
BAD_ROPE = [dict(dtype=7), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(table=None), dict(positions=None), dict(cfg=None), dict(b=0), dict(l=0), dict(l=-1), dict(heads=0),
            dict(kv=-1), dict(d=0), dict(d=129, ldq=999, ldk=999, ldqo=999, ldko=999), dict(d=62), dict(ldq=319), dict(ldk=319), dict(ldqo=319), dict(ldko=319), dict(b=1 << 16, l=1 << 15),
            dict(q=FAKE + 1), dict(qo=FAKE, ldqo=328), dict(ko=2 * FAKE), dict(table=FAKE + 4), dict(positions=FAKE + 2), dict(heads=1 << 30), dict(kv=1 << 30)]


def rope(a):
    return L.ad_rope_forward(a["dtype"], a["cfg"], a["table"], a["positions"], a["per"], a["q"], a["k"], a["b"], a["l"], a["heads"], a["kv"], a["d"], a["ldq"], a["ldk"], a["qo"], a["ko"],
                             a["ldqo"], a["ldko"], None)


def qk_norm(a):
    return L.ad_qk_norm_rope_forward(a["dtype"], a["norm"], a["cfg"], a["table"], a["positions"], a["per"], a["q"], a["k"], a["qg"], a["kg"], a["qb"], a["kb"], a["eps"], a["b"], a["l"],
                                     a["heads"], a["kv"], a["d"], a["ldq"], a["ldk"], a["qo"], a["ko"], a["ldqo"], a["ldko"], None)


@pytest.mark.parametrize("change", BAD_ROPE, ids=str)
def test_rope_refuses(change):
    assert rope({**GOOD_ROPE, **change}) == B.AD_ERR_INVALID
    assert b"rope" in L.ad_last_error()


@pytest.mark.parametrize("change", [c for c in BAD_ROPE if "cfg" not in c] + [dict(norm=2), dict(norm=-1), dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
                                                                             dict(norm=0, qb=FAKE), dict(norm=0, kb=FAKE), dict(qg=FAKE + 2), dict(kb=FAKE + 1)], ids=str)
def test_qk_norm_refuses(change):
    good = dict(GOOD_ROPE, norm=B.AD_NORM_LAYER, qg=FAKE, kg=FAKE, qb=FAKE, kb=FAKE, eps=1e-6)
    assert qk_norm({**good, **change}) == B.AD_ERR_INVALID
    assert b"qk norm" in L.ad_last_error()


GOOD_DIFF = dict(dtype=B.AD_BF16, q=FAKE, k=2 * FAKE, v=3 * FAKE, b=2, l=8, lk=16, heads=4, kv=2, d=64, ldq=512, ldk=256, ldv=256, ldo=512, lens=None, causal=0, lam=FAKE, gain=FAKE, eps=1e-5,
                 scale=1.0, out=4 * FAKE, ws=None, wsb=0)


@pytest.mark.parametrize("change", [dict(dtype=2), dict(q=None), dict(k=None), dict(v=None), dict(lam=None), dict(out=None), dict(b=0), dict(l=0), dict(lk=0), dict(lk=-5), dict(heads=0), dict(kv=0),
                                    dict(heads=5), dict(d=0), dict(d=60), dict(d=136, ldq=2000, ldk=2000, ldv=2000, ldo=2000), dict(dtype=B.AD_F32, d=6), dict(ldq=504), dict(ldk=248),
                                    dict(ldv=248), dict(ldo=504), dict(ldq=514), dict(ldk=260), dict(q=FAKE + 8), dict(v=FAKE + 2), dict(out=FAKE + 4), dict(lens=FAKE + 1), dict(lam=FAKE + 2),
                                    dict(gain=FAKE + 2), dict(ws=FAKE + 8), dict(eps=0.0), dict(eps=float("nan")), dict(scale=float("inf")), dict(b=1 << 20, l=1 << 20), dict(ldk=1 << 23), dict(ldv=1 << 24), dict(lk=0x7fff8000)], ids=str)
def test_differential_attention_refuses(change):
    a = {**GOOD_DIFF, **change}
    st = L.ad_diff_attention_forward(a["dtype"], a["q"], a["k"], a["v"], a["b"], a["l"], a["lk"], a["heads"], a["kv"], a["d"], a["ldq"], a["ldk"], a["ldv"], a["ldo"], a["lens"], a["causal"],
                                     a["lam"], a["gain"], a["eps"], a["scale"], a["out"], a["ws"], a["wsb"], None)
    assert st == B.AD_ERR_INVALID
    assert b"differential attention" in L.ad_last_error()


def test_workspace_of_differential_attention():
    size = L.ad_diff_attention_workspace_bytes
    assert size(B.AD_BF16, 2, 9216, 9216, 5, 5, 32) == 0                       # enough rows: nothing is shared out
    few = size(B.AD_BF16, 1, 1, 100000, 8, 8, 64)
    assert few > 0 and few % ((4 * 64 + 4) * 4 * 8) == 0                        # whole records of 8 rows
    assert size(B.AD_BF16, 1, 1, 16, 8, 8, 64) == 0                             # too few keys to share
    for bad in ((7, 1, 1, 100000, 8, 8, 64), (1, 0, 1, 100000, 8, 8, 64), (1, 1, 1, 100000, 8, 3, 64), (1, 1, 1, 100000, 8, 8, 256)):
        assert size(*bad) == 0


def test_lambda_from_learned_vectors():
    rng = np.random.default_rng(5)
    v = [np.float32(rng.standard_normal(64) * 0.1) for _ in range(4)]
    out = C.c_float()
    at = [x.ctypes.data for x in v]
    B.check(L.ad_diff_lambda(*at, 64, 0.8, C.byref(out)))
    want = math.exp(float(np.dot(v[0].astype(np.float64), v[1]))) - math.exp(float(np.dot(v[2].astype(np.float64), v[3]))) + float(np.float32(0.8))
    assert abs(out.value - want) <= 2.0 ** -23 * abs(want)
    assert L.ad_diff_lambda(None, *at[1:], 64, 0.8, C.byref(out)) == B.AD_ERR_INVALID
    assert L.ad_diff_lambda(*at, 0, 0.8, C.byref(out)) == B.AD_ERR_INVALID
