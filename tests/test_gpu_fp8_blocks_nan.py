"""NaN among the cached keys and values of the cache with block scales: each reaches the rows that see its token and no others, a value only
its own dim of the output, a key the whole row of its group's heads and their log-sum-exp."""
import numpy as np
import pytest

from paper_2605_15250_amd.harness import NUM_CUS
from test_gpu_fp8_blocks import D_R, World, attend, stored
from test_gpu_fp8_blocks_forms import FORMS, decode

pytestmark = pytest.mark.gpu


def world(lens, g, G, d_h, d_v, P, s_q, seed, bad_v=(), bad_k=()):
    """bad_v, bad_k: (sequence, token, group, dim) that are NaN"""
    w = World(lens, g, d_h, d_v, G=G, P=P, seed=seed, s_q=s_q)
    k, v, kr = w.draw_rows(sum(lens))
    begin = np.concatenate([[0], np.cumsum(lens)])
    for plane, bad in ((v, bad_v), (k, bad_k)):
        for b, t, j, d in bad:
            plane[begin[b] + t, j, d] = np.nan
    w.append(lens, rows=(k, v, kr))
    w.spoil()
    return w


def check(w, out, lse, q_c, q_r, first, lens, bad_v=(), bad_k=()):
    """Rows and dims that a NaN has to reach are NaN; all others are what they are with zeros in its place."""
    nan_out, nan_lse = np.zeros(out.shape, bool), np.zeros(lse.shape, bool)
    for b in range(w.B):
        n = first[b + 1] - first[b]
        pos = lens[b] - n + np.arange(n)
        for s, t, j, d in bad_v:
            if s == b:
                nan_out[first[b]:first[b + 1], w.G * j:w.G * (j + 1), d] |= (pos >= t)[:, None]
        for s, t, j, _ in bad_k:
            if s == b:
                nan_out[first[b]:first[b + 1], w.G * j:w.G * (j + 1)] |= (pos >= t)[:, None, None]
                nan_lse[first[b]:first[b + 1], w.G * j:w.G * (j + 1)] |= (pos >= t)[:, None]
    assert np.array_equal(np.isnan(out), nan_out), (np.argwhere(np.isnan(out) != nan_out)[:3], int((np.isnan(out) != nan_out).sum()))
    assert np.array_equal(np.isnan(lse), nan_lse), np.argwhere(np.isnan(lse) != nan_lse)[:3]
    for plane in w.K + w.V:                               # (codes of NaN: 0x7f and 0xff)
        plane.codes[(plane.codes & 0x7F) == 0x7F] = 0
    # rows that hold no NaN of a key's, in two passes: those, and (their other dims) the ones that hold a value's
    keep_out, keep_lse = out.copy(), lse.copy()
    want_out, want_lse = reference(w, q_c, q_r, first, lens)
    keep_out[nan_out], keep_lse[nan_lse] = want_out[nan_out], want_lse[nan_lse]
    w.check_attention(keep_out, keep_lse, q_c, q_r, first, lens)


def reference(w, q_c, q_r, first, lens):
    from oracle import fp8_blocks as FB
    out, lse = np.zeros((q_c.shape[0], w.g * w.G, w.d_v)), np.zeros((q_c.shape[0], w.g * w.G))
    for b in range(w.B):
        rows, L = slice(first[b], first[b + 1]), int(lens[b])
        if first[b] < first[b + 1]:
            out[rows], lse[rows], _ = FB.attend(q_c[rows], q_r[rows], w.K[b].values()[:L], w.V[b].values()[:L], stored(w.kr_held(b))[:L], L)
    return out, lse


@pytest.mark.parametrize("g,G,d_h,d_v,lens,ns,at", [
    (2, 4, 128, 128, [70, 40], [70, 11], [69, 39]), (2, 1, 128, 128, [64, 200], [64, 200], [40, 199]), (8, 16, 128, 128, [257], [130], [256]),
    (1, 3, 128, 128, [300, 33], [150, 33], [170, 1]), (5, 4, 192, 256, [200, 90], [70, 90], [140, 89]), (4, 5, 192, 256, [130], [130], [97]),
    (2, 4, 128, 128, [3000, 40], [3, 2], [2999, 39]), (5, 4, 192, 256, [1500], [250], [1300]),
])
def test_attention_with_a_value_that_only_some_rows_see(g, G, d_h, d_v, lens, ns, at):
    bad = [(b, t, b % g, 5 + 64 * b) for b, t in enumerate(at)] + [(0, at[0], g - 1, d_v - 1)]
    w = world(lens, g, G, d_h, d_v, 64, 1, 501 + g + G, bad_v=bad)
    q_c, q_r = stored(w.r.normal(size=(sum(ns), g * G, d_h))), stored(w.r.normal(size=(sum(ns), g * G, D_R)))
    out, lse, first, _ = attend(w, ns, lens, q_c, q_r)
    check(w, out, lse, q_c, q_r, first, lens, bad_v=bad)


@pytest.mark.parametrize("g,G,d_h,d_v,lens,ns,at", [
    (2, 4, 128, 128, [70, 40], [70, 11], [69, 3]), (4, 5, 192, 256, [130], [130], [97]), (2, 4, 128, 128, [3000, 40], [3, 2], [2999, 20]),
    (2, 4, 128, 128, [3000, 40], [3, 2], [700, 39]),
])
def test_attention_with_a_key(g, G, d_h, d_v, lens, ns, at):
    bad = [(b, t, b % g, 5) for b, t in enumerate(at)]
    w = world(lens, g, G, d_h, d_v, 64, 1, 511 + g + G, bad_k=bad)
    q_c, q_r = stored(w.r.normal(size=(sum(ns), g * G, d_h))), stored(w.r.normal(size=(sum(ns), g * G, D_R)))
    out, lse, first, _ = attend(w, ns, lens, q_c, q_r)
    check(w, out, lse, q_c, q_r, first, lens, bad_k=bad)


TEAMS = {"team": (8, 4, 128, 128, 2, 64, [513, 300], 0), "team_one_group": (1, 16, 128, 128, 2, 64, [900, 333], 0),
         "wide_team": (4, 5, 192, 256, 2, 64, [200, 450], 0)}


def step(form, **bad):
    g, G, d_h, d_v, s_q, P, lens, chunk = {**FORMS, **TEAMS}[form]
    w = world(lens, g, G, d_h, d_v, P, s_q, 521, **bad)
    q_c, q_r = stored(w.r.normal(size=(w.B * s_q, g * G, d_h))), stored(w.r.normal(size=(w.B * s_q, g * G, D_R)))
    out, lse = decode(w, q_c, q_r, chunk, NUM_CUS if form in TEAMS else 2)
    check(w, out, lse, q_c, q_r, np.arange(w.B + 1) * s_q, lens, **bad)


@pytest.mark.parametrize("form", {**FORMS, **TEAMS})
def test_step_with_a_value(form):
    """Of tokens that every row sees: the first ones, and the last of them."""
    g, d_v, s_q, lens = (({**FORMS, **TEAMS}[form])[i] for i in (0, 3, 4, 6))
    step(form, bad_v=[(0, 10, 0, 3), (1, lens[1] - s_q, g - 1, d_v - 1)])


@pytest.mark.parametrize("form", {**FORMS, **TEAMS})
def test_step_with_a_key(form):
    """In the first chunk of several, in the last, and (two rows) in the token that only the second row sees."""
    g, lens = {**FORMS, **TEAMS}[form][0], {**FORMS, **TEAMS}[form][6]
    step(form, bad_k=[(0, 10, 0, 3), (1, lens[1] - 1, g - 1, 127)])
