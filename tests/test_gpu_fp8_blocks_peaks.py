"""Rows that one token dominates, over block scales.  With probabilities rounded to p_i (1 + d_i), |d_i| <= 2^-8, and a denominator that
sums the rounded ones, the output is off by sum p_i d_i (v_i - o) / sum p_i (1 + d_i): for such a row hardly more than its own final rounding,
also where the dominating probability is no power of two (its reference, an earlier maximum, lags by up to 2^8)."""
import numpy as np
import pytest

from oracle import fp8_blocks as FB
from paper_2605_15250_amd.harness import NUM_CUS
from test_gpu_fp8_blocks import D_R, EPS, World, attend, stored
from test_gpu_fp8_blocks_forms import FORMS, decode

pytestmark = pytest.mark.gpu


def peaked_world(lens, g, G, d_h, d_v, P, s_q, seed, rows=2):
    """Key dim 0 is all that counts: 1 for one late token that a sequence's last `rows` rows see, 0 for the first token of every tile, -8 for
    the others."""
    w = World(lens, g, d_h, d_v, G=G, P=P, seed=seed, s_q=s_q)
    total = sum(lens)
    k, kr = np.zeros((total, g, d_h), np.float32), np.zeros((total, D_R), np.float32)
    v = np.sign(w.r.normal(size=(total, g, d_v))) * w.r.uniform(0.0, 0.25, (total, g, d_v))
    peaks, at = [], 0
    for n in lens:
        peak = max(0, n - rows - int(w.r.integers(0, 20)))
        k[at:at + n, :, 0] = -8.0
        k[at:at + n:32, :, 0] = 0.0
        k[at + peak, :, 0] = 1.0
        v[at + peak] *= w.r.uniform(4.0, 8.0, (g, d_v)) / 0.25
        peaks.append(peak)
        at += n
    w.append(lens, rows=(stored(k), stored(v), kr))
    w.spoil()
    return w, peaks


def queries(w, rows):
    """Logits of 6.5 to 7.9 (to base 2) for the dominating token."""
    q_c = np.zeros((rows, w.g * w.G, w.d_h))
    q_c[:, :, 0] = w.r.uniform(6.5, 7.9, (rows, w.g * w.G)) * np.log(2.0) * np.sqrt(w.d_h + D_R)
    return stored(q_c), np.zeros((rows, w.g * w.G, D_R), np.float32)


def check(w, peaks, out, lse, q_c, q_r, first, lens):
    sc = 1.0 / np.sqrt(w.d_h + D_R)
    for b in range(w.B):
        rows, L = slice(first[b], first[b + 1]), lens[b]
        n = first[b + 1] - first[b]
        K, V, kr = w.K[b].values(), w.V[b].values(), np.zeros((L, D_R))
        want, want_lse, weight = FB.attend(q_c[rows], q_r[rows], K, V, kr, L)
        dl = FB.logit_error(q_c[rows], q_r[rows], K, kr, sc)
        z = np.einsum("nhd,lhd->nhl", q_c[rows].astype(np.float64), np.repeat(K, w.G, 1)) * sc
        z[(np.arange(L)[None, :] > L - n + np.arange(n)[:, None])[:, None].repeat(w.g * w.G, 1)] = -np.inf
        p = np.exp(z - want_lse[:, :, None])
        # sum p_i |v_i - o| is at most twice the same about any other point, here the dominating value, also chunk by chunk
        spread = np.stack([[2 * p[i, h] @ np.abs(V[:, h // w.G] - V[peaks[b], h // w.G]) for h in range(w.g * w.G)] for i in range(n)])
        tol = EPS * np.abs(want) + 1.01 * EPS * spread + 2 * (2 * dl + 2.0 ** -20) * weight
        err = np.abs(out[rows] - want)
        assert np.all(err <= tol), (b, int((err > tol).sum()), err.size, float((err / tol).max()))
        assert np.all(np.abs(lse[rows] - want_lse) <= dl + 2.0 ** -20 * (1 + np.abs(want_lse)))


TEAMS = {"team": (8, 4, 128, 128, 1, 64, [513, 300], 0), "team_one_group": (1, 16, 128, 128, 2, 64, [900, 333], 0),
         "wide_team": (4, 5, 192, 256, 2, 64, [200, 450], 0)}


@pytest.mark.parametrize("form", list(FORMS) + list(TEAMS))
def test_decode_of_peaked_rows(form):
    g, G, d_h, d_v, s_q, P, lens, chunk = {**FORMS, **TEAMS}[form]
    w, peaks = peaked_world(lens, g, G, d_h, d_v, P, s_q, 401)
    q_c, q_r = queries(w, w.B * s_q)
    out, lse = decode(w, q_c, q_r, chunk, NUM_CUS if form in TEAMS else 2)
    check(w, peaks, out, lse, q_c, q_r, np.arange(w.B + 1) * s_q, lens)


@pytest.mark.parametrize("g,G,d_h,d_v,P,lens,ns", [
    (2, 4, 128, 128, 64, [300, 165, 97], [1, 1, 1]), (8, 16, 128, 128, 64, [257], [1]), (5, 4, 192, 256, 64, [200, 90], [1, 1]),
    (2, 4, 128, 128, 256, [3000, 740], [1, 1]), (4, 5, 192, 256, 256, [1500], [1]),
])
def test_attention_of_peaked_rows(g, G, d_h, d_v, P, lens, ns):
    w, peaks = peaked_world(lens, g, G, d_h, d_v, P, 1, 411)
    q_c, q_r = queries(w, sum(ns))
    out, lse, first, _ = attend(w, ns, lens, q_c, q_r)
    check(w, peaks, out, lse, q_c, q_r, first, lens)


def test_attention_of_peaked_chunks():
    lens, ns = [260, 190], [14, 14]
    w, peaks = peaked_world(lens, 2, 4, 128, 128, 64, 1, 421, rows=14)
    q_c, q_r = queries(w, sum(ns))
    out, lse, first, _ = attend(w, ns, lens, q_c, q_r)
    check(w, peaks, out, lse, q_c, q_r, first, lens)
