"""The block-scaled 8-bit expanded cache on the GPU: conversion and appends byte for byte against the oracle, both attention calls
against fp64 on the values the cache holds, the calls together as a server makes them, recorded and replayed."""
import numpy as np
import pytest
import torch

from oracle import fp8_blocks as FB
from oracle import gqla_oracle as O
from oracle import layout as Lay
from paper_2605_15250_amd import binding as B
from paper_2605_15250_amd.harness import NUM_CUS

pytestmark = pytest.mark.gpu

D_R, BASE, FILL = 64, 10000.0, 0xAA
EPS = 2.0 ** -8        # half a step of bf16, relative


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16)


def stored(x):
    return bf16(x).float().numpy()


def bits(x):
    return (np.ascontiguousarray(stored(x)).view(np.uint32) >> 16).astype(np.uint16)


class World:
    """Sequences with pages of their own in mixed order, their logical content (oracle) beside the device pool."""

    def __init__(self, lens_max, g=2, d_h=128, d_v=128, G=4, P=64, seed=0, s_q=1, table=True):
        self.r = np.random.default_rng(seed)
        self.B, self.g, self.G, self.d_h, self.d_v, self.P, self.s_q = len(lens_max), g, G, d_h, d_v, P, s_q
        self.max_pages = max(1, -(-max(lens_max) // P)) + 1
        if table:
            need = [max(0, -(-n // P)) for n in lens_max]
            perm = self.r.permutation(sum(need) + 2)
            self.table, at = np.full((self.B, self.max_pages), -1, np.int32), 0
            for b, n in enumerate(need):
                self.table[b, :n] = perm[at:at + n]
                at += n
            self.pages = sum(need) + 2
        else:
            self.table, self.pages = np.arange(self.B * self.max_pages, dtype=np.int32).reshape(self.B, -1), self.B * self.max_pages
        self.shape = B.make_shape(self.B, g * G, g, d_h, 512, D_R, s_q, B.GQLA_BF16, 0.0, d_v)
        self.bytes = FB.page_bytes(P, g, d_h, d_v, D_R)
        self.ref = np.full((self.pages, self.bytes), FILL, np.uint8)
        self.pool = torch.full((self.pages, self.bytes), FILL, dtype=torch.uint8, device="cuda")
        self.d_table = torch.from_numpy(self.table).cuda() if table else None
        self.d_lens = torch.zeros(self.B, dtype=torch.int32, device="cuda")
        self.K = [FB.Plane(g, d_h) for _ in range(self.B)]
        self.V = [FB.Plane(g, d_v) for _ in range(self.B)]
        self.kr = [np.zeros((0, D_R), np.float32) for _ in range(self.B)]

    def cache(self, pool=None, groups=None):
        return B.make_cache(self.pool if pool is None else pool, self.d_lens, self.d_table, self.P, self.max_pages, self.pages, groups or self.g)

    def lens(self):
        return np.array([len(k.codes) for k in self.K], np.int32)

    def sync_lens(self, lens=None):
        self.d_lens.copy_(torch.from_numpy(self.lens() if lens is None else np.asarray(lens, np.int32)))

    def draw_rows(self, n):
        """n rows whose blocks differ in size by powers of two."""
        size = lambda d: np.exp2(self.r.integers(-3, 6, (n, self.g, 1)))  # noqa: E731
        return (stored(self.r.normal(size=(n, self.g, self.d_h)) * size(0)), stored(self.r.normal(size=(n, self.g, self.d_v)) * size(0)),
                stored(self.r.normal(size=(n, D_R))))

    def append(self, ns, rows=None, strided=False, uniform=False, q=True, base=BASE):
        """Appends ns[b] rows per sequence on both sides; returns (q_r, q_rot, first, positions)."""
        k, v, kr = rows or self.draw_rows(sum(ns))
        first = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
        old = self.lens()
        total = int(first[-1])
        pos = np.concatenate([old[b] + np.arange(ns[b]) for b in range(self.B)]) if total else np.zeros(0, int)
        turned = O.rope(kr, pos, base) if base else kr
        for b in range(self.B):
            part = slice(first[b], first[b + 1])
            self.K[b].append(k[part])
            self.V[b].append(v[part])
            self.kr[b] = np.concatenate([self.kr[b], turned[part]])
        self.sync_lens()
        dk, dv, dr = bf16(k.reshape(total, -1)).cuda(), bf16(v.reshape(total, -1)).cuda(), bf16(kr).cuda()
        strides = {}
        if strided:
            joint = torch.full((total, dk.shape[1] + dv.shape[1] + D_R + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
            a, e = dk.shape[1] + 8, dk.shape[1] + 8 + dv.shape[1] + 8
            joint[:, :dk.shape[1]], joint[:, a:a + dv.shape[1]], joint[:, e:e + D_R] = dk, dv, dr
            dk, dv, dr = joint[:, :dk.shape[1]], joint[:, a:a + dv.shape[1]], joint[:, e:e + D_R]
            strides = dict(k_stride=joint.stride(0), v_stride=joint.stride(0), kr_stride=joint.stride(0))
        q_r = stored(self.r.normal(size=(total, self.g * self.G, D_R)))
        d_q = bf16(q_r).cuda()
        q_rot = torch.full_like(d_q, 7.0)
        d_first = None if uniform else torch.from_numpy(first).cuda()
        B.gqla_append_expanded_fp8_blocks(self.shape, B.make_new_rows(dk, dv, dr, d_q if q else None, q_rot if q else None, d_first, total, **strides),
                                          base, self.cache())
        torch.cuda.synchronize()
        return q_r, q_rot.float().cpu().numpy(), first, pos

    def check_pool(self):
        """Codes and scales equal, k_R within a rounding, every other byte as it was."""
        got = self.pool.cpu().numpy().copy()
        want = np.full_like(self.ref, FILL)
        dims = (self.P, self.g, self.d_h, self.d_v, D_R)
        for b in range(self.B):
            FB.store(want, self.table[b], self.P, self.K[b], self.V[b], bits(self.kr[b]))
        a, e = self.P * self.g * (self.d_h + self.d_v), self.P * (self.g * (self.d_h + self.d_v) + 2 * D_R)
        diff = ~FB.same_codes(got[:, :a], want[:, :a])
        assert not diff.any(), "%d codes differ, first at %s" % (diff.sum(), np.argwhere(diff)[0])
        assert np.array_equal(got[:, e:], want[:, e:]), "scales"
        got_r, want_r = got[:, a:e].copy().view(np.uint16), want[:, a:e].copy().view(np.uint16)
        value = lambda u: (u.astype(np.uint32) << 16).view(np.float32).astype(np.float64)  # noqa: E731
        owned = np.zeros(got_r.shape, bool)
        exact = np.zeros(got_r.shape)
        for b in range(self.B):
            t = np.arange(len(self.kr[b]))
            keep = t // self.P < self.max_pages
            pg = self.table[b][np.minimum(t // self.P, self.max_pages - 1)]
            keep &= (pg >= 0) & (pg < self.pages)
            o = FB.kr_offset(t[:, None] % self.P, np.arange(D_R), *dims) - a
            owned[pg[keep, None], o[keep] // 2] = True
            exact[pg[keep, None], o[keep] // 2] = self.kr[b][keep]
        assert np.array_equal(got_r[~owned], want_r[~owned])
        # one rounding to bf16 of a rotation formed in fp32 from two values of size |x| (2^-20: its own roundings and the angle's)
        assert np.all(np.abs(value(got_r)[owned] - exact[owned]) <= EPS * np.abs(exact[owned]) + 2.0 ** -20 * 8)

    def spoil(self):
        """NaN (codes and k_R) in every byte that belongs to no token."""
        a, b = np.zeros_like(self.ref), np.full_like(self.ref, 1)
        for pool in (a, b):
            for i in range(self.B):
                FB.store(pool, self.table[i], self.P, self.K[i], self.V[i], bits(self.kr[i]))
        self.pool[torch.from_numpy(a != b).cuda()] = 0xFF

    def check_attention(self, out, lse, q_c, q_rot, first, lens, hidden=None):
        sc = 1.0 / np.sqrt(self.d_h + D_R)
        for b in range(self.B):
            rows, L = slice(first[b], first[b + 1]), int(lens[b])
            if first[b] == first[b + 1]:
                continue
            K, V, kr = self.K[b].values()[:L], self.V[b].values()[:L], stored(self.kr_held(b))[:L]
            want, want_lse, weight = FB.attend(q_c[rows], q_rot[rows], K, V, kr, L, None if hidden is None else hidden[b][:L])
            dl = FB.logit_error(q_c[rows], q_rot[rows], K, kr, sc) if L else 0.0
            # the result's rounding, the probabilities' (to bf16, against sums that see them unrounded), the logits' errors in both sums
            tol = EPS * np.abs(want) + (EPS + 2 * (2 * dl + 2.0 ** -20)) * weight * 1.01 + 1e-30
            err = np.abs(out[rows] - want)
            assert np.all(err <= tol), (b, float((err - tol).max()), float(np.abs(want).max()))
            seen = np.isfinite(want_lse)
            assert np.array_equal(seen, np.isfinite(lse[rows])) and np.all(np.isneginf(lse[rows][~seen]))
            assert np.all(np.abs(lse[rows][seen] - want_lse[seen]) <= dl + 2.0 ** -20 * (1 + np.abs(want_lse[seen])))

    def kr_held(self, b):
        """k_R as the device holds it (bf16, its own rounding), so that attention is compared on equal inputs."""
        pool = self.pool.cpu().numpy()
        dims = (self.P, self.g, self.d_h, self.d_v, D_R)
        t = np.arange(len(self.kr[b]))
        keep = np.minimum(t // self.P, self.max_pages - 1)
        pg = np.clip(self.table[b][keep], 0, self.pages - 1)
        o = FB.kr_offset(t[:, None] % self.P, np.arange(D_R), *dims)
        u = pool[pg[:, None], o].astype(np.uint32) | pool[pg[:, None], o + 1].astype(np.uint32) << 8
        return (u << 16).view(np.float32)


# ---- conversion -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("g,d_h,d_v,P,lens", [
    (2, 128, 128, 64, [1, 64, 65, 200]), (5, 192, 256, 64, [33, 31, 0, 97]), (1, 128, 128, 256, [700, 15]), (8, 128, 128, 128, [130]),
])
def test_quantize_is_the_rule_byte_for_byte(g, d_h, d_v, P, lens):
    w = World([max(n, 1) for n in lens], g, d_h, d_v, P=P, seed=11 + g)
    rows = [w.draw_rows(n) for n in lens]
    for b, (k, v, kr) in enumerate(rows):
        if lens[b] > 40:                      # a block of zeros, tiny and huge values, infinities and NaN among them
            k[0:32], v[32:40] = 0.0, 0.0
            k[40], v[3], v[4, :, 5] = stored(1e-37), stored(3e38), np.inf
            k[41, 0, 7], k[42, 0, 8], v[37, 0, 9] = -np.inf, np.nan, np.nan
        w.K[b].append(k), w.V[b].append(v)
        w.kr[b] = kr
    wide = Lay.pack_expanded_pool([x[0] for x in rows], [x[1] for x in rows], [x[2] for x in rows], w.table, w.pages, P, fill=np.nan)
    d_wide = torch.from_numpy(wide).to(torch.bfloat16).cuda()
    w.sync_lens(lens)
    B.gqla_quantize_expanded_fp8_blocks(w.shape, w.cache(d_wide), w.cache())
    torch.cuda.synchronize()
    w.check_pool()


# ---- appends ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("g,d_h,d_v,P,steps", [
    (2, 128, 128, 64, [[70, 0, 1], [1, 33, 31], [1, 0, 1], [2, 2, 2], [40, 95, 0], [1, 1, 64]]),
    (1, 128, 128, 128, [[5], [27], [1], [31], [300], [3]]),
    (5, 192, 256, 64, [[1, 40], [1, 1], [5, 63], [64, 2]]),
])
@pytest.mark.parametrize("strided", [False, True])
def test_append_is_the_rule_byte_for_byte(g, d_h, d_v, P, steps, strided):
    total = np.sum(steps, axis=0)
    w = World([int(n) for n in total], g, d_h, d_v, P=P, seed=21 + g)
    for ns in steps:
        q_r, q_rot, first, pos = w.append(ns, strided=strided)
        w.check_pool()
        want = O.rope(q_r, pos[:, None], BASE)
        assert np.all(np.abs(q_rot - want) <= EPS * np.abs(want) + 2.0 ** -20 * 8)


def test_append_more_than_64_sequences_and_uniform_steps():
    w = World([40] * 130, 2, G=2, seed=31, s_q=2)
    w.append([int(x) for x in w.r.integers(0, 36, 130)])
    w.check_pool()
    for _ in range(2):
        w.append([2] * 130, uniform=True)
        w.check_pool()


def test_append_edges():
    """Infinities, NaN, zeros, values beyond the scales; no rotation and no queries; the same rows again."""
    w = World([90, 64 + 3], 2, seed=41)
    k, v, kr = w.draw_rows(77)
    k[3, 0, 5], k[9, 1, 2], v[11, 0, 7], v[12, 1, 0] = np.inf, np.nan, -np.inf, np.nan
    k[40:], v[40:45] = 0.0, stored(3.2e38)
    w.append([37, 40], rows=(k, v, kr), q=False, base=0.0)
    w.check_pool()
    rows = w.draw_rows(3)
    w.append([3, 0], rows=rows)
    w.check_pool()
    for bad in (np.nan, np.inf, -np.inf):                 # alone in a step's row, K and V
        k1, v1, kr1 = w.draw_rows(2)
        k1[0, 0, 3], v1[0, 1, 100], v1[1, 0, 127] = bad, bad, bad
        w.append([1, 1], rows=(k1, v1, kr1))
        w.check_pool()
    rows = w.draw_rows(3)
    w.append([3, 0], rows=rows)
    before = w.pool.clone()
    first = torch.tensor([0, 3, 3], dtype=torch.int32, device="cuda")
    new = B.make_new_rows(bf16(rows[0].reshape(3, -1)).cuda(), bf16(rows[1].reshape(3, -1)).cuda(), bf16(rows[2]).cuda(), first=first, total=3)
    B.gqla_append_expanded_fp8_blocks(w.shape, new, BASE, w.cache())
    torch.cuda.synchronize()
    assert torch.equal(before, w.pool)


def test_append_drops_what_has_no_place():
    """More rows than the length counts (positions below 0), pages outside the pool, rows that no sequence owns."""
    w = World([64, 64, 64], 2, seed=51)
    w.table[1, 0] = w.pages + 5
    w.d_table = torch.from_numpy(w.table).cuda()
    k, v, kr = w.draw_rows(30)
    total, first = 30, np.array([2, 12, 17, 24], np.int32)       # rows 0, 1 and 24 .. 29 belong to nobody
    w.d_lens.copy_(torch.tensor([6, 5, 7], dtype=torch.int32))     # the first sequence has 10 rows and 6 positions
    q = bf16(w.r.normal(size=(total, 8, D_R))).cuda()
    q_rot = torch.full_like(q, 7.0)
    new = B.make_new_rows(bf16(k.reshape(total, -1)).cuda(), bf16(v.reshape(total, -1)).cuda(), bf16(kr).cuda(), q, q_rot,
                          torch.from_numpy(first).cuda(), total)
    B.gqla_append_expanded_fp8_blocks(w.shape, new, BASE, w.cache())
    torch.cuda.synchronize()
    for b, part in ((0, slice(6, 12)), (2, slice(17, 24))):
        w.K[b].append(k[part]), w.V[b].append(v[part])
        w.kr[b] = O.rope(kr[part], np.arange(part.stop - part.start), BASE)
    w.check_pool()
    got, src = q_rot.float().cpu().numpy(), q.float().cpu().numpy()
    for rows in (slice(0, 6), slice(24, 30)):
        assert np.all(got[rows] == 7.0)
    want = O.rope(src[12:17], np.arange(5)[:, None], BASE)          # its page is missing, its queries are not
    assert np.all(np.abs(got[12:17] - want) <= EPS * np.abs(want) + 2.0 ** -20 * 8)


@pytest.mark.parametrize("dtype,g,d_h,d_v,P", [("bf16", 2, 128, 128, 64), ("bf16", 5, 192, 256, 128), ("f32", 3, 24, 40, 24), ("f32", 1, 128, 16, 64)])
def test_append_to_the_wide_cache(dtype, g, d_h, d_v, P):
    r = np.random.default_rng(61 + g)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    steps, G = [[70, 0, 1], [1, 33, 9], [2, 1, 7]], 3
    lens = np.zeros(3, np.int64)
    total = np.sum(steps, axis=0)
    need = [-(-int(n) // P) for n in total]
    max_pages, pages = max(need), sum(need) + 1
    table, perm, at = np.full((3, max_pages), -1, np.int32), r.permutation(pages), 0
    for b in range(3):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    hold = (lambda x: stored(x)) if dtype == "bf16" else (lambda x: np.asarray(x, np.float32))
    seqs = [[np.zeros((0, g, d_h)), np.zeros((0, g, d_v)), np.zeros((0, D_R))] for _ in range(3)]
    pool = torch.full((pages, P * (g * (d_h + d_v) + D_R)), -5.0, dtype=dt, device="cuda")
    shape = B.make_shape(3, g * G, g, d_h, 512, D_R, 1, B.GQLA_BF16 if dtype == "bf16" else B.GQLA_F32, 0.0, d_v)
    d_lens, d_table = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.from_numpy(table).cuda()
    for ns in steps:
        n = sum(ns)
        k, v, kr, q = hold(r.normal(size=(n, g, d_h))), hold(r.normal(size=(n, g, d_v))), hold(r.normal(size=(n, D_R))), hold(r.normal(size=(n, g * G, D_R)))
        first = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
        pos = np.concatenate([lens[b] + np.arange(ns[b]) for b in range(3)])
        turned = O.rope(kr, pos, BASE)
        for b in range(3):
            part = slice(first[b], first[b + 1])
            seqs[b] = [np.concatenate([s, x[part]]) for s, x in zip(seqs[b], (k, v, turned))]
        lens += ns
        d_lens.copy_(torch.from_numpy(lens.astype(np.int32)))
        to = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dt).cuda()  # noqa: E731
        d_q = to(q)
        new = B.make_new_rows(to(k), to(v), to(kr), d_q, d_q, torch.from_numpy(first).cuda(), n)     # queries in place
        B.gqla_append_expanded(shape, new, BASE, B.make_cache(pool, d_lens, d_table, P, max_pages, pages, g))
        torch.cuda.synchronize()
        want = Lay.pack_expanded_pool([s[0].astype(np.float32) for s in seqs], [s[1].astype(np.float32) for s in seqs],
                                      [s[2].astype(np.float32) for s in seqs], table, pages, P, fill=-5.0).reshape(pages, -1)
        got = pool.float().cpu().numpy()
        a = P * g * (d_h + d_v)
        assert np.array_equal(got[:, :a], want[:, :a])
        half = EPS if dtype == "bf16" else 2.0 ** -24
        tol = lambda x: half * np.abs(x) + 2.0 ** -20 * 8  # noqa: E731
        assert np.all(np.abs(got[:, a:] - want[:, a:]) <= tol(want[:, a:]))
        exact = O.rope(q, pos[:, None], BASE)
        assert np.all(np.abs(d_q.float().cpu().numpy() - exact) <= tol(exact))


# ---- attention --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("g,G,d_h,d_v,s_q,lens,chunk", [
    (8, 16, 128, 128, 2, [300, 2, 129, 65], 0), (8, 4, 128, 128, 1, [513, 40], 0), (8, 1, 128, 128, 1, [2000, 31], 8),
    (4, 16, 128, 128, 1, [700], 0), (4, 32, 128, 128, 2, [300, 65], 0), (1, 16, 128, 128, 2, [300, 33, 2], 0),
    (3, 5, 128, 128, 1, [77, 256], 0), (4, 5, 192, 256, 2, [200, 3, 450], 0), (5, 4, 192, 256, 1, [130], 1), (2, 40, 192, 256, 1, [90], 0),
])
def test_decode(g, G, d_h, d_v, s_q, lens, chunk):
    w = World(lens, g, d_h, d_v, G=G, seed=71 + g + G, s_q=s_q)
    w.append(lens)
    w.spoil()
    first = np.arange(w.B + 1) * s_q
    q_c, q_r = stored(w.r.normal(size=(w.B * s_q, g * G, d_h))), stored(w.r.normal(size=(w.B * s_q, g * G, D_R)))
    plan = B.gqla_plan_create(w.shape, w.lens(), w.P, NUM_CUS, B.GQLA_PATH_GQA, chunk)
    try:
        ws = torch.empty(B.gqla_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
        B.gqla_plan_upload(plan, ws)
        out = torch.full((w.B * s_q, g * G, d_v), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((w.B * s_q, g * G), float("nan"), device="cuda")
        B.gqla_decode_gqa_fp8_blocks(w.shape, plan, bf16(q_c).cuda(), bf16(q_r).cuda(), w.cache(), out, lse, ws)
        torch.cuda.synchronize()
        w.check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), q_c, q_r, first, w.lens())
    finally:
        B.gqla_plan_destroy(plan)


@pytest.mark.parametrize("g,G,s_q,P,lens,chunk", [
    (4, 5, 2, 64, [450, 3, 200, 193, 64], 3), (8, 4, 1, 64, [700, 31, 33, 640], 4), (4, 20, 2, 64, [400, 97, 520], 5), (4, 32, 1, 128, [1000, 129, 2], 2),
    (5, 4, 2, 64, [700, 3, 200, 193, 64], 3), (3, 7, 1, 64, [1030, 65], 6), (1, 16, 2, 64, [900, 130, 2], 4), (7, 20, 2, 64, [390, 450], 7),
])
def test_decode_with_two_tiles_in_flight(g, G, s_q, P, lens, chunk):
    """(192, 256), chunks of six tiles and more, on a plan for so few units that no chunk is shared out: odd and even numbers of tiles,
    sequences that end early in a chunk, a page that is not there."""
    w = World(lens, g, 192, 256, G=G, P=P, seed=75 + g + G, s_q=s_q)
    w.append(lens)
    w.spoil()
    first = np.arange(w.B + 1) * s_q
    q_c, q_r = stored(w.r.normal(size=(w.B * s_q, g * G, 192))), stored(w.r.normal(size=(w.B * s_q, g * G, D_R)))
    hidden = [np.zeros(n, bool) for n in lens]
    hidden[0][P:2 * P] = True
    held = [w.kr_held(b) for b in range(w.B)]             # (read through the whole table)
    w.kr_held = lambda b: held[b]
    w.table[0, 1] = w.pages
    w.d_table = torch.from_numpy(w.table).cuda()
    plan = B.gqla_plan_create(w.shape, w.lens(), P, 2, B.GQLA_PATH_GQA, chunk)
    try:
        ws = torch.empty(B.gqla_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
        B.gqla_plan_upload(plan, ws)
        out = torch.full((w.B * s_q, g * G, 256), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((w.B * s_q, g * G), float("nan"), device="cuda")
        B.gqla_decode_gqa_fp8_blocks(w.shape, plan, bf16(q_c).cuda(), bf16(q_r).cuda(), w.cache(), out, lse, ws)
        torch.cuda.synchronize()
        w.check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), q_c, q_r, first, w.lens(), hidden)
    finally:
        B.gqla_plan_destroy(plan)


def attend(w, ns, lens, q_c, q_r, extra=0, max_pages=None):
    first = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
    total = int(first[-1]) + extra
    heads = w.g * w.G
    out = torch.full((total, heads, w.d_v), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((total, heads), 7.0, device="cuda")
    pad = lambda x: torch.cat([bf16(x), torch.full((extra,) + x.shape[1:], float("nan"), dtype=torch.bfloat16)]).cuda()  # noqa: E731
    d_first = torch.from_numpy(first).cuda()
    w.sync_lens(lens)
    cache = w.cache()
    need = B.gqla_attend_gqa_workspace_bytes(w.shape, d_first, total, cache)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None
    B.gqla_attend_gqa_fp8_blocks(w.shape, d_first, total, pad(q_c), pad(q_r), cache, out, lse, ws)
    torch.cuda.synchronize()
    if extra:
        assert bool((out[total - extra:] == 7.0).all()) and bool((lse[total - extra:] == 7.0).all())
    return out.float().cpu().numpy(), lse.cpu().numpy(), first, need


@pytest.mark.parametrize("g,G,d_h,d_v,P,lens,ns", [
    (2, 4, 128, 128, 64, [300, 65, 1, 64], [7, 65, 1, 0]), (8, 16, 128, 128, 64, [257], [130]), (1, 16, 128, 128, 128, [520, 200], [9, 200]),
    (5, 4, 192, 256, 64, [200, 90], [70, 90]), (3, 1, 128, 128, 64, [1, 33, 700], [1, 33, 300]), (4, 5, 192, 256, 128, [400], [33]),
    (2, 3, 128, 128, 64, [40] * 70, [5, 0, 3, 40, 1, 0, 9] * 10),
])
def test_attend(g, G, d_h, d_v, P, lens, ns):
    w = World(lens, g, d_h, d_v, G=G, P=P, seed=81 + g + G)
    w.append(lens)
    w.spoil()
    q_c, q_r = stored(w.r.normal(size=(sum(ns), g * G, d_h))), stored(w.r.normal(size=(sum(ns), g * G, D_R)))
    out, lse, first, _ = attend(w, ns, lens, q_c, q_r, extra=3)
    w.check_attention(out, lse, q_c, q_r, first, lens)


@pytest.mark.parametrize("g,G,d_h,d_v,B_", [(8, 4, 128, 128, 40), (5, 4, 192, 256, 32)])
def test_attend_rows_enough_for_the_large_tile(g, G, d_h, d_v, B_):
    """A workgroup for 128 rows, not 64: the chip is full of them."""
    ns = [100, 64, 97, 65, 129, 1, 96, 112] * (B_ // 8)
    lens = [n + (17 * b) % 50 for b, n in enumerate(ns)]
    w = World(lens, g, d_h, d_v, G=G, seed=86 + g)
    w.append(lens)
    w.spoil()
    q_c, q_r = stored(w.r.normal(size=(sum(ns), g * G, d_h))), stored(w.r.normal(size=(sum(ns), g * G, D_R)))
    out, lse, first, _ = attend(w, ns, lens, q_c, q_r, extra=1)
    w.check_attention(out, lse, q_c, q_r, first, lens)


@pytest.mark.parametrize("B_", [4, 70])
def test_row_bounds_that_fall_stay_in_bounds(B_):
    """`first` is the caller's; whatever it holds, nothing ahead of or behind the buffers is written."""
    g, G, total, guard = 2, 4, 1200, 2000
    w = World([64] * B_, g, G=G, seed=95)
    w.append([40] * B_)
    bad = np.zeros(B_ + 1, np.int32)
    bad[1:3] = 1000, 1100                                 # sequence 1 has rows, the ones behind it begin at 0 again
    bad[-1] = -5
    d_first = torch.from_numpy(bad).cuda()
    heads = g * G
    rows = lambda d: torch.full((total + 2 * guard, heads, d), 7.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q_c, q_r, q_rot, out = rows(128), rows(D_R), rows(D_R), rows(128)
    lse = torch.full((total + 2 * guard, heads), 7.0, device="cuda")
    mid = slice(guard, guard + total)
    w.sync_lens([64] * B_)
    cache = w.cache()
    need = B.gqla_attend_gqa_workspace_bytes(w.shape, d_first, total, cache)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    B.gqla_attend_gqa_fp8_blocks(w.shape, d_first, total, q_c[mid], q_r[mid], cache, out[mid], lse[mid], ws)
    k, v = (torch.zeros((total, g, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    k_r = torch.zeros((total, D_R), dtype=torch.bfloat16, device="cuda")
    new = B.make_new_rows(k, v, k_r, q_r[mid], q_rot[mid], d_first, total)
    B.gqla_append_expanded_fp8_blocks(w.shape, new, BASE, cache)
    torch.cuda.synchronize()
    for x in (out, lse, q_rot):
        assert bool((x[:guard] == 7.0).all()) and bool((x[guard + total:] == 7.0).all())


def test_attend_rows_that_see_nothing_and_missing_pages():
    lens = [3, 200, 70]
    w = World([64, 200, 70], 2, G=4, seed=91)
    w.append([3, 200, 70])
    ns = [8, 40, 70]                                      # five rows of the first sequence lie ahead of its first token
    q_c, q_r = stored(w.r.normal(size=(sum(ns), 8, 128))), stored(w.r.normal(size=(sum(ns), 8, D_R)))
    w.table[1, 1], w.table[2, 0] = w.pages, -7            # tokens 64 .. 127 of the second, 0 .. 63 of the third are not there
    w.d_table = torch.from_numpy(w.table).cuda()
    hidden = [np.zeros(n, bool) for n in lens]
    hidden[1][64:128], hidden[2][:64] = True, True
    out, lse, first, _ = attend(w, ns, lens, q_c, q_r)
    w.check_attention(out, lse, q_c, q_r, first, lens, hidden)
    assert np.all(out[:5] == 0) and np.all(np.isneginf(lse[:5])) and np.all(out[48:48 + 64] == 0)


@pytest.mark.parametrize("g,G,d_h,d_v,lens,ns", [(2, 4, 128, 128, [3000, 40], [3, 2]), (4, 5, 192, 256, [1500], [20]), (1, 1, 128, 128, [5000], [1]),
                                                  (5, 4, 192, 256, [1500], [250]), (4, 8, 128, 128, [1100], [300])])
def test_attend_splits_a_long_context(g, G, d_h, d_v, lens, ns):
    w = World(lens, g, d_h, d_v, G=G, P=256, seed=101 + g)
    w.append(lens)
    q_c, q_r = stored(w.r.normal(size=(sum(ns), g * G, d_h))), stored(w.r.normal(size=(sum(ns), g * G, D_R)))
    out, lse, first, need = attend(w, ns, lens, q_c, q_r, extra=2)
    assert need > 0
    w.check_attention(out, lse, q_c, q_r, first, lens)


@pytest.mark.parametrize("g,G,d_h,d_v", [(4, 8, 128, 128), (4, 5, 192, 256)])
def test_log_sum_exps_have_fp32_accuracy(g, G, d_h, d_v):
    """Logits are sums of d_h + d_R products in fp32: each addition is off by at most 2^-24 of a partial sum, at random, so the sum by
    about sqrt(d_h + d_R) * 2^-24 = 1e-6 of the partial sums' size, which is the logits' own (cancellation leaves a fraction of them, a
    sum over hundreds of tokens averages).  Relative to the log-sum-exps, in the 2-norm: below 1e-6."""
    lens, ns = [700, 300], [40, 60]
    w = World(lens, g, d_h, d_v, G=G, seed=171 + g)
    w.append(lens)
    q_c, q_r = stored(w.r.normal(size=(100, g * G, d_h))), stored(w.r.normal(size=(100, g * G, D_R)))
    _, lse, first, _ = attend(w, ns, lens, q_c, q_r)
    want = np.concatenate([FB.attend(q_c[first[b]:first[b + 1]], q_r[first[b]:first[b + 1]], w.K[b].values(), w.V[b].values(),
                                     stored(w.kr_held(b)), lens[b])[1] for b in range(2)])
    assert np.linalg.norm(lse - want) <= 1e-6 * np.linalg.norm(want)


def test_a_nan_stays_in_its_sequence():
    """One sequence's NaN (a value of an old token) reaches its own rows and no others'."""
    lens = [90, 70]
    w = World(lens, 2, G=4, seed=111)
    k, v, kr = w.draw_rows(160)
    v[3, 0, 0] = np.nan
    w.append(lens, rows=(k, v, kr))
    q_c, q_r = stored(w.r.normal(size=(20, 8, 128))), stored(w.r.normal(size=(20, 8, D_R)))
    out, lse, _, _ = attend(w, [10, 10], lens, q_c, q_r)
    assert np.all(np.isnan(out[:10, :4, 0])) and np.all(np.isfinite(out[:10, :, 1:])) and np.all(np.isfinite(out[10:])) and np.all(np.isfinite(lse))


def test_pages_beyond_4_gib():
    """Pages at the end of a pool of 5.2 GB: appends, conversion, both attention calls."""
    lens = [130, 70]
    w = World(lens, 8, G=2, seed=151, s_q=1)
    pages = 38000
    w.table = np.where(w.table >= 0, w.table + pages - w.pages, -1).astype(np.int32)
    w.d_table = torch.from_numpy(w.table).cuda()
    w.pool = torch.zeros((pages, w.bytes), dtype=torch.uint8, device="cuda")
    assert int(w.table[w.table >= 0].min()) * w.bytes > 1 << 32
    shift, w.pages = pages - w.pages, pages
    w.append(lens)
    # the few pages that hold something, as a pool of their own
    small = World(lens, 8, G=2, seed=151, s_q=1)
    small.K, small.V, small.kr = w.K, w.V, w.kr
    small.pool = w.pool[shift:].clone()
    assert not bool(w.pool[:shift].any())
    q_c, q_r = stored(w.r.normal(size=(30, 16, 128))), stored(w.r.normal(size=(30, 16, D_R)))
    out, lse, first, _ = attend(w, [20, 10], lens, q_c, q_r)
    small.check_attention(out, lse, q_c, q_r, first, lens)
    plan = B.gqla_plan_create(w.shape, w.lens(), w.P, NUM_CUS, B.GQLA_PATH_GQA)
    ws = torch.empty(B.gqla_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    B.gqla_plan_upload(plan, ws)
    out, lse = torch.empty((2, 16, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 16), device="cuda")
    B.gqla_decode_gqa_fp8_blocks(w.shape, plan, bf16(q_c[:2]).cuda(), bf16(q_r[:2]).cuda(), w.cache(), out, lse, ws)
    torch.cuda.synchronize()
    B.gqla_plan_destroy(plan)
    small.check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), q_c[:2], q_r[:2], [0, 1, 2], lens)


# ---- together -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("g,G,d_h,d_v", [(8, 4, 128, 128), (4, 5, 192, 256)])
def test_prompts_then_steps(g, G, d_h, d_v):
    """Two chunks of a prompt appended and attended, then decode steps: each against fp64 on what the cache holds."""
    w = World([150, 90, 80], g, d_h, d_v, G=G, seed=121 + g, s_q=2)
    for ns in ([70, 33, 1], [64, 40, 65]):
        q_r, q_rot, first, _ = w.append(ns)
        q_c = stored(w.r.normal(size=(sum(ns), g * G, d_h)))
        out, lse, first, _ = attend(w, ns, w.lens(), q_c, q_rot)
        w.check_attention(out, lse, q_c, q_rot, first, w.lens())
    for _ in range(2):
        _, q_rot, first, _ = w.append([2, 2, 2], uniform=True)
        q_c = stored(w.r.normal(size=(6, g * G, d_h)))
        plan = B.gqla_plan_create(w.shape, w.lens(), w.P, NUM_CUS, B.GQLA_PATH_GQA)
        ws = torch.empty(B.gqla_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
        B.gqla_plan_upload(plan, ws)
        out, lse = torch.empty((6, g * G, d_v), dtype=torch.bfloat16, device="cuda"), torch.empty((6, g * G), device="cuda")
        B.gqla_decode_gqa_fp8_blocks(w.shape, plan, bf16(q_c).cuda(), bf16(q_rot).cuda(), w.cache(), out, lse, ws)
        torch.cuda.synchronize()
        B.gqla_plan_destroy(plan)
        w.check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), q_c, q_rot, first, w.lens())
    w.check_pool()


def test_recorded_append_and_attend_serve_other_lengths():
    """One graph of append and attention, replayed with other lengths, bounds and rows in the same buffers, equals eager calls."""
    g, G, cap = 2, 4, 96
    w = World([200, 200], g, G=G, seed=131)
    w.append([50, 20])
    first, lens = torch.tensor([0, 30, 70], dtype=torch.int32, device="cuda"), torch.tensor([80, 60], dtype=torch.int32, device="cuda")
    w.d_lens = lens
    make = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    k, v, kr, q_r, q_rot, q_c = make(cap, g * 128), make(cap, g * 128), make(cap, D_R), make(cap, g * G, D_R), make(cap, g * G, D_R), make(cap, g * G, 128)
    out, lse = torch.zeros_like(q_c), torch.zeros((cap, g * G), device="cuda")
    ws = torch.empty(max(16, B.gqla_attend_gqa_workspace_bytes(w.shape, first, cap, w.cache())), dtype=torch.uint8, device="cuda")
    start = w.pool.clone()

    def step():
        B.gqla_append_expanded_fp8_blocks(w.shape, B.make_new_rows(k, v, kr, q_r, q_rot, first, cap), BASE, w.cache())
        B.gqla_attend_gqa_fp8_blocks(w.shape, first, cap, q_c, q_rot, w.cache(), out, lse, ws)

    def inputs(seed, f, n):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for t in (k, v, kr, q_r, q_c):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        first.copy_(torch.tensor(f, dtype=torch.int32))
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        w.pool.copy_(start)
        out.fill_(7.0), lse.fill_(7.0), q_rot.fill_(7.0)
        torch.cuda.synchronize()

    inputs(1, [0, 30, 70], [80, 60])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed, f, n in ((2, [0, 30, 70], [80, 60]), (3, [0, 1, 1], [51, 20]), (4, [0, 0, 96], [50, 116]), (5, [3, 60, 61], [107, 21])):
        inputs(seed, f, n)
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (w.pool, out, lse, q_rot)]
        inputs(seed, f, n)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (w.pool, out, lse, q_rot)):
            assert torch.equal(a, b), (seed, f)


def test_two_streams_at_once():
    worlds = [World([300, 100], 2, G=4, seed=141 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in worlds]
    jobs = []
    for w in worlds:
        w.append([300, 100])
        q_c, q_r = stored(w.r.normal(size=(50, 8, 128))), stored(w.r.normal(size=(50, 8, D_R)))
        first = torch.tensor([0, 30, 50], dtype=torch.int32, device="cuda")
        out, lse = torch.zeros((50, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((50, 8), device="cuda")
        ws = torch.empty(max(16, B.gqla_attend_gqa_workspace_bytes(w.shape, first, 50, w.cache())), dtype=torch.uint8, device="cuda")
        jobs.append((w, first, bf16(q_c).cuda(), bf16(q_r).cuda(), out, lse, ws, q_c, q_r))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (w, first, dq, dr, out, lse, ws, _, _) in zip(streams, jobs):
            B.gqla_attend_gqa_fp8_blocks(w.shape, first, 50, dq, dr, w.cache(), out, lse, ws, stream=s)
    torch.cuda.synchronize()
    for w, _, _, _, out, lse, _, q_c, q_r in jobs:
        w.check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), q_c, q_r, [0, 30, 50], w.lens())


def test_decoder_from_the_cache_switch():
    """The harness's way: latent cache expanded, converted to block scales, a step's rows appended, decoded; and the same step as
    a chunk: both attention calls agree on the same rows."""
    import synth_inputs as S
    from test_gpu_parity import Case
    cfg = S.CONFIGS["C3"].with_(B=2, L=0, paged=True, seed=990)
    case = Case(cfg, lens=[200, 66])
    dec = case.dec
    try:
        dec.alloc_expanded(fill=0.0)
        dec.expand(case.d_w_uk, case.d_w_uv)
        dec.alloc_expanded_blocks()
        dec.quantize_expanded_blocks()
        gen = torch.Generator(device="cuda").manual_seed(3)
        new = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
        q_r = new(4, cfg.h_q, cfg.d_r)
        q_rot = dec.append_expanded(BASE, new(4, cfg.g * cfg.d_h), new(4, cfg.g * cfg.d_h), new(4, cfg.d_r), q_r, blocks=True)
        out, lse = dec.decode_gqa_blocks(case.d_q_c, q_rot.view(2, 2, cfg.h_q, cfg.d_r))
        out2, lse2 = dec.attend_gqa_blocks(case.d_q_c.view(4, cfg.h_q, cfg.d_h), q_rot)
        torch.cuda.synchronize()
        a, b = out.float().view(4, cfg.h_q, -1), out2.float()
        # both round the probabilities (2^-8 of a value each, values up to max |V| of the row) and the result
        assert float((a - b).abs().max()) <= 4 * EPS * 5.0
        assert float((lse.view(4, -1) - lse2).abs().max()) <= 1e-4
    finally:
        case.close()


def test_decoder_takes_one_row_and_none():
    """A tensor of one row may name any stride; one of none has no address."""
    import synth_inputs as S
    from test_gpu_parity import Case
    cfg = S.CONFIGS["C3"].with_(B=1, L=0, s_q=1, paged=True, seed=991)
    case = Case(cfg, lens=[40])
    dec = case.dec
    try:
        row = lambda d: torch.randn(d, device="cuda").to(torch.bfloat16)  # noqa: E731
        k, v, kr = row(cfg.g * cfg.d_h), row(cfg.g * cfg.d_h), row(cfg.d_r)
        pools = []
        for odd in (False, True):
            shaped = [torch.as_strided(x, (1, x.numel()), (1, 1)) if odd else x.view(1, -1) for x in (k, v, kr)]
            pool = dec.alloc_expanded_blocks()
            dec.append_expanded(BASE, *shaped, blocks=True)
            pools.append(pool)
        torch.cuda.synchronize()
        assert bool((pools[0] != 0xAA).any()) and torch.equal(*pools)
        before = pools[1].clone()
        none = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        first = torch.zeros(2, dtype=torch.int32, device="cuda")
        q_rot = dec.append_expanded(BASE, none(0, cfg.g * cfg.d_h), none(0, cfg.g * cfg.d_h), none(0, cfg.d_r), none(0, cfg.h_q, cfg.d_r), first, blocks=True)
        out, lse = dec.attend_gqa_blocks(none(0, cfg.h_q, cfg.d_h), q_rot, first)
        torch.cuda.synchronize()
        assert out.shape == (0, cfg.h_q, cfg.d_h) and torch.equal(pools[1], before)
    finally:
        case.close()
