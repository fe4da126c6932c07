"""The block-scaled 8-bit expanded cache without a GPU: the oracle's rule and page against their definitions, the refusals of the
entry points, the sizes that they report."""
import numpy as np
import pytest

from oracle import fp8_blocks as FB
from oracle import fp8_cache as F8
from oracle import gqla_oracle as O
from paper_2605_15250_amd import binding as B


def _refused(status, fn, *args, **kw):
    with pytest.raises(B.GqlaError) as e:
        fn(*args, **kw)
    assert e.value.status == status, (B.status_string(e.value.status), B.status_string(status))


@pytest.mark.parametrize("amax,e", [(448.0, 0), (449.0, 1), (447.0, 0), (224.0, -1), (1.0, -8), (1.75, -8), (1.7578125, -7), (0.0, -100),
                                    (2.0 ** -120, -100), (448.0 * 2.0 ** -100, -100), (450.0 * 2.0 ** -100, -99), (3e38, 118)])
def test_exponent_of_a_block(amax, e):
    assert FB.block_exponent([amax, -amax / 3, float("nan"), float("inf")]) == e


def test_oracle_append_is_independent_of_the_cuts_where_codes_stay_normal():
    r = np.random.default_rng(5)
    x = np.sign(r.normal(size=(77, 2, 32))) * r.uniform(1.0, 2.0, (77, 2, 32)) * 2.0 ** r.integers(0, 4, (77, 1, 1))
    x = x.astype(np.float32)
    whole = FB.Plane(2, 32).append(x)
    cuts = FB.Plane(2, 32)
    for a, b in ((0, 1), (1, 31), (31, 40), (40, 40), (40, 64), (64, 77)):
        cuts.append(x[a:b])
    assert np.array_equal(whole.e, cuts.e) and np.array_equal(whole.codes, cuts.codes)
    # every value within half a step of its code: 2^-4 relative (normal codes)
    assert np.all(np.abs(whole.values() - x) <= 2.0 ** -4 * np.abs(x))


def test_oracle_page_is_tiled_once():
    P, g, d_h, d_v, d_r = 64, 2, 64, 96, 16
    seen = np.zeros(FB.page_bytes(P, g, d_h, d_v, d_r), int)
    for s in range(P):
        for d in range(d_r):
            o = FB.kr_offset(s, d, P, g, d_h, d_v, d_r)
            seen[o: o + 2] += 1
        for j in range(g):
            for d in range(d_h):
                seen[FB.k_offset(j, s, d, P, g, d_h, d_v, d_r)] += 1
            for d in range(d_v):
                seen[FB.v_offset(j, s, d, P, g, d_h, d_v, d_r)] += 1
    for j in range(g):
        for T in range(P // 32):
            for kind in range(2):
                o = FB.scale_offset(j, T, kind, P, g, d_h, d_v, d_r)
                seen[o: o + 4] += 1
    assert np.all(seen == 1)
    # the planes of codes are those of the cache with one scale
    assert FB.k_offset(1, 37, 45, P, g, 64, 64, 16) == F8.k8_offset(0, 1, 37, 45, P, g, 64, 16)
    assert FB.v_offset(1, 37, 45, P, g, 64, 64, 16) == F8.v8_offset(0, 1, 37, 45, P, g, 64, 16)


def test_oracle_attend_is_the_decode_of_its_last_rows():
    r = np.random.default_rng(6)
    L, n, g, h_q, d_h, d_r, d_v = 21, 6, 2, 6, 16, 8, 24
    K, V, kR = r.normal(size=(L, g, d_h)), r.normal(size=(L, g, d_v)), r.normal(size=(L, d_r))
    qC, qR = r.normal(size=(n, h_q, d_h)), r.normal(size=(n, h_q, d_r))
    o, lse, _ = FB.attend(qC, qR, K, V, kR, L)
    want, want_lse = O.decode_gqa(qC, qR, K, V, kR)
    assert np.max(np.abs(o - want)) < 1e-12 and np.max(np.abs(lse - want_lse)) < 1e-12
    o, lse, _ = FB.attend(qC, qR, K[:2], V[:2], kR[:2], 2)        # four rows ahead of the first token
    assert np.all(o[:4] == 0) and np.all(np.isneginf(lse[:4])) and np.all(np.isfinite(lse[4:]))


A = 0x10000


def _shape(batch=2, h_q=32, g=8, d_h=128, s_q=1, dtype=B.GQLA_BF16, d_v=0):
    return B.make_shape(batch, h_q, g, d_h, 512, 64, s_q, dtype, 0.0, d_v)


def _cache(page=64, max_pages=4, num_pages=8, groups=8, pool=A, lens=A, table=None):
    return B.make_cache(pool, lens, table, page, max_pages, num_pages, groups)


def _rows(k_c=A, v=A, k_r=A, q_r=None, q_rot=None, first=A, total=5, **strides):
    return B.make_new_rows(k_c, v, k_r, q_r, q_rot, first, total, **strides)


@pytest.mark.parametrize("fn", ["gqla_append_expanded", "gqla_append_expanded_fp8_blocks"])
def test_append_refusals(fn):
    call = lambda shape=_shape(), rows=_rows(), base=1e4, cache=_cache(): getattr(B, fn)(shape, rows, base, cache, stream=0)  # noqa: E731
    for missing in ({"k_c": None}, {"v": None}, {"k_r": None}, {"q_r": A}, {"q_rot": A}):
        _refused(B.GQLA_ERR_NULL, call, rows=_rows(**missing))
    for odd in ({"k_c": A + 2}, {"v": A + 8}, {"k_r": A + 4}, {"q_r": A + 8, "q_rot": A}, {"q_r": A, "q_rot": A + 8}, {"first": A + 2},
                {"k_stride": 1028}, {"v_stride": 1025}, {"kr_stride": 66}):
        _refused(B.GQLA_ERR_ALIGN, call, rows=_rows(**odd))
    for wrong in ({"total": -1}, {"total": (1 << 23) + 1}, {"k_stride": 1016}, {"v_stride": 8}, {"kr_stride": 56}, {"k_stride": -1024},
                  {"first": None, "total": 3}):
        _refused(B.GQLA_ERR_SHAPE, call, rows=_rows(**wrong))
    for base in (1.0, -2.0, 0.5, float("nan"), float("inf")):
        _refused(B.GQLA_ERR_SHAPE, call, base=base)
    _refused(B.GQLA_ERR_SHAPE, call, cache=_cache(groups=4))
    _refused(B.GQLA_ERR_SHAPE, call, shape=_shape(d_h=192))
    _refused(B.GQLA_ERR_NULL, call, cache=_cache(pool=None))
    _refused(B.GQLA_ERR_NULL, call, cache=_cache(lens=None))
    _refused(B.GQLA_ERR_ALIGN, call, cache=_cache(pool=A + 8))
    _refused(B.GQLA_ERR_PAGE, call, cache=_cache(page=48))
    _refused(B.GQLA_ERR_PAGE, call, cache=_cache(max_pages=0))
    _refused(B.GQLA_ERR_PAGE, call, cache=_cache(num_pages=7))           # without a table every row has its own pages
    if fn == "gqla_append_expanded_fp8_blocks":
        _refused(B.GQLA_ERR_DTYPE, call, shape=_shape(d_h=16, dtype=B.GQLA_F32), cache=_cache(page=16))
    call(rows=_rows(total=0))                                            # nothing to do: no launch
    call(shape=_shape(batch=0), cache=_cache())
    call(shape=_shape(batch=0, s_q=2), rows=_rows(first=None, total=0))


def test_calls_without_rows_take_buffers_without_an_address():
    """An empty tensor's address is NULL: a step in which no sequence has a new token."""
    none = _rows(k_c=None, v=None, k_r=None, total=0)
    for fn in (B.gqla_append_expanded, B.gqla_append_expanded_fp8_blocks):
        fn(_shape(), none, 1e4, _cache(), stream=0)
        fn(_shape(), _rows(k_c=None, v=None, k_r=None, q_r=A, total=0), 1e4, _cache(), stream=0)
    B.gqla_attend_gqa_fp8_blocks(_shape(), A, 0, None, None, _cache(), None, None, None, 0, stream=0)
    _refused(B.GQLA_ERR_ALIGN, B.gqla_attend_gqa_fp8_blocks, _shape(), A, 0, A + 8, None, _cache(), None, None, None, 0, stream=0)


def test_quantize_and_decode_refusals():
    q = lambda shape=_shape(), a=_cache(), b=_cache(): B.gqla_quantize_expanded_fp8_blocks(shape, a, b, stream=0)  # noqa: E731
    _refused(B.GQLA_ERR_DTYPE, q, shape=_shape(d_h=16, dtype=B.GQLA_F32))
    _refused(B.GQLA_ERR_SHAPE, q, shape=_shape(d_h=192))
    _refused(B.GQLA_ERR_SHAPE, q, b=_cache(groups=4))
    _refused(B.GQLA_ERR_SHAPE, q, a=_cache(groups=16), b=_cache(groups=16))
    _refused(B.GQLA_ERR_NULL, q, a=_cache(lens=None))
    _refused(B.GQLA_ERR_NULL, q, b=_cache(pool=None))
    _refused(B.GQLA_ERR_ALIGN, q, b=_cache(pool=A + 4))
    _refused(B.GQLA_ERR_PAGE, q, b=_cache(page=128))
    _refused(B.GQLA_ERR_PAGE, q, b=_cache(max_pages=3))
    _refused(B.GQLA_ERR_PAGE, q, b=_cache(num_pages=7))
    q(shape=_shape(batch=0))
    sh = _shape()
    plan = B.gqla_plan_create(sh, [100, 200], 64, 256, B.GQLA_PATH_GQA)
    try:
        d = lambda shape=sh, p=plan, qc=A, cache=_cache(), out=A: B.gqla_decode_gqa_fp8_blocks(shape, p, qc, A, cache, out, None, A, 1 << 40, stream=0)  # noqa: E731
        _refused(B.GQLA_ERR_DTYPE, d, shape=_shape(d_h=16, dtype=B.GQLA_F32))
        _refused(B.GQLA_ERR_NULL, d, qc=None)
        _refused(B.GQLA_ERR_ALIGN, d, out=A + 8)
        _refused(B.GQLA_ERR_PLAN, d, shape=_shape(s_q=2))
        _refused(B.GQLA_ERR_SEQLEN, d, cache=_cache(max_pages=3))
        _refused(B.GQLA_ERR_WORKSPACE, d)                                # the plan's table is in no workspace
    finally:
        B.gqla_plan_destroy(plan)


def test_attend_refusals_and_workspace():
    sh = _shape()

    def call(shape=sh, first=A, total=5, q_c=A, q_r=A, cache=_cache(), out=A, lse=A, ws=A, ws_bytes=1 << 40):
        B.gqla_attend_gqa_fp8_blocks(shape, first, total, q_c, q_r, cache, out, lse, ws, ws_bytes, stream=0)
    _refused(B.GQLA_ERR_DTYPE, call, shape=_shape(d_h=16, dtype=B.GQLA_F32), cache=_cache(page=16))
    for null in ("q_c", "q_r", "out"):
        _refused(B.GQLA_ERR_NULL, call, **{null: None})
    for odd in ({"q_c": A + 8}, {"q_r": A + 2}, {"out": A + 4}, {"lse": A + 2}, {"ws": A + 4}, {"first": A + 1}):
        _refused(B.GQLA_ERR_ALIGN, call, **odd)
    _refused(B.GQLA_ERR_SHAPE, call, total=-1)
    _refused(B.GQLA_ERR_SHAPE, call, first=None, total=7)
    _refused(B.GQLA_ERR_SHAPE, call, shape=_shape(h_q=1 << 14, g=8), total=1 << 20)      # 2^31 query rows of a group
    _refused(B.GQLA_ERR_SHAPE, call, shape=_shape(h_q=1 << 12, g=1 << 11), cache=_cache(groups=1 << 11), total=1 << 20)   # 2^25 workgroups
    _refused(B.GQLA_ERR_SHAPE, call, shape=_shape(batch=(1 << 20) + 1), cache=_cache(num_pages=1 << 23))
    _refused(B.GQLA_ERR_SHAPE, call, shape=_shape(h_q=1 << 16, g=1 << 14), cache=_cache(groups=1 << 14, page=1024), total=8)   # a page of 2^32 bytes
    _refused(B.GQLA_ERR_SHAPE, call, cache=_cache(groups=7))
    _refused(B.GQLA_ERR_PAGE, call, cache=_cache(page=96))
    call(total=0)
    call(shape=_shape(batch=0))
    # few rows over a long context need partial outputs: whole (rows, splits) of d_v + 1 floats; many rows none
    long = _cache(max_pages=512, num_pages=1024)
    need = B.gqla_attend_gqa_workspace_bytes(sh, A, 5, long)
    assert need > 0 and need % (5 * 32 * 129 * 4) == 0
    _refused(B.GQLA_ERR_WORKSPACE, call, cache=long, ws_bytes=need - 1)
    _refused(B.GQLA_ERR_WORKSPACE, call, cache=long, ws=None)
    assert B.gqla_attend_gqa_workspace_bytes(sh, A, 1 << 20, long) == 0
    assert B.gqla_attend_gqa_workspace_bytes(sh, A, 0, long) == 0
    assert B.gqla_attend_gqa_workspace_bytes(sh, A, -3, long) == 0


def test_page_bytes():
    for P, g, d_h, d_v in ((64, 8, 128, 128), (128, 5, 192, 256), (1024, 1, 128, 128)):
        assert B.gqla_expanded_fp8_blocks_page_bytes(g, d_h, d_v, 64, P) == FB.page_bytes(P, g, d_h, d_v, 64)
        assert FB.page_bytes(P, g, d_h, d_v, 64) % 16 == 0
    for bad in ((0, 128, 128, 64, 64), (8, 0, 128, 64, 64), (8, 128, 128, 64, 48), (8, 128, 128, 64, 0), (8, 128, -1, 64, 64)):
        assert B.gqla_expanded_fp8_blocks_page_bytes(*bad) == 0
