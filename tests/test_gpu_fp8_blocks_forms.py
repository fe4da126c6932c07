"""The forms that the decode over block scales takes where no chunk is shared out among waves, each with odd and even numbers of tiles,
sequences that end early and a page that is not there; the rotation of many heads, two tokens a workgroup, far out; the calls without a
page table or row bounds, and in tables far longer than the sequences."""
import numpy as np
import pytest
import torch

from oracle import gqla_oracle as O
from paper_2605_15250_amd import binding as B
from test_gpu_fp8_blocks import BASE, D_R, EPS, World, bf16, stored

pytestmark = pytest.mark.gpu

# (g, G, d_h, d_v, s_q, P, lens, pages of a chunk); planned for two units, whose 16 waves (8 of 192 dims) have more items than that
FORMS = {
    # two tiles of codes in flight: k_R shared by the eight waves of a workgroup, chunks long against the rows of a group
    "two_tiles": (8, 4, 128, 128, 1, 64, [700, 31, 33, 640], 4),
    "two_tiles_16_groups": (16, 2, 128, 128, 2, 64, [450, 3, 193, 64], 2),
    "two_tiles_32_rows": (8, 16, 128, 128, 2, 64, [1200, 577], 9),
    "two_tiles_large_pages": (8, 3, 128, 128, 1, 256, [1500, 255], 1),
    # one tile: more rows or short chunks; two and four waves with a shared k_R; no shared k_R
    "shared_32_rows": (8, 16, 128, 128, 2, 64, [450, 193, 2], 2),
    "shared_one_page": (8, 4, 128, 128, 1, 64, [300, 65, 1], 1),
    "two_waves": (2, 16, 128, 128, 2, 64, [500, 100], 3),
    "four_waves": (4, 20, 128, 128, 1, 64, [400, 97, 520], 3),
    "own_k_r": (3, 5, 128, 128, 2, 64, [700, 130], 3),
    "two_row_blocks": (4, 32, 128, 128, 2, 64, [300, 129, 65], 2),
    # 192 key dims, chunks of less than six tiles
    "wide_shared": (4, 5, 192, 256, 2, 64, [450, 3, 200], 2),
    "wide_shared_one_page": (8, 4, 192, 256, 1, 64, [300, 33, 65], 1),
    "wide_own_k_r": (5, 4, 192, 256, 2, 64, [300, 130], 2),
    "wide_one_group": (1, 16, 192, 256, 2, 64, [600, 130], 1),
    "wide_two_waves": (2, 20, 192, 256, 1, 64, [500, 70], 2),
    "wide_row_blocks": (2, 40, 192, 256, 1, 64, [200, 90], 2),
    "wide_two_tiles": (4, 5, 192, 256, 2, 64, [450, 3, 200, 193], 3),
}


def decode(w, q_c, q_r, chunk=0, units=2):
    """q_c, q_r [sequences * s_q][heads][dim] -> out, lse as the call leaves them"""
    plan = B.gqla_plan_create(w.shape, w.lens(), w.P, units, B.GQLA_PATH_GQA, chunk)
    try:
        ws = torch.empty(B.gqla_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
        B.gqla_plan_upload(plan, ws)
        out = torch.full((w.B * w.s_q, w.g * w.G, w.d_v), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((w.B * w.s_q, w.g * w.G), 7.0, device="cuda")
        B.gqla_decode_gqa_fp8_blocks(w.shape, plan, bf16(q_c).cuda(), bf16(q_r).cuda(), w.cache(), out, lse, ws)
        torch.cuda.synchronize()
    finally:
        B.gqla_plan_destroy(plan)
    return out.float().cpu().numpy(), lse.cpu().numpy()


@pytest.mark.parametrize("form", FORMS)
def test_decode_without_teams(form):
    g, G, d_h, d_v, s_q, P, lens, chunk = FORMS[form]
    w = World(lens, g, d_h, d_v, G=G, P=P, seed=201 + sorted(FORMS).index(form), s_q=s_q)
    w.append(lens)
    w.spoil()
    first = np.arange(w.B + 1) * s_q
    q_c, q_r = stored(w.r.normal(size=(w.B * s_q, g * G, d_h))), stored(w.r.normal(size=(w.B * s_q, g * G, D_R)))
    out, lse = decode(w, q_c, q_r, chunk)
    w.check_attention(out, lse, q_c, q_r, first, w.lens())
    hidden = [np.zeros(n, bool) for n in lens]
    hidden[0][P:2 * P] = True
    held = [w.kr_held(b) for b in range(w.B)]             # (read through the whole table)
    w.kr_held = lambda b: held[b]
    w.table[0, 1] = w.pages
    w.d_table = torch.from_numpy(w.table).cuda()
    out, lse = decode(w, q_c, q_r, chunk)
    w.check_attention(out, lse, q_c, q_r, first, w.lens(), hidden)


@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("g,G,d_h,d_v", [(8, 4, 128, 128), (4, 32, 128, 128), (8, 16, 192, 256)])
def test_rotation_of_many_heads_far_out(g, G, d_h, d_v, blocks):
    """More rows than a step's and 32 heads or more: two tokens a workgroup.  Rows begin at odd and even positions inside a block, up to a hundred
    thousand.  The angle is reduced in double, then within 2 pi 2^-25 of its fp32 form; sine, cosine and rotation within 2^-22 of
    |x|, which is below 8: 2^-20 * 8 for all of that, and the result's own rounding."""
    P, ns, old = 64, [37, 5, 66, 1], [40001, 98302, 0, 65535]
    r = np.random.default_rng(301 + g + G)
    lens = np.array(old) + ns
    max_pages = int(-(-lens.max() // P))
    table, at = np.full((4, max_pages), -1, np.int32), 0
    for b in range(4):
        for p in range(old[b] // P, (int(lens[b]) - 1) // P + 1):
            table[b, p], at = at, at + 1
    total, heads = sum(ns), g * G
    pos = np.concatenate([old[b] + np.arange(ns[b]) for b in range(4)])
    q, kr = stored(r.normal(size=(total, heads, D_R))), stored(r.normal(size=(total, D_R)))
    assert np.abs(q).max() < 8 and np.abs(kr).max() < 8
    first = torch.from_numpy(np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)).cuda()
    d_lens, d_table = torch.from_numpy(lens.astype(np.int32)).cuda(), torch.from_numpy(table).cuda()
    shape = B.make_shape(4, heads, g, d_h, 512, D_R, 1, B.GQLA_BF16, 0.0, d_v)
    codes = g * (d_h + d_v) * (1 if blocks else 2)        # bytes of a token's keys and values
    page = B.gqla_expanded_fp8_blocks_page_bytes(g, d_h, d_v, D_R, P) if blocks else P * (codes + 2 * D_R)
    pool = torch.zeros((at, page), dtype=torch.uint8, device="cuda")
    zeros = lambda d: torch.zeros((total, g * d), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    k, v, d_kr, d_q = zeros(d_h), zeros(d_v), bf16(kr).cuda(), bf16(q).cuda()
    q_rot = torch.full_like(d_q, 7.0)
    call = B.gqla_append_expanded_fp8_blocks if blocks else B.gqla_append_expanded
    call(shape, B.make_new_rows(k, v, d_kr, d_q, q_rot, first, total), BASE, B.make_cache(pool, d_lens, d_table, P, max_pages, at, g))
    torch.cuda.synchronize()
    want = O.rope(q, pos[:, None], BASE)
    assert np.all(np.abs(q_rot.float().cpu().numpy() - want) <= EPS * np.abs(want) + 2.0 ** -20 * 8)
    seq = np.repeat(np.arange(4), ns)
    held = pool[:, P * codes: P * (codes + 2 * D_R)].contiguous().view(torch.bfloat16).view(at, D_R // 8, P, 8).float().cpu().numpy()
    got = held[table[seq, pos // P], :, pos % P].reshape(total, D_R)
    want = O.rope(kr, pos, BASE)
    assert np.all(np.abs(got - want) <= EPS * np.abs(want) + 2.0 ** -20 * 8)


@pytest.mark.parametrize("g,G,d_h,d_v,P", [(2, 4, 128, 128, 64), (8, 16, 128, 128, 1024), (5, 4, 192, 256, 128)])
def test_without_a_page_table_and_without_row_bounds(g, G, d_h, d_v, P):
    """Sequence b's pages are b max_pages ..; every sequence has s_q rows: appended, attended as a chunk and decoded, in a cache whose rows of pages
    are longer than the sequences."""
    lens = [300, 2, 129]
    w = World([n + 2 for n in lens], g, d_h, d_v, G=G, P=P, seed=231 + g, s_q=2, table=False)
    w.append(lens)
    _, q_rot, first, _ = w.append([2, 2, 2], uniform=True)
    w.check_pool()
    w.spoil()
    q_c = stored(w.r.normal(size=(6, g * G, d_h)))
    out, lse = decode(w, q_c, q_rot, units=256)
    w.check_attention(out, lse, q_c, q_rot, first, w.lens())
    out = torch.full((6, g * G, d_v), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((6, g * G), 7.0, device="cuda")
    need = B.gqla_attend_gqa_workspace_bytes(w.shape, None, 6, w.cache())
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    B.gqla_attend_gqa_fp8_blocks(w.shape, None, 6, bf16(q_c).cuda(), bf16(q_rot).cuda(), w.cache(), out, lse, ws)
    torch.cuda.synchronize()
    w.check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), q_c, q_rot, first, w.lens())


@pytest.mark.parametrize("g,G,d_h,d_v", [(8, 4, 128, 128), (4, 5, 192, 256)])
def test_attention_in_tables_far_longer_than_the_sequences(g, G, d_h, d_v):
    """Ranges for contexts that no sequence has: most see nothing, and the joined result is the one without them."""
    lens, ns = [150, 1, 97, 200], [150, 1, 60, 130]
    w = World(lens, g, d_h, d_v, G=G, seed=241 + g)
    w.append(lens)
    w.spoil()
    table = np.full((w.B, 2048), w.pages + 7, np.int32)   # 131072 tokens; entries behind a sequence name no page
    table[:, :w.max_pages] = w.table
    wide = torch.from_numpy(table).cuda()
    q_c, q_r = stored(w.r.normal(size=(sum(ns), g * G, d_h))), stored(w.r.normal(size=(sum(ns), g * G, D_R)))
    first = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
    d_first = torch.from_numpy(first).cuda()
    cache = B.make_cache(w.pool, w.d_lens, wide, w.P, 2048, w.pages, g)
    need = B.gqla_attend_gqa_workspace_bytes(w.shape, d_first, sum(ns), cache)
    assert need > B.gqla_attend_gqa_workspace_bytes(w.shape, d_first, sum(ns), w.cache())
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((sum(ns), g * G, d_v), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((sum(ns), g * G), 7.0, device="cuda")
    B.gqla_attend_gqa_fp8_blocks(w.shape, d_first, sum(ns), bf16(q_c).cuda(), bf16(q_r).cuda(), cache, out, lse, ws)
    torch.cuda.synchronize()
    w.check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), q_c, q_r, first, lens)
