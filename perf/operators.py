"""The expanded cache filled from rows and read in blocks of 8 bits: each operator in its plain form and as the library's call.

    op               what one pass runs
    append           rows K_C | V | k_R of new tokens into the 16-bit (or fp32) expanded cache, k_R and the queries rotated
    append_blocks    the same into the 8-bit cache with a scale per block of 32 tokens and group
    quantize         a 16-bit expanded cache converted into the 8-bit one
    decode           a step of one or two tokens per sequence over the 8-bit cache
    attend           prompt chunks, any number of query rows per sequence, over the 8-bit cache

The 8-bit page of P tokens and g groups (bytes; d_h, d_v multiples of 32):
    K8     [g][d_h/32][2][P][2][8]     dim 32 x + 16 u + 8 h + i of slot s at [x][h][s][u][i]
    V8     [g][P/32][d_v][2][2][8]     slot 32 T + 16 u + 8 h + i of dim d at [T][d][h][u][i]
    k_R    [d_r/8][P][8] bf16          scales [g][P/32][2] fp32, the block's powers of two for K and V
A block's exponent is the smallest e in [-100, 118] with max |x| <= 448 * 2^e; a code is E4M3(x * 2^-e).  Rows appended to a block
that holds older tokens raise its exponent where they need to, and the older codes are rounded to it.

Lengths are part of the case (ragged ones are drawn from the case's own numbers); values and page tables follow the seed.
"""
import math
import random

import torch

own = False

BASE = 10000.0
BLOCK = 32
E_MIN, E_MAX = -100, 118

# (h_q, g, d_h, d_v): 128 heads in 8 or 4 groups, 64 and 32 heads, one rank's 16 heads, 20 heads with dims of their own
HEADS = {
    "h128g8": (128, 8, 128, 128),
    "h128g4": (128, 4, 128, 128),
    "h64g8": (64, 8, 128, 128),
    "h32g8": (32, 8, 128, 128),
    "h16g1": (16, 1, 128, 128),
    "h20g4": (20, 4, 192, 256),
    "h20g5": (20, 5, 192, 256),
}


# ---- cases ------------------------------------------------------------------------------------------------------------
def _case(name, op, heads, batch, l_min, l_max, n_min=0, n_max=0, page=64, paged=True, fused=False, dtype="bf16"):
    """l_min .. l_max: tokens cached ahead of the call (decode, quantize: all of them); n_min .. n_max: new tokens a sequence,
    0 .. 0 where there are none; fused: the new rows are parts of one buffer, as a joint projection writes them."""
    h_q, g, d_h, d_v = HEADS[heads] if isinstance(heads, str) else heads
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "h_q": h_q, "g": g, "d_h": d_h, "d_v": d_v, "d_r": 64,
            "l_min": l_min, "l_max": l_max, "n_min": n_min, "n_max": n_max, "page": page, "paged": paged, "fused": fused}


def listed():
    return [
        # one user's next token enters the cache: latency
        _case("append_one", "append_blocks", "h32g8", 1, 1000, 1000, 1, 1),
        # a loaded server's step with one multi-token-prediction head; blocks at every state of filling
        _case("append_step_b64", "append_blocks", "h128g8", 64, 3000, 12000, 2, 2),
        # ragged prompts behind a common beginning, rows as the joint projection left them
        _case("append_prompts", "append_blocks", "h32g8", 8, 0, 700, 500, 4000, fused=True),
        # prompts into the 16-bit cache, key and value dims of their own
        _case("append_prompts_16bit", "append", "h20g4", 4, 0, 300, 300, 3000),
        # a short session's cache converted
        _case("quantize_one", "quantize", "h32g8", 1, 333, 333),
        # the caches of a ragged batch converted after the cache switch
        _case("quantize_b32", "quantize", "h128g8", 32, 2049, 6143),
        # one user's next token: latency of the attention
        _case("decode_one", "decode", "h32g8", 1, 1000, 1000, 1, 1),
        # a few users, key and value dims of their own, two step tokens
        _case("decode_h20_b4", "decode", "h20g4", 4, 1500, 7500, 2, 2),
        # the benchmark's batch and context, two step tokens
        _case("decode_b64", "decode", "h128g8", 64, 8192, 8192, 2, 2),
        # a few new tokens over a long document: few rows, a long axis
        _case("attend_few", "attend", "h32g8", 2, 20000, 32000, 9, 16),
        # chunks of prompts behind what is cached, key and value dims of their own
        _case("attend_chunks_h20", "attend", "h20g5", 4, 1000, 3000, 100, 512),
        # whole prompts, ragged: the matrix cores' work, the largest
        _case("attend_prompts", "attend", "h128g8", 2, 0, 500, 2500, 4000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _floor_s(case):
    w = work(case)
    return max(w["bytes"] / 8e12, w["flops"] / 2.5e15)


def draw(rng):
    op = rng.choice(["append", "append_blocks", "append_blocks", "quantize", "decode", "decode", "attend", "attend"])
    most = max(_floor_s(c) for c in listed())
    heads = rng.choice(sorted(HEADS))
    page = rng.choice([64, 64, 128])
    paged = rng.random() < 0.7
    if op == "append" and rng.random() < 0.4:      # fp32: any dims that are multiples of 8
        g = rng.choice([1, 2, 3, 4])
        heads = (g * rng.randint(1, 6), g, 8 * rng.randint(2, 16), 8 * rng.randint(2, 16))
        case = _case("", op, heads, _log_int(rng, 1, 32), 0, 0, page=rng.choice([16, 24, 64]), paged=paged, dtype="f32")
    else:
        case = _case("", op, heads, _log_int(rng, 1, 128), 0, 0, page=page, paged=paged)
    del case["name"]
    case["fused"] = rng.random() < 0.5 and op in ("append", "append_blocks")
    ratio = rng.choice([1.0, 0.5, 0.1])
    l_max = _log_int(rng, 40, 32768)
    n_max = 0
    if op == "decode":
        n_max = rng.randint(1, 2)
    elif op == "attend" or (op in ("append", "append_blocks") and rng.random() < 0.5):
        n_max = _log_int(rng, 3, 4000)
    elif op != "quantize":
        n_max = rng.randint(1, 2)
    steps = n_max <= 2
    while True:
        case["l_max"], case["l_min"] = l_max, max(2 if op in ("decode", "quantize") else 0, int(l_max * ratio))
        case["n_max"], case["n_min"] = n_max, n_max if steps else int(n_max * ratio)
        logits = 4 * case["batch"] * case["h_q"] * n_max * (l_max + n_max) if op == "attend" else 0
        padded = 8 * case["batch"] * (l_max + n_max) * case["g"] * (case["d_h"] + case["d_v"])
        if _floor_s(case) <= most and logits <= 2e10 and padded <= 2e10:
            return case
        l_max = max(40, int(l_max * 0.7))
        if not steps:
            n_max = max(3, int(n_max * 0.8))
        if l_max == 40 and (steps or n_max == 3):
            case["batch"] = max(1, case["batch"] // 2)


def _lengths(case):
    """(cached tokens with the new ones, new tokens) of each sequence."""
    r = random.Random("%(batch)d %(l_min)d %(l_max)d %(n_min)d %(n_max)d" % case)
    n = [r.randint(case["n_min"], case["n_max"]) for _ in range(case["batch"])]
    if case["n_max"] > 0:
        n[0] = max(1, n[0])
    base = [r.randint(case["l_min"], case["l_max"]) for _ in range(case["batch"])]
    if case["op"] in ("decode", "quantize"):     # the step's tokens are counted already
        return base, n
    return [a + b for a, b in zip(base, n)], n


def work(case):
    lens, new = _lengths(case)
    g, d_h, d_v, d_r, h_q = (case[k] for k in ("g", "d_h", "d_v", "d_r", "h_q"))
    eb = 4 if case["dtype"] == "f32" else 2
    row, row8 = (g * (d_h + d_v) + d_r) * eb, g * (d_h + d_v) + 2 * d_r + g * 8 / BLOCK
    rows, tokens = sum(new), sum(lens)
    q_rot = 2 * rows * h_q * d_r * eb
    if case["op"] == "append":
        return {"bytes": 2 * rows * row + q_rot, "flops": 3 * rows * (h_q + 1) * d_r}
    if case["op"] == "append_blocks":
        return {"bytes": rows * (row + row8) + q_rot, "flops": 3 * rows * (h_q + 1) * d_r + 2 * rows * g * (d_h + d_v)}
    if case["op"] == "quantize":
        return {"bytes": tokens * (row + row8), "flops": 2 * tokens * g * (d_h + d_v)}
    pairs = sum(n * (L - n) + n * (n + 1) / 2 for L, n in zip(lens, new))
    return {"bytes": tokens * row8 + rows * h_q * ((d_h + d_r + d_v) * 2 + 4), "flops": 2 * h_q * (d_h + d_r + d_v) * pairs}


# ---- the pages --------------------------------------------------------------------------------------------------------
def _blocks_view(pool, c):
    """K8, V8 codes (uint8), k_R (bf16) and scales (fp32) of a pool [pages][page bytes]."""
    P, g, d_h, d_v, d_r = (c[k] for k in ("page", "g", "d_h", "d_v", "d_r"))
    n = pool.shape[0]
    a, b, e = P * g * d_h, P * g * (d_h + d_v), P * (g * (d_h + d_v) + 2 * d_r)
    return (pool[:, :a].view(n, g, d_h // 32, 2, P, 2, 8), pool[:, a:b].view(n, g, P // 32, d_v, 2, 2, 8),
            pool[:, b:e].view(torch.bfloat16).view(n, d_r // 8, P, 8), pool[:, e:].view(torch.float32).view(n, g, P // 32, 2))


def _plain_view(pool, c):
    """K_C, V and k_R of a 16-bit or fp32 pool [pages][page elements]."""
    P, g, d_h, d_v, d_r = (c[k] for k in ("page", "g", "d_h", "d_v", "d_r"))
    n = pool.shape[0]
    a, b = P * g * d_h, P * g * (d_h + d_v)
    return pool[:, :a].view(n, g, d_h // 8, P, 8), pool[:, a:b].view(n, g, P // 8, d_v, 8), pool[:, b:].view(n, d_r // 8, P, 8)


def _block_bytes(c):
    P = c["page"]
    return P * (c["g"] * (c["d_h"] + c["d_v"]) + 2 * c["d_r"]) + c["g"] * (P // 32) * 8


def _exponent(amax):
    """Smallest e in [E_MIN, E_MAX] with amax <= 448 * 2^e, for fp32 amax."""
    m, k = torch.frexp(amax)                              # amax = m 2^k, m in [1/2, 1); 448 = 0.875 * 2^9
    e = k - 9 + (m > 0.875).to(k.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX)


def _pow2(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _code(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _value(code):
    return code.view(torch.float8_e4m3fn).float()


def _finite_max(x, dims):
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x)).abs().amax(dims)


# ---- inputs -----------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    randn = lambda *shape: torch.randn(shape, generator=gen, device=dev)  # noqa: E731
    B, h_q, g, d_h, d_v, d_r, P = (c[k] for k in ("batch", "h_q", "g", "d_h", "d_v", "d_r", "page"))
    lens, new = _lengths(c)
    need = [-(-L // P) for L in lens]
    max_pages = max(1, max(need))
    pages = max(1, sum(need)) if c["paged"] else B * max_pages
    perm = torch.randperm(pages, generator=gen, device=dev).tolist() if c["paged"] else None
    rows, at = [], 0
    for b in range(B):                                    # entries behind a sequence's last page hold -1
        mine = perm[at:at + need[b]] if c["paged"] else [b * max_pages + p for p in range(need[b])]
        at += need[b]
        rows.append(mine + [-1] * (max_pages - need[b]))
    first = [0]
    for n in new:
        first.append(first[-1] + n)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    s = {"c": c, "lens": i32(lens), "table": i32(rows), "first": i32(first), "rows": first[-1], "pages": pages,
         "max_pages": max_pages, "n_max": max(new), "l_max": max(lens)}

    R = first[-1]
    if c["op"] in ("append", "append_blocks"):
        # a head's values have a size of their own, and every eighth channel or so stands out: what scales are for
        size = lambda *shape: torch.exp(0.7 * randn(*shape)) * torch.where(randn(*shape) > 1.2, 4.0, 1.0)  # noqa: E731
        parts = [(randn(R, g, d_h) * size(g, d_h)).reshape(R, -1), (randn(R, g, d_v) * size(g, 1)).reshape(R, -1), randn(R, d_r)]
        if c["fused"]:
            joint = torch.cat(parts, 1).to(dt).contiguous()
            s["k_c"], s["v"], s["k_r"] = joint.split([g * d_h, g * d_v, d_r], 1)
        else:
            s["k_c"], s["v"], s["k_r"] = (p.to(dt).contiguous() for p in parts)
        s["q_r"] = randn(R, h_q, d_r).to(dt)
        s["q_rot"] = torch.zeros_like(s["q_r"])
    if c["op"] in ("decode", "attend"):
        s["q_c"], s["q_r"] = randn(R, h_q, d_h).to(dt), randn(R, h_q, d_r).to(dt)
        s["out"] = torch.zeros((R, h_q, d_v), dtype=dt, device=dev)
        s["lse"] = torch.zeros((R, h_q), dtype=torch.float32, device=dev)
    if c["op"] in ("append", "quantize"):                 # every slot holds something, also those that no token owns
        s["wide"] = randn(pages, P * (g * (d_h + d_v) + d_r)).to(dt)
        if c["op"] == "quantize":
            k, v, _ = _plain_view(s["wide"], c)
            k.mul_(torch.exp(0.7 * randn(pages, g, d_h // 8, 1, 8)).to(dt))
            v.mul_(torch.exp(0.7 * randn(pages, g, P // 8, 1, 1)).to(dt))
    if c["op"] != "append":
        s["pool"] = torch.empty((pages, _block_bytes(c)), dtype=torch.uint8, device=dev)
        k8, v8, k_r, scales = _blocks_view(s["pool"], c)
        T = P // 32
        size = torch.exp(0.7 * randn(pages, g, T, 2)) * torch.where(randn(pages, g, T, 2) > 2.0, 8.0, 1.0)
        step = max(1, (1 << 28) // (P * g * (d_h + d_v)))  # a GiB of fp32 at a time
        for p in range(0, pages, step):
            n = min(step, pages - p)
            x = randn(n, g, d_h // 32 * 2, T, 512) * size[p:p + n, :, None, :, :1]
            y = randn(n, g, T, d_v * 32) * size[p:p + n, :, :, 1:]
            e = _exponent(torch.stack([x.abs().amax((2, 4)), y.abs().amax(3)], 3))
            scales[p:p + n] = _pow2(e)
            k8[p:p + n] = _code(x * _pow2(-e[:, :, None, :, :1])).view(n, g, d_h // 32, 2, P, 2, 8)
            v8[p:p + n] = _code(y * _pow2(-e[..., 1:])).view(n, g, T, d_v, 2, 2, 8)
        k_r.copy_(randn(pages, d_r // 8, P, 8))
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps beside its buffers: the library's structs, the split plan with its workspace."""
    from paper_2605_15250_amd import binding as B
    from paper_2605_15250_amd.harness import NUM_CUS
    c = s["c"]
    dtype = B.GQLA_F32 if c["dtype"] == "f32" else B.GQLA_BF16
    s_q = c["n_max"] if c["op"] == "decode" else 1
    s["shape"] = B.make_shape(c["batch"], c["h_q"], c["g"], c["d_h"], 512, c["d_r"], s_q, dtype, 0.0, c["d_v"])
    cache = lambda pool: B.make_cache(pool, s["lens"], s["table"], c["page"], s["max_pages"], s["pages"], c["g"])  # noqa: E731
    if "wide" in s:
        s["wide_cache"] = cache(s["wide"])
    if "pool" in s:
        s["cache"] = cache(s["pool"])
    if c["op"] in ("append", "append_blocks"):
        s["new"] = B.make_new_rows(s["k_c"], s["v"], s["k_r"], s["q_r"], s["q_rot"], s["first"], s["rows"],
                                   s["k_c"].stride(0), s["v"].stride(0), s["k_r"].stride(0))
    if c["op"] == "decode":
        plan = B.gqla_plan_create(s["shape"], s["lens"].cpu().numpy(), c["page"], NUM_CUS, B.GQLA_PATH_GQA)
        s["plan"] = _Plan(B, plan)
        s["ws"] = torch.empty(B.gqla_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
        B.gqla_plan_upload(plan, s["ws"])
    if c["op"] == "attend":
        need = B.gqla_attend_gqa_workspace_bytes(s["shape"], s["first"], s["rows"], s["cache"])
        s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")


class _Plan:
    def __init__(self, binding, handle):
        self.binding, self.handle = binding, handle

    def __del__(self):
        self.binding.gqla_plan_destroy(self.handle)


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(s):
    op = s["c"]["op"]
    if own:
        from paper_2605_15250_amd import binding as B
        if op == "append":
            B.gqla_append_expanded(s["shape"], s["new"], BASE, s["wide_cache"])
        elif op == "append_blocks":
            B.gqla_append_expanded_fp8_blocks(s["shape"], s["new"], BASE, s["cache"])
        elif op == "quantize":
            B.gqla_quantize_expanded_fp8_blocks(s["shape"], s["wide_cache"], s["cache"])
        elif op == "decode":
            B.gqla_decode_gqa_fp8_blocks(s["shape"], s["plan"].handle, s["q_c"], s["q_r"], s["cache"], s["out"], s["lse"], s["ws"])
        else:
            B.gqla_attend_gqa_fp8_blocks(s["shape"], s["first"], s["rows"], s["q_c"], s["q_r"], s["cache"], s["out"], s["lse"], s["ws"])
    else:
        {"append": _append, "append_blocks": _append_blocks, "quantize": _quantize, "decode": _attend, "attend": _attend}[op](s)
    if op in ("decode", "attend"):
        return {"out": s["out"], "lse": s["lse"]}
    if op == "append":
        return {"cache": s["wide"], "q": s["q_rot"]}
    k8, v8, k_r, scales = _blocks_view(s["pool"], s["c"])
    got = {"k": k8.view(torch.float8_e4m3fn), "v": v8.view(torch.float8_e4m3fn), "k_r": k_r, "scales": scales}
    if op == "append_blocks":
        got["q"] = s["q_rot"]
    return got


def _places(s):
    """Of each new row: its sequence, its position, and the page and slot it goes to."""
    P = s["c"]["page"]
    row = torch.arange(s["rows"], device=s["lens"].device)
    first = s["first"].long()
    b = torch.searchsorted(first, row, right=True) - 1
    t = s["lens"].long()[b] - first[b + 1] + row
    return b, t, s["table"].long()[b, t // P], t % P


def _rotate(x, t):
    """x [rows][..][d_r] turned at the rows' positions t: angles in 64 bits, the rest in 32."""
    d_r = x.shape[-1]
    pair = torch.arange(d_r // 2, device=x.device, dtype=torch.float64)
    angle = t.double()[:, None] * torch.pow(torch.tensor(BASE, dtype=torch.float64, device=x.device), -2 * pair / d_r)
    shape = [x.shape[0]] + [1] * (x.dim() - 2) + [d_r // 2]
    cs, sn = torch.cos(angle).float().view(shape), torch.sin(angle).float().view(shape)
    y = x.float()
    a, b = y[..., 0::2], y[..., 1::2]
    return torch.stack([a * cs - b * sn, a * sn + b * cs], -1).flatten(-2)


def _append(s):
    c = s["c"]
    g, d_h, d_v, d_r = (c[k] for k in ("g", "d_h", "d_v", "d_r"))
    k, v, k_r = _plain_view(s["wide"], c)
    _, t, page, slot = _places(s)
    R = s["rows"]
    k.permute(0, 3, 1, 2, 4)[page, slot] = s["k_c"].reshape(R, g, d_h // 8, 8)
    v.permute(0, 2, 4, 1, 3)[page, slot // 8, slot % 8] = s["v"].reshape(R, g, d_v)
    k_r.permute(0, 2, 1, 3)[page, slot] = _rotate(s["k_r"], t).view(R, d_r // 8, 8).to(k_r.dtype)
    s["q_rot"].copy_(_rotate(s["q_r"], t))


def _append_blocks(s):
    c = s["c"]
    P, g, d_h, d_v, d_r = (c[k] for k in ("page", "g", "d_h", "d_v", "d_r"))
    R, T = s["rows"], P // 32
    k8, v8, k_r, scales = _blocks_view(s["pool"], c)
    _, t, page, slot = _places(s)
    k, v = s["k_c"].reshape(R, g, d_h).float(), s["v"].reshape(R, g, d_v).float()
    # the blocks' new exponents
    amax = torch.zeros((s["pages"] * T, g, 2), device=k.device)
    block = page * T + slot // 32
    top = torch.stack([_finite_max(k, 2), _finite_max(v, 2)], 2)
    amax.scatter_reduce_(0, block[:, None, None].expand_as(top), top, "amax")
    amax = amax.view(s["pages"], T, g, 2)
    # blocks that hold older tokens: the one where a sequence's new rows begin
    first, lens = s["first"].long(), s["lens"].long()
    begin = lens - (first[1:] - first[:-1])
    some = ((begin % 32 != 0) & (first[1:] > first[:-1])).nonzero()[:, 0]
    begin = begin[some]
    pg, tl, old_slots = s["table"].long()[some, begin // P], begin % P // 32, begin % 32
    e_was = torch.frexp(scales.permute(0, 2, 1, 3)[pg, tl])[1] - 1
    e_now = _exponent(amax)
    e_old = torch.maximum(e_was, e_now[pg, tl])
    e_now[pg, tl] = e_old
    shrink = _pow2(e_was - e_old)
    lane = torch.arange(32, device=k.device)
    is_old = lane[None, :] < old_slots[:, None]
    kv = k8.view(-1, g, d_h // 32, 2, T, 32, 2, 8).permute(0, 4, 1, 2, 3, 5, 6, 7)
    x = kv[pg, tl]
    kv[pg, tl] = torch.where(is_old[:, None, None, None, :, None, None], _code(_value(x) * shrink[:, :, 0, None, None, None, None, None]), x)
    vv = v8.permute(0, 2, 1, 3, 5, 4, 6)                    # slots as (u, h, i)
    x = vv[pg, tl]
    vv[pg, tl] = torch.where(is_old.view(-1, 1, 1, 2, 2, 8), _code(_value(x) * shrink[:, :, 1, None, None, None, None]), x)
    # the new rows
    tile = slot // 32
    e_row = e_now[page, tile]
    scales.permute(0, 2, 1, 3)[page, tile] = _pow2(e_row)
    kc = _code(k * _pow2(-e_row[:, :, :1])).view(R, g, d_h // 32, 2, 2, 8)       # dims as (x, u, h, i)
    k8.permute(0, 4, 1, 2, 5, 3, 6)[page, slot] = kc
    vc = _code(v * _pow2(-e_row[:, :, 1:]))
    v8.permute(0, 2, 5, 4, 6, 1, 3)[page, tile, slot % 32 // 16, slot % 16 // 8, slot % 8] = vc
    k_r.permute(0, 2, 1, 3)[page, slot] = _rotate(s["k_r"], t).view(R, d_r // 8, 8).to(torch.bfloat16)
    s["q_rot"].copy_(_rotate(s["q_r"], t))


def _quantize(s):
    c = s["c"]
    P, g, d_h, d_v = (c[k] for k in ("page", "g", "d_h", "d_v"))
    T, N = P // 32, s["pages"]
    k16, v16, r16 = _plain_view(s["wide"], c)
    k8, v8, k_r, scales = _blocks_view(s["pool"], c)
    # tokens that a page holds
    count = torch.zeros(N, dtype=torch.long, device=k8.device)
    held = (s["lens"].long()[:, None] - P * torch.arange(s["max_pages"], device=k8.device)).clamp(0, P)
    table = s["table"].long()
    count.scatter_reduce_(0, table.clamp(min=0).reshape(-1), torch.where(table >= 0, held, 0).reshape(-1), "amax")
    live = torch.arange(P, device=k8.device) < count[:, None]
    k = k16.view(N, g, d_h // 32, 2, 2, T, 32, 8).permute(0, 1, 2, 4, 5, 6, 3, 7).float()   # (x, u, h, T, slot, i) -> (x, h, T, slot, u, i)
    v = v16.view(N, g, T, 2, 2, d_v, 8).permute(0, 1, 2, 5, 4, 3, 6).float()                # (T, u, h, d, i) -> (T, d, h, u, i)
    live_k = live.view(N, 1, 1, 1, T, 32, 1, 1)
    live_v = live.view(N, 1, T, 1, 2, 2, 8).transpose(4, 5)
    zero = torch.zeros((), device=k8.device)
    top = torch.stack([_finite_max(torch.where(live_k, k, zero), (2, 3, 5, 6, 7)), _finite_max(torch.where(live_v, v, zero), (3, 4, 5, 6))], 3)
    e = _exponent(top)
    some = live.view(N, 1, T, 32)[..., :1]
    scales.copy_(torch.where(some, _pow2(e), scales))
    kc = _code(k * _pow2(-e[:, :, None, None, :, 0, None, None, None]))
    k8.copy_(torch.where(live_k, kc, k8.view(N, g, d_h // 32, 2, T, 32, 2, 8)).reshape(k8.shape))
    v8.copy_(torch.where(live_v, _code(v * _pow2(-e[:, :, :, 1, None, None, None, None])), v8))
    k_r.copy_(torch.where(live[:, None, :, None], r16, k_r))


def _attend(s):
    c = s["c"]
    P, g, h_q, d_h, d_v, d_r = (c[k] for k in ("page", "g", "h_q", "d_h", "d_v", "d_r"))
    B, G, T, M, n_max = c["batch"], h_q // g, P // 32, s["max_pages"], s["n_max"]
    dev = s["lens"].device
    k8, v8, k_r, scales = _blocks_view(s["pool"], c)
    pages = s["table"].long().clamp(min=0)                                                  # [B][M]
    # keys [B][g][tokens][d_h + d_r] and values [B][g][tokens][d_v]
    k = _value(k8[pages].view(B, M, g, d_h // 32, 2, T, 32, 2, 8).permute(0, 2, 1, 5, 6, 3, 7, 4, 8).reshape(B, g, M, T, 32, d_h))
    sc = scales[pages].permute(0, 2, 1, 3, 4)                                               # [B][g][M][T][2]
    k = (k * sc[..., 0, None, None]).view(B, g, M * P, d_h)
    v = _value(v8[pages].permute(0, 2, 1, 3, 6, 5, 7, 4).reshape(B, g, M, T, 32, d_v))
    v = (v * sc[..., 1, None, None]).view(B, g, M * P, d_v)
    r = k_r[pages].permute(0, 1, 3, 2, 4).reshape(B, 1, M * P, d_r).float().expand(B, g, M * P, d_r)
    # queries, padded to the longest chunk: [B][n_max] rows
    first = s["first"].long()
    n = first[1:] - first[:-1]
    i = torch.arange(n_max, device=dev)
    row = (first[:-1, None] + i).clamp(max=s["rows"] - 1)
    here = i < n[:, None]
    q = torch.cat([s["q_c"], s["q_r"]], 2).float()[row].view(B, n_max, g, G, d_h + d_r).permute(0, 2, 1, 3, 4)
    q = q.reshape(B * g, n_max * G, d_h + d_r)
    keys = torch.cat([k, r], 3).view(B * g, M * P, d_h + d_r).transpose(1, 2).contiguous()
    logits = torch.bmm(q, keys).view(B, g, n_max, G, M * P).mul_(1.0 / math.sqrt(d_h + d_r))
    pos = s["lens"].long()[:, None] - n[:, None] + i                                        # [B][n_max]
    hidden = torch.arange(M * P, device=dev) > pos[:, :, None]
    logits.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    top = logits.amax(4, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = logits.sub_(top).exp_()
    den = p.sum(4, keepdim=True)
    o = torch.bmm(p.view(B * g, n_max * G, M * P), v.reshape(B * g, M * P, d_v)).view(B, g, n_max, G, d_v) / den
    lse = (torch.log(den) + top)[..., 0]
    s["out"][row[here]] = o.permute(0, 2, 1, 3, 4).reshape(B, n_max, h_q, d_v)[here].to(s["out"].dtype)
    s["lse"][row[here]] = lse.permute(0, 2, 1, 3).reshape(B, n_max, h_q)[here]


# ---- the definition in 64 bits, one sequence at a time -----------------------------------------------------------------
def _e4m3(q):
    """The values that E4M3 holds next to q (fp64), ties to even, beyond 448 the largest."""
    mag = q.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(mag.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(q) * (torch.round(mag / step) * step).clamp(max=448.0)


def _scale_of(amax):
    e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448.0))
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where((amax <= 448.0 * torch.exp2(e - 1)), e - 1, e)
    return torch.exp2(e.clamp(E_MIN, E_MAX))


def _offsets(c, slot):
    """Where an 8-bit page keeps the K codes [slot][g][d_h] and the V codes [slot][g][d_v]: byte offsets."""
    P, g, d_h, d_v = (c[k] for k in ("page", "g", "d_h", "d_v"))
    dev = slot.device
    j, d, dv = (torch.arange(n, device=dev) for n in (g, d_h, d_v))
    sl = slot[:, None, None]
    k = ((j[:, None] * (d_h // 16) + 2 * (d // 32) + d // 8 % 2) * P + sl) * 16 + 8 * (d // 16 % 2) + d % 8
    r = sl % 32
    v = g * P * d_h + (((j[:, None] * (P // 32) + sl // 32) * d_v + dv) * 2 + r // 8 % 2) * 16 + 8 * (r // 16) + r % 8
    return k, v


def _turned(x, t):
    d_r = x.shape[-1]
    z = torch.view_as_complex(x.double().reshape(*x.shape[:-1], d_r // 2, 2).contiguous())
    angle = t.double()[:, None] * BASE ** (-2.0 * torch.arange(d_r // 2, device=x.device).double() / d_r)
    return torch.view_as_real(z * torch.polar(torch.ones_like(angle), angle).view(len(t), *[1] * (x.dim() - 2), -1)).flatten(-2)


def _held(flat, at):
    return flat[at].view(torch.float8_e4m3fn).double()


def exact(case, seed):
    if work(case)["flops"] > 3e12:
        return None
    s = prepare(case, seed)
    c = s["c"]
    P, g, h_q, d_h, d_v, d_r, B = (c[k] for k in ("page", "g", "h_q", "d_h", "d_v", "d_r", "batch"))
    lens, new = _lengths(c)
    dev = s["lens"].device
    ar = lambda a, b: torch.arange(a, b, device=dev)  # noqa: E731
    first = s["first"].tolist()
    op = c["op"]
    if op == "append":
        pool = s["wide"].double()
        flat, size = pool.view(-1), pool.shape[1]
    else:
        size, flat = s["pool"].shape[1], s["pool"].view(-1)
        a, e = P * g * (d_h + d_v), P * (g * (d_h + d_v) + 2 * d_r)
        values = s["pool"][:, :a].view(torch.float8_e4m3fn).double() if op in ("append_blocks", "quantize") else None
        k_rope, scales = s["pool"][:, a:e].view(torch.bfloat16).double(), s["pool"][:, e:].view(torch.float32).double()
    out = torch.zeros((s["rows"], h_q, d_v), dtype=torch.float64, device=dev) if "out" in s else None
    lse = torch.zeros((s["rows"], h_q), dtype=torch.float64, device=dev) if "out" in s else None
    q_rot = torch.zeros((s["rows"], h_q, d_r), dtype=torch.float64, device=dev)
    for b in range(B):
        L, n, f = lens[b], new[b], first[b]
        t = ar(0, L)
        page, slot = s["table"][b].long()[t // P], t % P
        if op == "append":
            t, page, slot, rows = t[L - n:], page[L - n:], slot[L - n:], slice(f, f + n)
            j, d, dv, dr = ar(0, g)[:, None], ar(0, d_h), ar(0, d_v), ar(0, d_r)
            sl, base = slot[:, None, None], (page * size)[:, None, None]
            flat[base + ((j * (d_h // 8) + d // 8) * P + sl) * 8 + d % 8] = s["k_c"][rows].double().reshape(n, g, d_h)
            flat[base + g * P * d_h + ((j * (P // 8) + sl // 8) * d_v + dv) * 8 + sl % 8] = s["v"][rows].double().reshape(n, g, d_v)
            flat[base[:, 0] + g * P * (d_h + d_v) + (dr // 8 * P + slot[:, None]) * 8 + dr % 8] = _turned(s["k_r"][rows], t)
            q_rot[rows] = _turned(s["q_r"][rows], t)
            continue
        k_off, v_off = _offsets(c, slot)
        at = (page * size)[:, None, None]
        block = (slot // 32)[:, None] * 2 + ar(0, g) * (P // 32) * 2                    # [L][g]: place of K's scale
        if op in ("decode", "attend"):
            if not n:
                continue
            rows = slice(f, f + n)
            k = _held(flat, at + k_off) * scales[page[:, None], block][..., None]
            v = _held(flat, at + v_off) * scales[page[:, None], block + 1][..., None]
            r = k_rope.view(-1, d_r // 8, P, 8)[page, :, slot].reshape(L, d_r)
            for j in range(g):
                heads = slice(j * (h_q // g), (j + 1) * (h_q // g))
                x = torch.cat([s["q_c"][rows, heads], s["q_r"][rows, heads]], 2).double().view(-1, d_h + d_r)
                z = (x @ torch.cat([k[:, j], r], 1).t().contiguous()).view(n, h_q // g, L) / math.sqrt(d_h + d_r)
                z = z.masked_fill((t > L - n + ar(0, n)[:, None])[:, None, :], -math.inf)
                lse[rows, heads] = torch.logsumexp(z, 2)
                out[rows, heads] = (torch.softmax(z, 2).view(-1, L) @ v[:, j].contiguous()).view(n, h_q // g, d_v)
            continue
        lo = L - n if op == "append_blocks" else 0
        for b0 in range(lo // 32 * 32, L, 32 * 64):                                     # 64 blocks at a time
            x0, x1 = max(b0, lo), min(b0 + 32 * 64, L)
            if op == "append_blocks":
                k_new = s["k_c"][f + x0 - lo:f + x1 - lo].double().reshape(-1, g, d_h)
                v_new = s["v"][f + x0 - lo:f + x1 - lo].double().reshape(-1, g, d_v)
            else:
                wide, pg, sl = s["wide"].view(-1), page[x0:x1, None, None] * s["wide"].shape[1], slot[x0:x1, None, None]
                j, d, dv = ar(0, g)[:, None], ar(0, d_h), ar(0, d_v)
                k_new = wide[pg + ((j * (d_h // 8) + d // 8) * P + sl) * 8 + d % 8].double()
                v_new = wide[pg + g * P * d_h + ((j * (P // 8) + sl // 8) * d_v + dv) * 8 + sl % 8].double()
            for kind, (x, off) in enumerate(((k_new, k_off), (v_new, v_off))):
                top = torch.zeros((64, g), dtype=torch.float64, device=dev)
                which = (ar(x0, x1) - b0) // 32
                top.scatter_reduce_(0, which[:, None].expand(-1, g), x.abs().amax(2), "amax")
                scale = _scale_of(top)
                if x0 > b0:                                                             # older tokens in the first block
                    was = scales[page[b0], block[b0] + kind]
                    scale[0] = torch.maximum(scale[0], was)
                    old = slice(b0, x0)
                    place = page[old, None, None] * values.shape[1] + off[old]
                    values.view(-1)[place] = _e4m3(values.view(-1)[place] * (was / scale[0])[:, None])
                values.view(-1)[page[x0:x1, None, None] * values.shape[1] + off[x0:x1]] = _e4m3(x / scale[which][..., None])
                scales[page[x0:x1, None], block[x0:x1] + kind] = scale[which]
        rope = k_rope.view(-1, d_r // 8, P, 8)
        if op == "append_blocks":
            rows = slice(f, f + n)
            rope[page[lo:], :, slot[lo:]] = _turned(s["k_r"][rows], t[lo:]).view(n, d_r // 8, 8)
            q_rot[rows] = _turned(s["q_r"][rows], t[lo:])
        else:
            r16 = _plain_view(s["wide"], c)[2]
            rope[page, :, slot] = r16[page, :, slot].double()
    if op == "append":
        return {"cache": pool, "q": q_rot}
    if op in ("decode", "attend"):
        return {"out": out, "lse": lse}
    k_part = P * g * d_h
    got = {"k": values[:, :k_part].reshape(-1, g, d_h // 32, 2, P, 2, 8), "v": values[:, k_part:].reshape(-1, g, P // 32, d_v, 2, 2, 8),
           "k_r": k_rope.view(-1, d_r // 8, P, 8), "scales": scales.view(-1, g, P // 32, 2)}
    if op == "append_blocks":
        got["q"] = q_rot
    return got
