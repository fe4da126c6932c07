"""What the harness hands to the library for rows of new tokens and for the attention of prompt chunks, on the CPU: the entry points are
replaced by functions that read the memory they are given, as the kernels would."""
import ctypes

import numpy as np
import pytest
import torch

import synth_inputs as S
from paper_2605_15250_amd import harness as H

CFG = S.CONFIGS["C3"].with_(B=3)
G_D, D_R = CFG.g * CFG.d_h, CFG.d_r


def decoder():
    d = H.Decoder.__new__(H.Decoder)
    d.cfg, d.groups, d.num_pages, d.max_pages = CFG, CFG.g, 4, 4
    d.shape = d.shape_gqa = H.B.make_shape(CFG.B, CFG.h_q, CFG.g, CFG.d_h, CFG.r_kv, CFG.d_r, CFG.s_q, H.B.GQLA_BF16)
    d.d_lens = d.d_table = d.expanded_pool = d.expanded_blocks_pool = torch.zeros(16, dtype=torch.int32)
    return d


def read(address, rows, row, stride):
    """rows x row 16-bit words from an address on, as the library reads them"""
    stride = stride or row
    words = np.ctypeslib.as_array((ctypes.c_uint16 * ((rows - 1) * stride + row)).from_address(address))
    return np.stack([words[i * stride: i * stride + row] for i in range(rows)]).copy()


def words(t):
    return t.contiguous().view(torch.int16).numpy().view(np.uint16).reshape(t.shape[0], -1)


@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("layout", ["packed", "parts", "one_row_for_all", "dims_apart", "heads_apart"])
def test_appended_rows_arrive_as_the_tensors_say(monkeypatch, layout, blocks):
    """Rows that are parts of a joint buffer, a row expanded over all tokens (stride 0), dims or heads that do not follow each other."""
    n = 5
    new = lambda *s: torch.randn(s, generator=torch.Generator().manual_seed(sum(s))).to(torch.bfloat16)  # noqa: E731
    k, v, kr, q = new(n, G_D), new(n, G_D + 0), new(n, D_R), new(n, CFG.h_q, D_R)
    if layout == "parts":
        joint = new(n, 2 * G_D + D_R + 8)
        k, v, kr = joint[:, :G_D], joint[:, G_D:2 * G_D], joint[:, 2 * G_D:2 * G_D + D_R]
        q = new(n, CFG.h_q, CFG.d_h + D_R)[..., CFG.d_h:]
    elif layout == "one_row_for_all":
        k, v, kr = k[:1].expand(n, -1), v[:1].expand(n, -1), kr[:1].expand(n, -1)
        q = q[:1].expand(n, -1, -1)
    elif layout == "dims_apart":
        k, v, kr = new(G_D, n).t(), new(n, 2 * G_D)[:, ::2], new(D_R, n).t()
        q = new(n, D_R, CFG.h_q).transpose(1, 2)
    elif layout == "heads_apart":
        q = new(CFG.h_q, n, D_R).transpose(0, 1)
    seen = {}

    def call(shape, rows, base, cache):
        assert rows.total == n
        for x, at, stride in ((k, rows.k_c, rows.k_stride), (v, rows.v, rows.v_stride), (kr, rows.k_r, rows.kr_stride)):
            assert np.array_equal(read(at, n, x.shape[1], stride), words(x))
        got = read(rows.q_r, n, CFG.h_q * D_R, 0)
        assert np.array_equal(got, words(q))
        ctypes.memmove(rows.q_rot, got.ctypes.data, got.nbytes)     # "rotated" by nothing
        seen["called"] = True
    monkeypatch.setattr(H.B, "gqla_append_expanded_fp8_blocks" if blocks else "gqla_append_expanded", call)
    q_rot = decoder().append_expanded(1e4, k, v, kr, q, blocks=blocks)
    assert seen and q_rot.is_contiguous() and torch.equal(q_rot, q)


def test_parts_of_a_joint_buffer_are_not_copied(monkeypatch):
    joint = torch.zeros((4, 2 * G_D + D_R + 8), dtype=torch.bfloat16)
    parts = joint[:, :G_D], joint[:, G_D:2 * G_D], joint[:, 2 * G_D:2 * G_D + D_R]
    monkeypatch.setattr(H.B, "gqla_append_expanded", lambda shape, rows, base, cache: seen.append(rows))
    seen = []
    decoder().append_expanded(1e4, *parts)
    assert [seen[0].k_c, seen[0].v, seen[0].k_r] == [x.data_ptr() for x in parts]
    assert seen[0].k_stride == seen[0].v_stride == seen[0].kr_stride == joint.stride(0)


def test_every_attention_call_has_a_workspace_of_its_own(monkeypatch):
    """A recorded call goes on using its workspace, and calls on two streams overlap: none is shared, and none kept and freed for a larger one."""
    sizes, taken = iter([4096, 0, 4096, 8192]), []
    empty = torch.empty
    monkeypatch.setattr(H.torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw))
    monkeypatch.setattr(H.B, "gqla_attend_gqa_workspace_bytes", lambda *a: next(sizes))
    monkeypatch.setattr(H.B, "gqla_attend_gqa_fp8_blocks", lambda *a: taken.append(a[-1]))
    d = decoder()
    for _ in range(4):
        d.attend_gqa_blocks(torch.zeros((2, CFG.h_q, CFG.d_h), dtype=torch.bfloat16), torch.zeros((2, CFG.h_q, D_R), dtype=torch.bfloat16))
    assert [0 if w is None else w.numel() for w in taken] == [4096, 0, 4096, 8192]
    assert len({w.data_ptr() for w in taken if w is not None}) == 3
    assert not any(torch.is_tensor(x) and x.dtype == torch.uint8 for x in vars(d).values())
