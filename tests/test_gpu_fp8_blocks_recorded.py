"""Attention of prompt chunks through the harness, recorded twice: each graph keeps a workspace of its own, whatever runs between replays."""
import pytest
import torch

import synth_inputs as S
from paper_2605_15250_amd import binding as B
from test_gpu_parity import Case

pytestmark = pytest.mark.gpu


def test_two_graphs_and_a_larger_call_between_their_replays():
    cfg = S.CONFIGS["C3"].with_(B=1, L=0, s_q=1, paged=True, seed=992)
    case = Case(cfg, lens=[3000])
    dec = case.dec
    try:
        gen = torch.Generator(device="cuda").manual_seed(5)
        new = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
        first = torch.zeros(2, dtype=torch.int32, device="cuda")
        dec.alloc_expanded_blocks()
        first[1] = 3000
        dec.append_expanded(1e4, new(3000, cfg.g * cfg.d_h), new(3000, cfg.g * cfg.d_h), new(3000, cfg.d_r), first=first, blocks=True)
        jobs = []
        for n in (3, 5):
            f = torch.tensor([0, n], dtype=torch.int32, device="cuda")
            q_c, q_r = new(n, cfg.h_q, cfg.d_h), new(n, cfg.h_q, cfg.d_r)
            assert B.gqla_attend_gqa_workspace_bytes(dec.shape_gqa, f, n, dec.expanded_blocks_cache()) > 0
            want = [x.clone() for x in dec.attend_gqa_blocks(q_c, q_r, f)]
            out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                dec.attend_gqa_blocks(q_c, q_r, f, out, lse)
            jobs.append((graph, out, lse, want, (f, q_c, q_r)))
        f = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
        q_c, q_r = new(40, cfg.h_q, cfg.d_h), new(40, cfg.h_q, cfg.d_r)
        for _ in range(3):
            big = dec.attend_gqa_blocks(q_c, q_r, f)
            later = [torch.full((1 << 18,), 7.0, device="cuda") for _ in range(64)]   # takes the place of whatever was freed
            for graph, out, lse, _, _ in jobs:
                out.fill_(0.0), lse.fill_(0.0)
                graph.replay()
            torch.cuda.synchronize()
            assert all(bool((x == 7.0).all()) for x in later)
            for _, out, lse, want, _ in jobs:
                assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            again = dec.attend_gqa_blocks(q_c, q_r, f)
            torch.cuda.synchronize()
            assert torch.equal(again[0], big[0]) and torch.equal(again[1], big[1])
    finally:
        case.close()
