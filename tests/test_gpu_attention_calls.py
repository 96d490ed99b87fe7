"""Attention over bags as programs call it: long lists that grow between the replays of a graph, two calls at once, and the most heads
there may be."""
import numpy as np
import pytest
import torch

import paper_2202_12429_amd as bp
import test_gpu_operators as ops
from test_gpu_operators import DEV, LOG, Batch, dev
from test_gpu_workspaces import filled, grown

pytestmark = pytest.mark.gpu


def sizes(b):
    return (bp.bp_embbag_attn_fwd_workspace_bytes(b.cfg, b.at, b.n, b.bags, True),
            bp.bp_embbag_attn_bwd_workspace_bytes(b.cfg, b.at, b.rp, b.n, b.bags))


@pytest.mark.parametrize("layout", [("bf16", 8, 2, 32, False), ("f32", 4, 4, 16, True)], ids=["grouped", "narrow"])
def test_lists_that_grow_between_replays(layout):
    b = grown(layout, [4096] * 3, [1, 0, 4096], bias=(LOG, False))
    b.slots.clamp_(0, 900)
    fw, bw = (filled(0xff)(n) for n in sizes(b))
    out, lse, w = torch.empty_like(b.q), torch.empty(b.q.shape[:2], device=DEV), torch.zeros(b.n, device=DEV)
    gq, gr, gb, go = torch.empty_like(b.q), torch.zeros(b.n, b.dim, device=DEV), torch.empty_like(b.table), dev(b.grad_out)

    def work(stream):
        bp.bp_embbag_attn_fwd(b.cfg, b.at, b.cache, b.slots, b.off, b.bags, b.q, out, lse, fw, stream=stream, weight_out=w, **b.given)
        bp.bp_embbag_attn_bwd(b.cfg, b.at, b.cache, b.slots, b.off, b.bags, b.q, out, lse, go, gq, gr, gb, bw, stream=stream, **b.given)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(torch.cuda.current_stream().cuda_stream)
    for step, lengths in enumerate(([1, 0, 4096], [300, 2000, 129], [0, 0, 0], [128, 129, 4095], [4096, 4096, 4096])):
        b.given["bag_lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        b.q_pos.copy_(torch.tensor(lengths, dtype=torch.int32))
        w.zero_(), gr.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, w, gq, gr, gb)]
        w.zero_(), gr.zero_()
        work(None)
        torch.cuda.synchronize()
        for x, y in zip(got, (out, lse, w, gq, gr, gb)):
            assert torch.equal(x, y), (step, lengths)


def test_two_calls_at_once():
    """Two streams, each with a workspace of its own, against one after the other."""
    batches = [Batch("bf16", 16, 4, 64, False, [3000, 1, 1025, 2000], bias=(LOG, True), seed=s) for s in (1, 2)]

    def both(streams):
        got = []
        for b, s in zip(batches, streams):
            with torch.cuda.stream(s):
                o, l, w = b.forward()
                got.append((o, l, w, *b.backward(o, l)))
        return got

    torch.cuda.synchronize()
    want = both([torch.cuda.default_stream()] * 2)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = both(streams)
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


@pytest.mark.parametrize("layout", [("bf16", 1024, 64, 8, True), ("bf16", 512, 32, 8, False), ("f32", 512, 32, 8, True), ("bf16", 64, 64, 8, True),
                                    ("f32", 16, 16, 16, True), ("bf16", 32, 32, 16, True)], ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("lengths", [[1, 0, 33, 300], [2100]], ids=["short", "long"])
def test_the_most_heads(layout, lengths, monkeypatch):
    monkeypatch.setattr(ops, "scratch", filled(0xff))
    Batch(*layout, lengths, cap=3.0, bias=(list(range(1, 64)), True), room=True).check()


def test_a_cache_of_one_row():
    b = Batch("f32", 4, 2, 16, False, [5, 0, 200])
    cfg = bp.make_config(1, 1, b.dim)
    b.cfg, b.cache = cfg, b.cache[:1].contiguous()
    b.slots.copy_(torch.where(torch.arange(b.n, device=DEV) % 3 == 0, 0, 1))             # 1: outside
    out, lse, w = b.forward()
    v = b.cache[0, 32:].view(2, 1, 16).expand(2, 2, 16).reshape(4, 16)
    assert (out[0] - v).abs().max() < 1e-6 and (out[2] - v).abs().max() < 1e-6 and (out[1] == 0).all()
    k = (torch.arange(5) % 3 == 0).sum().item()
    assert (w[:5][torch.arange(5) % 3 == 0] - dev(b.weight)[:5][torch.arange(5) % 3 == 0] - 4 / k).abs().max() < 1e-5
