"""The trainer's calls on a stream of the caller's: what they allocate and fill first is done on that stream."""
import numpy as np
import pytest
import torch

import paper_2202_12429_amd as bp
from paper_2202_12429_amd.runner import CachedEmbeddingTrainer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def trainer(n):
    cfg = bp.make_config(100, 90, 32, "f32", "sgd", lookahead=2, lr=0.1)
    W = torch.ones(100, 32, device=DEV)
    tr = CachedEmbeddingTrainer(cfg, W, None)
    tr.plan(torch.arange(n, device=DEV) % 50, np.array([0, n], dtype=np.int64))
    tr.maintain(0)
    return tr, W


@pytest.mark.parametrize("given", ["stream", "handle", "0", "none"])
def test_counters_are_cleared_on_the_stream_of_the_call(given, monkeypatch):
    """They have to be zero when the backward pass starts, so the fill goes in front of it."""
    import paper_2202_12429_amd.binding as binding
    side, seen = torch.cuda.Stream(), []
    make = binding.bwd_tickets
    monkeypatch.setattr(binding, "bwd_tickets", lambda *a, **k: seen.append(torch.cuda.current_stream().cuda_stream) or make(*a, **k))
    tr, W = trainer(60)
    kw = dict(stream=dict(stream=side), handle=dict(stream=side.cuda_stream), none={})
    kw["0"] = dict(stream=0)
    q, off = torch.zeros(20, 2, 16, device=DEV), torch.arange(0, 61, 3, device=DEV)
    at = bp.make_attn(2, 2, 16, 0)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.default_stream() if given in ("stream", "handle") else side):
        out, lse = tr.attend(0, at, off, 20, q, **kw[given])
        tr.attend_backward_update(0, at, off, 20, q, out, lse, torch.ones_like(q), **kw[given])
    torch.cuda.synchronize()
    assert seen == [torch.cuda.default_stream().cuda_stream if given == "0" else side.cuda_stream]
    tr.flush()
    # every bag pools three rows of ones: each gets a third of the gradient, ten of the rows are looked up twice
    want = torch.ones(100, device=DEV)
    want[:50] -= 0.1 / 3
    want[:10] -= 0.1 / 3
    assert (W - want[:, None]).abs().max() < 1e-6


@pytest.mark.parametrize("stream", ["side", "default"])
def test_on_a_stream(stream):
    tr, _ = trainer(3)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with tr._on(0 if stream == "default" else side.cuda_stream):
            assert torch.cuda.current_stream().cuda_stream == (torch.cuda.default_stream() if stream == "default" else side).cuda_stream
        assert torch.cuda.current_stream().cuda_stream == side.cuda_stream
