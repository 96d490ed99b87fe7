"""What a workspace holds before a call changes nothing: the operators for sequences of cached rows with workspaces of zeros and of
0xFF bytes (NaN as floats), above all attention over long lists that use little of their room, whose parts several workgroups share."""
import numpy as np
import pytest
import torch

import paper_2202_12429_amd as bp
import test_gpu_operators as ops
from test_gpu_operators import DEV, LOG, Batch, Lists, dev, within

pytestmark = pytest.mark.gpu
FILLS = (0xff, 0x00, 0x7f)


def filled(byte):
    return lambda n: torch.full((n,), byte, dtype=torch.uint8, device=DEV)


def grown(layout, stretches, used, **kw):
    """A batch whose lists use the first `used` entries of their stretches."""
    b = Batch(*layout, stretches, **kw)
    starts = np.concatenate([[0], np.cumsum(stretches)])[:-1]
    b.spans = b.ref.spans = [(int(s), int(s) + u) for s, u in zip(starts, used)]
    b.used = np.zeros(b.n, dtype=bool)
    for a, e in b.spans:
        b.used[a:e] = True
    b.ref.seen = b.ref.seen & b.used
    b.given["bag_lengths"] = dev(np.asarray(used, np.int32))
    return b


RAGGED = [int(x) for x in np.random.default_rng(5).integers(1, 2001, 10)]
#            stretches, used (None: all of them)
LISTS = {
    "unequal": ([1280, 128, 128], None),
    "five": ([768, 256, 1280, 1024, 512], None),
    "ragged": (RAGGED, None),
    "one, growing": ([8192], [300]),
    "one of 2,048": ([2048], [300]),
    "eight, growing": ([4096] * 8, [1000] * 8),
    "sixteen, short": ([8192] * 16, [200] * 16),
    "nearly empty": ([4096] * 4, [0, 1, 0, 130]),
    "empty": ([4096] * 3, [0, 0, 0]),
    "one full among empty": ([4096] * 5, [0, 0, 4096, 0, 0]),
}
LAYOUTS = [("f32", 2, 1, 16, False), ("bf16", 8, 2, 32, False), ("f32", 4, 4, 16, True), ("bf16", 16, 4, 64, False), ("bf16", 2, 1, 256, True)]


@pytest.mark.parametrize("lists", list(LISTS))
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda x: "-".join(map(str, x)))
def test_attention_over_lists_with_room(layout, lists, monkeypatch):
    stretches, used = LISTS[lists]
    if layout[3] > 64:
        stretches, used = stretches[:4], used and used[:4]
    b = Batch(*layout, stretches) if used is None else grown(layout, stretches, used)
    got = []
    for byte in FILLS:
        monkeypatch.setattr(ops, "scratch", filled(byte))
        b.check()
        out, lse, w = b.forward()
        got.append((out, lse, w, *b.forward(weights=False)[:2], *b.backward(out, lse)[:2]))
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert torch.equal(x, y)


def test_attention_over_a_list_that_grows(monkeypatch):
    """One workspace all along, as a program that generates keeps it: each length's result is what a fresh workspace gives."""
    b = grown(("bf16", 8, 2, 32, False), [4096, 4096], [4096, 4096])
    b.slots.clamp_(0, 900)
    kept = filled(0xff)(bp.bp_embbag_attn_fwd_workspace_bytes(b.cfg, b.at, b.n, b.bags, True))
    monkeypatch.setattr(ops, "scratch", filled(0))
    for n in (4096, 1, 127, 128, 129, 700, 2000, 0):
        b.given["bag_lengths"].copy_(torch.tensor([n, 4096 - n], dtype=torch.int32))
        for x, y in zip(b.forward(ws=kept), b.forward()):
            assert torch.equal(x, y), n


@pytest.mark.parametrize("lengths", ["short", "edges", "many"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda x: "-".join(map(str, x)))
def test_attention_with_bias(layout, lengths, monkeypatch):
    for byte in FILLS[:2]:
        monkeypatch.setattr(ops, "scratch", filled(byte))
        Batch(*layout, ops.LENGTHS[lengths], cap=4.0, bias=(LOG, True), room=True).check()


@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (2, 3, 65, 130), (1, 2, 700, 40)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_bias_gradient(shape, dtype):
    rp = bp.make_relpos(LOG, True)
    g = torch.randn(shape, device=DEV).to(dtype)
    got = []
    for byte in FILLS:
        out = torch.full((bp.relpos_rows(rp), shape[1]), 9.0, device=DEV)
        bp.bp_relpos_bias_bwd(rp, g, 3, out, filled(byte)(bp.bp_relpos_bias_bwd_workspace_bytes(rp, *shape)))
        got.append(out)
    within(got[0].sum(0), g.double().sum((0, 2, 3)).cpu().numpy(), g.double().abs().sum((0, 2, 3)).cpu().numpy() * 512 * 2.0 ** -24, "sum of the rows")
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("stretch,budget", [([50] * 40, 31), ([5000, 10, 4097], 4000), ([70_001, 3, 40_000], 8_193)])
def test_eviction(stretch, budget, monkeypatch):
    for byte in FILLS[:2]:
        monkeypatch.setattr(ops, "scratch", filled(byte))
        Lists(sum(stretch), stretch, budget, 2, 8, room=True).check()
