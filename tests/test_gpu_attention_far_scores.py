"""Attention over bags with scores so far from zero that the logarithm of a sum no longer holds the sum."""
import numpy as np
import pytest
import torch

from test_gpu_operators import DEV, HEADS, MANY, Batch, dev, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("lengths", [[3, 1, 0, 40], [700, 5], [3000, 1, 1025], MANY], ids=["short", "middle", "long", "many"])
@pytest.mark.parametrize("layout", [x for x in HEADS if x[0] == "f32"][:4] + [x for x in HEADS if x[0] == "bf16"][:4], ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("low", [torch.finfo(torch.float32).min, -1e30, -1e9])
def test_bags_that_a_mask_of_low_values_covers_whole(layout, lengths, low):
    """A table entry so low that it swallows the score (|score| < 32 is below half a unit of 1e9) masks its keys where others are
    left; where none is left all weigh the same, 1 / n, and together 1: in the output, the weights and the gradients."""
    b = Batch(*layout, lengths, bias=([10], True))
    b.slots.clamp_(0, 995)
    hq, hk, d, v0 = b.at.q_heads, b.at.kv_heads, b.at.head_dim, b.at.value_offset
    b.q_pos.fill_(100)
    b.pos.fill_(0)                                       # far: table row 1
    b.table[1] = low
    b.q.mul_(0.1)
    out, lse, w = b.forward()
    gq, gr, gb = b.backward(out, lse)
    count = torch.tensor(lengths, device=DEV)
    bag = torch.repeat_interleave(torch.arange(b.bags, device=DEV), count)
    p = (1.0 / count.double())[bag]
    start = dev(b.weight).double()
    n = max(lengths)
    # equal weights: their sum of n, a quotient and two or three functions' units
    rel = (n + 16) * U
    within(w, (start + hq * p).cpu().numpy(), ((hq * p) * (rel + hq * U) + U * (start + hq * p)).cpu().numpy(), "weights")
    go = dev(b.grad_out).double()[bag].view(b.n, hk, -1, d)
    v = b.cache[b.slots.long(), v0:v0 + hk * d].double()
    want = (p[:, None, None] * go.sum(2)).view(b.n, -1)
    bound = (p[:, None, None] * go.abs().sum(2)).view(b.n, -1) * (rel + 16 * U)
    if v0:
        within(gr[:, v0:v0 + hk * d], want.cpu().numpy(), bound.cpu().numpy(), "gradient of the values")
    mean = torch.zeros(b.bags, hk * d, dtype=torch.float64, device=DEV).index_add_(0, bag, v * p[:, None])
    size = torch.zeros(b.bags, hk * d, dtype=torch.float64, device=DEV).index_add_(0, bag, v.abs() * p[:, None])
    to_q = lambda x: x.view(b.bags, hk, 1, d).expand(-1, -1, hq // hk, -1).reshape(b.bags, hq, d)
    within(out, to_q(mean).cpu().numpy(), to_q(size * rel + 1e-37).cpu().numpy(), "out")
    # of the bias: weights times what differs from the mean, summed: zero, up to the roundings of its terms
    dots = (go * v.view(b.n, hk, 1, d)).abs().sum(3).view(b.n, hq) * p[:, None]
    of = (dev(b.grad_out).double() * to_q(size)).abs().sum((0, 2)) + dots.sum(0)
    assert (gb[0] == 0).all() and (gb[1].double().abs() <= 4 * of * (rel + (d + 4 + n) * U)).all()
    # one key of another row: the others weigh nothing
    b.pos[0] = 95
    if lengths[0] > 1:
        out, lse, w = b.forward()
        gq, gr, gb = b.backward(out, lse)
        assert torch.equal(w[1:lengths[0]], dev(b.weight)[1:lengths[0]]) and (gr[1:lengths[0]] == 0).all()


@pytest.mark.parametrize("layout", [("f32", 4, 4, 16, True), ("bf16", 8, 2, 32, False)], ids=["narrow", "grouped"])
def test_scores_far_from_zero_without_a_mask(layout):
    """Scores of some 100,000, which differ by hundreds: one entry weighs everything, or exactly equal ones share."""
    b = Batch(*layout, [40, 6])
    b.slots.copy_(torch.arange(46, dtype=torch.int32, device=DEV))
    b.slots[40:] = 7
    b.q.mul_(1e5)
    out, lse, w = b.forward()
    gq, gr, _ = b.backward(out, lse)
    hq, hk, d, v0 = b.at.q_heads, b.at.kv_heads, b.at.head_dim, b.at.value_offset
    got = (w - dev(b.weight)).double()
    assert abs(got[:40].sum().item() - hq) < 1e-3 and abs(got[40:].sum().item() - hq) < 1e-3
    if v0:
        # a score is off by (d + 4) U of its products, and lse by U of itself: a weight of 1 / 6 by that factor (exp of 4 of these)
        go = dev(b.grad_out).double()[1].view(hk, -1, d)
        size = (b.q[1].double().abs().view(hk, -1, d) * b.cache[7, :hk * d].double().abs().view(hk, 1, d)).sum(2) * b.at.scale
        rel = torch.expm1(4 * ((d + 4) * U * size + U * lse[1].double().abs().view(hk, -1))) + 64 * U
        assert ((gr[40:, v0:].double() - (go.sum(1) / 6).view(-1)).abs() <= ((go.abs() * rel[..., None]).sum(1) / 6).view(-1)).all()
