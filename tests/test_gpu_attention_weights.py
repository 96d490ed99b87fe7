"""Attention over bags where single weights decide: bags in which one entry weighs everything, NaN in them, and scores so far from
zero that the logarithm of a sum no longer holds the sum."""
import numpy as np
import pytest
import torch

import paper_2202_12429_amd as bp
from test_gpu_operators import DEV, HEADS, LOG, MANY, Batch, dev, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def one_seen(layout, lengths, **kw):
    """A batch whose bags each see one entry, somewhere among their others."""
    b = Batch(*layout, lengths, **kw)
    rng = np.random.default_rng(1)
    slots = np.full(b.n, -1, np.int32)
    for a, e in b.spans:
        if e > a:
            slots[rng.integers(a, e)] = rng.integers(0, 996)
    b.slots = dev(slots)
    if b.pos is not None:
        b.pos.zero_()
        b.q_pos.copy_(torch.arange(b.bags, device=DEV) % 50)
    return b, torch.from_numpy(np.nonzero(slots >= 0)[0]).to(DEV)


@pytest.mark.parametrize("lengths", [[1] * 9, [1, 3, 70, 0, 300], [3000, 1, 1500], MANY], ids=["ones", "mixed", "long", "many"])
@pytest.mark.parametrize("extra", [dict(), dict(cap=4.0, bias=(LOG, True))], ids=["plain", "cap and bias"])
@pytest.mark.parametrize("layout", HEADS, ids=lambda x: "-".join(map(str, x)))
def test_an_entry_alone_has_no_gradient_of_its_score(layout, extra, lengths):
    """Its weight is 1 whatever its score, so nothing reaches the query, its key or the bias: exactly, since a step of Adagrad would
    make a step of full size of the noise.  Its value has the gradient of the output, up to the weight's roundings."""
    b, at = one_seen(layout, lengths, **extra)
    out, lse, _ = b.forward()
    gq, gr, gb = b.backward(out, lse)
    w, v0 = b.at.kv_heads * b.at.head_dim, b.at.value_offset
    assert (gq == 0).all() and (gb is None or (gb == 0).all())
    assert v0 == 0 or (gr[at, :w] == 0).all()
    bag = torch.searchsorted(b.off, at, right=True) - 1
    go = dev(b.grad_out).double()[bag].view(len(at), b.at.kv_heads, -1, b.at.head_dim)
    # p = exp(score - lse): the score's products add up in another order than in the forward pass, each off by (d + 4) U of them
    q = b.q.double()[bag].view(go.shape)
    k = b.cache[b.slots[at].long(), :w].double().view(len(at), b.at.kv_heads, 1, -1)
    score = (q.abs() * k.abs()).sum(3) * b.at.scale
    off = 2 * (b.at.head_dim + 12) * U * score + 16 * U * (1 + lse.double()[bag].view(score.shape).abs())
    bound = (go.abs() * (off + (go.shape[2] + 8) * U)[..., None]).sum(2).view(len(at), w)
    within(gr[at, v0:v0 + w], go.sum(2).view(len(at), w).cpu().numpy(), bound.cpu().numpy(), "values")


@pytest.mark.parametrize("lengths", [[1] * 4, [1] * 4 + MANY], ids=["few", "many"])
@pytest.mark.parametrize("layout", HEADS, ids=lambda x: "-".join(map(str, x)))
def test_nan_in_an_entry_alone_goes_through(layout, lengths):
    b = Batch(*layout, lengths)
    group, d, v0 = b.at.q_heads // b.at.kv_heads, b.at.head_dim, b.at.value_offset
    b.cache[:4] = 1.0
    b.slots[:4] = torch.arange(4, dtype=torch.int32, device=DEV)
    b.slots[4:].clamp_(4, 900)
    b.cache[1, v0 + 3] = float("nan")                # a value (and, where keys are values, a key) of kv head 0
    b.grad_out[2, -1, d - 1] = float("nan")          # the last query head's
    out, lse, _ = b.forward()
    gq, gr, _ = b.backward(out, lse)
    assert gq[1, :group].isnan().all() and torch.isfinite(gq[1, group:]).all()
    assert gq[2, -1].isnan().all() and torch.isfinite(gq[2, :-1]).all()
    assert torch.isfinite(gq[0]).all() and torch.isfinite(gq[3]).all()
    assert gr[1, :d].isnan().all() and torch.isfinite(gr[1, d:v0 or None]).all()
    last = (b.at.kv_heads - 1) * d
    assert gr[2, last:last + d].isnan().all() and torch.isfinite(gr[0]).all() and torch.isfinite(gr[3]).all()


@pytest.mark.parametrize("score", [16.0, 100.0, 1000.0])
@pytest.mark.parametrize("layout", [("f32", 2, 1, 16, False), ("bf16", 2, 1, 32, False), ("f32", 1, 1, 128, False), ("bf16", 1, 1, 256, False)],
                         ids=lambda x: "-".join(map(str, x)))
def test_a_dominant_entry_keeps_its_gradient(layout, score):
    """Two entries whose scores are 11.7 apart (the lesser weighs 8e-6): their score gradients add up to zero."""
    b = Batch(*layout, [2, 2])
    d = b.at.head_dim
    b.at = bp.make_attn(b.at.q_heads, 1, d, d, scale=1.0)
    cache, q, go = np.zeros((997, 2 * d)), np.zeros(tuple(b.q.shape), np.float32), np.zeros(tuple(b.q.shape), np.float32)
    # keys 1 and 1 - x, x a power of two or a sum of two (exact in bf16), q = 11.7 / x: an offset of `score` through the second element
    cache[1, :2], cache[2, :2] = (1.0, 1.0), (0.5, 1.0)
    cache[1, d], cache[2, d] = 1.0, -1.0
    q[..., 0], q[..., 1], go[..., 0] = 23.4375, score - 23.4375, 1.0
    b.cache, b.q, b.grad_out = torch.from_numpy(cache).to(DEV, b.cache.dtype), dev(q), go
    b.slots = torch.tensor([1, 2, 2, 1], dtype=torch.int32, device=DEV)
    out, lse, _ = b.forward()
    gq, gr, _ = b.backward(out, lse)
    r = b.ref
    r.q, r.rows, r.seen, r.scale = q.astype(np.float64), cache[[1, 2, 2, 1]], np.ones(4, bool), 1.0
    (o, l, _), _ = r.forward()
    (want_q, want_r, _), _ = r.backward(o, l, go)
    # dz = p (dp - against): both are sums of one product of 1, so each is off by a few roundings of 1 at most; p by the score's
    # rounding, relative to its 1.6e-5 (score U 4 of it: nothing).  Five roundings of 1 times keys of 1 and of 0.5, q of `score`.
    for got, want, most in ((gq, want_q, 1.0), (gr[:, :d], want_r[:, :d], max(score, 23.5))):
        assert np.abs(got.double().cpu().numpy() - want).max() <= 5 * U * most + 8 * U * score * np.abs(want).max()
    assert (gq[..., 0].abs() > 5e-6).all() and (gq[..., 0] > 0).all()        # 8.1e-6 * 2 * 0.5
    assert (gr[[0, 3], 0] > 5e-6).all() and (gr[[1, 2], 0] < -5e-6).all()


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
        go = dev(b.grad_out).double()[1].view(hk, -1, d).sum(1).view(-1)
        assert ((gr[40:, v0:].double() - go / 6).abs() <= 64 * U * dev(b.grad_out).double().abs().sum((1,))[1].max()).all()
