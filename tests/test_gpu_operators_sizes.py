"""The operators for sequences of cached rows at the largest sizes they accept."""
import pytest
import torch

import paper_2202_12429_amd as bp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("lists", [1, 131_100], ids=["by pieces", "whole"])
def test_eviction_from_a_list_of_all_there_may_be(lists):
    """A list that ends at 2^31 - 1: its last steps of 64 places go past what 31 bits hold."""
    n, gone = (1 << 31) - 1, 100
    off = torch.full((lists + 1,), n, dtype=torch.int64, device=DEV)
    off[:lists] = 0                                          # the last list holds everything
    places = torch.cat([torch.arange(0, 50), torch.arange(50) * 7 + n - 350]).tolist()
    weight = torch.ones(n, device=DEV)
    weight[torch.tensor(places, device=DEV)] = -torch.arange(1.0, gone + 1, device=DEV)
    slots = torch.arange(n, dtype=torch.int32, device=DEV)
    kept = torch.full((n,), 77, dtype=torch.int32, device=DEV)
    i32 = lambda k: torch.full((k,), 77, dtype=torch.int32, device=DEV)
    lens, out, ends = i32(lists), i32(gone + 5), torch.full((lists + 1,), 77, dtype=torch.int64, device=DEV)
    ws = torch.full((bp.bp_evict_by_weight_workspace_bytes(n, lists),), 0xff, dtype=torch.uint8, device=DEV)
    bp.bp_evict_by_weight(off, None, lists, n - gone, 0, 0, weight, None, slots, None, None, kept, None, None, lens, None, out, ends, ws)
    assert out.tolist() == places + [-1] * 5
    assert ends[-1].item() == gone and (ends[:-1] == 0).all() and lens[-1].item() == n - gone and (lens[:-1] == 0).all()
    for i, (a, e) in enumerate(zip([-1] + places, places + [n])):          # what stays between two that left moves up by i places
        assert torch.equal(kept[a + 1 - i:e - i], slots[a + 1:e]), i
    assert (kept[n - gone:] == 77).all()


@pytest.mark.parametrize("dim", [8, 16], ids=["matrix instructions", "without"])
def test_gradient_of_the_bias_over_a_long_list(dim):
    """All entries of a list of 2^28 in one bucket, with equal terms: the table's gradient is their number times the term, up to fp32
    sums of 1,024 terms at most (each addition off by half a unit of its sum: 1,024 U of all of it; U for the last rounding)."""
    n, one = 1 << 28, torch.zeros(1, 1, dim, device=DEV)
    cfg, at, rp = bp.make_config(4, 4, dim), bp.make_attn(1, 1, dim, 0), bp.make_relpos([])
    cache, table, lse, go = torch.ones(4, dim, device=DEV), torch.zeros(1, 1, device=DEV), torch.full((1, 1), 1 / 3, device=DEV), torch.full_like(one, 1 / dim)
    pos, slots, rows = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV), torch.empty(n, dim, device=DEV)

    def gradient(k):
        gb = torch.empty(1, 1, device=DEV)
        ws = torch.empty(bp.bp_embbag_attn_bwd_workspace_bytes(cfg, at, rp, k, 1), dtype=torch.uint8, device=DEV)
        bp.bp_embbag_attn_bwd(cfg, at, cache, slots[:k], torch.tensor([0, k], device=DEV), 1, one, one, lse, go, torch.empty_like(one), rows[:k], gb, ws,
                              relpos=rp, q_pos=pos[:1], lookup_pos=pos[:k], bias_table=table)
        return gb.item()

    term = gradient(1)                                       # exp(-1/3)
    assert abs(term - 0.716531) < 1e-5
    assert abs(gradient(n) / n - term) <= 1025 * 2.0 ** -24 * term


def test_bias_of_more_rows_than_one_dimension_of_a_launch_holds():
    """A column of 2^30 - 1 queries is 2^25 workgroups of 256 threads."""
    lq, far = (1 << 30) - 1, 1 << 29
    rp, table = bp.make_relpos([far]), torch.tensor([[1.0], [2.0]], device=DEV)
    out = torch.full((1, lq, 1), 7.0, dtype=torch.bfloat16, device=DEV)
    bp.bp_relpos_bias_fwd(rp, table, 0, out)
    assert (out[0, :far] == 1).all() and (out[0, far:] == 2).all()


def test_attention_over_more_bags_than_one_dimension_of_a_launch_holds():
    """More than 2^24 bags of 64 entries, with weights: 2^24 and more workgroups of 256 threads in two launches."""
    bags, each, d = (1 << 24) + 3, 64, 8
    n = bags * each
    cfg, at = bp.make_config(1000, 1000, d), bp.make_attn(1, 1, d, 0)
    cache, q = torch.randn(1000, d, device=DEV), torch.randn(bags, 1, d, device=DEV)
    slots = (torch.arange(n, dtype=torch.int32, device=DEV) % 997)
    off = torch.arange(bags + 1, dtype=torch.int64, device=DEV) * each
    out, lse, w = torch.full_like(q, float("nan")), torch.full((bags, 1), float("nan"), device=DEV), torch.full((n,), float("nan"), device=DEV)
    ws = torch.full((bp.bp_embbag_attn_fwd_workspace_bytes(cfg, at, n, bags, True),), 0xff, dtype=torch.uint8, device=DEV)
    bp.bp_embbag_attn_fwd(cfg, at, cache, slots, off, bags, q, out, lse, ws, weight_out=w)
    for a in (0, bags // 2, 1 << 22, (1 << 23) - 50, 1 << 23, bags - 1000):
        e = min(a + 1000, bags)
        k = cache[slots[a * each:e * each].long()].view(-1, each, d).double()
        c = (k * q[a:e].double()).sum(2) * at.scale
        p = c.softmax(1)
        # scores of about 10 terms, sums of 64: a hundred roundings of values below 10 at most
        assert (out[a:e, 0].double() - (p[..., None] * k).sum(1)).abs().max() <= 100 * 10 * 2.0 ** -24
        assert (lse[a:e, 0].double() - c.logsumexp(1)).abs().max() <= 100 * 10 * 2.0 ** -24
        assert (w[a * each:e * each].double().view(-1, each) - p).abs().max() <= 100 * 10 * 2.0 ** -24
    assert not out.isnan().any() and not lse.isnan().any() and not w.isnan().any()


@pytest.mark.parametrize("batch,heads", [(1, 65_535), (65_535, 1), (300, 300)])
def test_bias_of_the_most_heads_and_batches(batch, heads):
    rp, lq, lk = bp.make_relpos([1, 2], True), 3, 5
    table, out = torch.randn(6, heads, device=DEV), torch.empty(heads, lq, lk, device=DEV)
    bp.bp_relpos_bias_fwd(rp, table, 1, out)
    distance = 1 + torch.arange(lq, device=DEV)[:, None] - torch.arange(lk, device=DEV)
    row = torch.where(distance < 0, 3, 0) + distance.abs().clamp(max=2)
    assert torch.equal(out, table.t()[:, row])
    g = torch.randint(-8, 9, (batch, heads, lq, lk), device=DEV).float()                 # whole numbers: exact sums
    got = torch.empty_like(table)
    ws = torch.full((bp.bp_relpos_bias_bwd_workspace_bytes(rp, batch, heads, lq, lk),), 0xff, dtype=torch.uint8, device=DEV)
    bp.bp_relpos_bias_bwd(rp, g, 1, got, ws)
    want = torch.stack([g[:, :, row == r].sum((0, 2)) for r in range(6)])
    assert torch.equal(got, want)
