"""The 64-bit forms that the GPU tests compare with, against torch's autograd in float64 and against differences; the
refusals of the operators' entry points, which need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

import operators_reference as ref
import paper_2202_12429_amd as bp


@pytest.mark.parametrize("shared,cap,bias", [(False, 0.0, False), (False, 3.0, True), (True, 0.0, True), (True, 2.0, False)])
def test_attention_reference_against_autograd(shared, cap, bias):
    rng = np.random.default_rng(5)
    bags, hq, hk, d, n = 3, 4, 2, 8, 17
    w = hk * d
    value_at, dim = (0, w) if shared else (w, 2 * w)
    q, rows = rng.normal(size=(bags, hq, d)), rng.normal(size=(n, dim))
    spans, seen = [(0, 9), (9, 9), (9, 17)], rng.random(n) < 0.8
    table, table_row = (rng.normal(size=(5, hq)), rng.integers(0, 5, n)) if bias else (None, None)
    att = ref.Attention(q, rows, seen, spans, hk, value_at, d ** -0.5, cap, table, table_row)
    (out, lse, weight), _ = att.forward()
    go = rng.normal(size=out.shape)
    got, _ = att.backward(out, lse, go)
    t = [torch.tensor(x, requires_grad=True) for x in (q, rows)] + ([torch.tensor(table, requires_grad=True)] if bias else [])
    total = torch.zeros((), dtype=torch.float64)
    for b, (a, e) in enumerate(spans):
        pick = [k for k in range(a, e) if seen[k]]
        if not pick:
            assert np.all(out[b] == 0) and np.all(np.isneginf(lse[b]))
            continue
        for h in range(hq):
            kv = h // (hq // hk)
            c = (t[1][pick, kv * d:(kv + 1) * d] @ t[0][b, h]) * d ** -0.5
            if cap:
                c = cap * torch.tanh(c / cap)
            if bias:
                c = c + t[2][table_row[pick], h]
            o = torch.softmax(c, 0) @ t[1][pick, value_at + kv * d:value_at + (kv + 1) * d]
            assert np.allclose(o.detach().numpy(), out[b, h], rtol=1e-12, atol=1e-12)
            assert abs(torch.logsumexp(c, 0).item() - lse[b, h]) < 1e-12
            total = total + (o * torch.tensor(go[b, h])).sum()
    total.backward()
    for x, g in zip(t, got):
        assert np.allclose(x.grad.numpy(), g, rtol=1e-10, atol=1e-12)
    assert np.isclose(weight.sum(), hq * 2)


def test_bias_reference_is_linear_in_its_table():
    rng = np.random.default_rng(1)
    borders = [1, 2, 5, 9]
    table, step = rng.normal(size=(10, 3)), rng.normal(size=(10, 3))
    a, rows = ref.bias_grid(table, borders, True, 7, 11, 3)
    b, _ = ref.bias_grid(table + step, borders, True, 7, 11, 3)
    g = rng.normal(size=(2, 3, 7, 11))
    grad, _ = ref.bias_grad(g, rows, 10)
    assert np.isclose(((b - a)[None] * g).sum(), (grad * step).sum())


@pytest.mark.parametrize("buckets,far", [(1, 5), (2, 1), (5, 20), (32, 128), (16, 300), (64, 65_536), (64, (1 << 24) - 1)])
def test_borders(buckets, far):
    got = bp.bp_relpos_borders(buckets, far).tolist()
    e = max(1, buckets // 2)
    k, to, want = buckets - e, max(far, e + 1), list(range(1, e))
    for t in range(k):                                  # the smallest n with (n / e)^k >= (to / e)^t, by trying
        n = 1 if not want else want[-1] + 1
        guess = int(e * (to / e) ** (t / k)) - 2
        n = max(n, guess)
        while n > (want[-1] + 1 if want else 1) and (n - 1) ** k * e ** t >= to ** t * e ** k:
            n -= 1
        while n ** k * e ** t < to ** t * e ** k:
            n += 1
        want.append(n)
    assert got == want and len(got) == buckets - 1


def refused(status, call, *args, **kw):
    with pytest.raises(bp.BagpipeError) as e:
        call(*args, **kw)
    assert e.value.status == status, str(e.value)


def test_refusals_of_the_bias():
    rp = bp.make_relpos([1, 2, 4], True)
    for bad in ([0], [2, 2], [3, 1], [1 << 30]):
        refused(-1, bp.bp_relpos_bias_bwd_workspace_bytes, bp.make_relpos(bad), 1, 1, 4, 4)
    refused(-1, bp.bp_relpos_bias_bwd_workspace_bytes, bp.make_relpos(range(1, 65)), 1, 1, 4, 4)
    refused(-6, bp.bp_relpos_bias_bwd_workspace_bytes, rp, 1, 70_000, 4, 4)
    refused(-6, bp.bp_relpos_bias_bwd_workspace_bytes, rp, 1, 64, 1 << 20, 1 << 20)
    refused(-1, bp.bp_relpos_bias_bwd_workspace_bytes, rp, 1, 2, -1, 4)
    refused(-1, bp.bp_relpos_borders, 65, 100)
    refused(-1, bp.bp_relpos_borders, 8, 0)
    refused(-1, bp.bp_relpos_borders, 8, 1 << 24)
    table, out = torch.zeros(8, 2), torch.zeros(2, 3, 5)
    lib = bp.load_library()
    p = ctypes.byref(rp)
    t, o = table.data_ptr(), out.data_ptr()
    for args in ((p, None, 2, 3, 5, 0, o, 0, 0, 0, None), (p, t, 2, 3, 5, 0, None, 0, 0, 0, None), (p, t, 2, 3, 5, 0, o, 7, 0, 0, None),
                 (p, t, 2, 3, 5, 0, o, 0, 4, 0, None), (p, t, 2, 3, 5, 0, o, 0, 5, 14, None), (p, t, 2, 3, 5, 1 << 30, o, 0, 0, 0, None),
                 (p, t, 2, 3, 5, 0, o + 1, 0, 0, 0, None), (p, t, -2, 3, 5, 0, o, 0, 0, 0, None), (None, t, 2, 3, 5, 0, o, 0, 0, 0, None)):
        assert lib.bp_relpos_bias_fwd(*args) == -1
    assert lib.bp_relpos_bias_fwd(p, t, 2, 0, 5, 0, o, 0, 0, 0, None) == 0             # nothing to write
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    at = -ws.data_ptr() % 256
    need = bp.bp_relpos_bias_bwd_workspace_bytes(rp, 1, 2, 3, 5)
    g = torch.zeros(1, 2, 3, 5)
    refused(-3, bp.bp_relpos_bias_bwd, rp, g, 0, table, ws[at:at + need - 1], stream=0)
    refused(-1, bp.bp_relpos_bias_bwd, rp, g, 0, table, ws[at + 1:], stream=0)
    with pytest.raises(ValueError):
        bp.bp_relpos_bias_fwd(rp, table[:7], 0, out, stream=0)
    with pytest.raises(ValueError):
        bp.bp_relpos_bias_fwd(rp, table, 0, out.double(), stream=0)
    with pytest.raises(ValueError):
        bp.bp_relpos_bias_fwd(rp, table, 0, out.transpose(1, 2), stream=0)
    cfg = bp.make_config(10, 10, 4, optimizer="adagrad")
    refused(-1, bp.bp_relpos_update, cfg, rp, table, None, table.clone(), stream=0)
    with pytest.raises(ValueError):
        bp.bp_relpos_update(cfg, rp, table, torch.zeros(3), table.clone(), stream=0)


def test_refusals_of_attention():
    cfg = bp.make_config(100, 100, 64)
    ok = bp.make_attn(4, 2, 16)
    size = bp.bp_embbag_attn_fwd_workspace_bytes
    assert size(cfg, ok, 10, 2) >= 0 and bp.bp_embbag_attn_bwd_workspace_bytes(cfg, ok, None, 10, 2) >= 0
    for bad in (bp.make_attn(3, 2, 16), bp.make_attn(0, 1, 16), bp.make_attn(34, 2, 16), bp.make_attn(2, 2, 12), bp.make_attn(1, 1, 264),
                bp.make_attn(4, 4, 16, 32), bp.make_attn(2, 2, 16, 36), bp.make_attn(4, 4, 16), bp.make_attn(2, 1, 16, cap=-1.0),
                bp.make_attn(2, 1, 16, scale=float("inf")), bp.make_attn(2, 0, 16), bp.make_attn(65, 65, 8)):
        refused(-1, size, cfg, bad, 10, 2)
    refused(-1, size, cfg, ok, -1, 2)
    refused(-6, size, cfg, ok, 1 << 31, 2)
    refused(-6, size, cfg, ok, 4, 1 << 31)
    refused(-1, size, bp.make_config(100, 100, 62), ok, 4, 2)
    w, slots, off = torch.zeros(100, 64), torch.zeros(5, dtype=torch.int32), torch.tensor([0, 5])
    q, lse = torch.zeros(1, 4, 16), torch.zeros(1, 4)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:]
    rp, pos, one, table = bp.make_relpos([1, 2]), torch.zeros(5, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(3, 4)
    fwd = lambda **kw: bp.bp_embbag_attn_fwd(cfg, ok, w, slots, off, 1, q, kw.pop("out", q.clone()), lse, kw.pop("ws", ws), stream=0, **kw)
    refused(-1, fwd, relpos=rp)
    refused(-1, fwd, relpos=rp, q_pos=one, lookup_pos=pos)
    refused(-1, fwd, q_pos=one)
    refused(-1, fwd, weight_in=torch.zeros(5))
    refused(-1, fwd, out=torch.zeros(65)[1:].view(1, 4, 16))                         # not 16-byte aligned
    if size(cfg, ok, 5, 1):
        refused(-3, fwd, ws=ws[:size(cfg, ok, 5, 1) - 1])
    for kw in (dict(bag_lengths=torch.zeros(1, dtype=torch.int64)), dict(weight_out=torch.zeros(4)), dict(out=torch.zeros(1, 4, 15)),
               dict(relpos=rp, q_pos=one, lookup_pos=pos[:4], bias_table=table), dict(relpos=rp, q_pos=one, lookup_pos=pos, bias_table=table[:2])):
        with pytest.raises(ValueError):
            fwd(**kw)
    with pytest.raises(ValueError):
        bp.bp_embbag_attn_fwd(cfg, ok, w, slots, off, 2, q, q.clone(), lse, ws, stream=0)           # offsets, q for one bag
    with pytest.raises(AttributeError):
        bp.bp_embbag_attn_fwd(cfg, ok, w, None, off, 1, q, q.clone(), lse, ws, stream=0)
    bwd = lambda gb, **kw: bp.bp_embbag_attn_bwd(cfg, ok, w, slots, off, 1, q, q, lse, q, q.clone(), torch.zeros(5, 64), gb, ws, stream=0, **kw)
    refused(-1, bwd, table.clone())                                                  # a table's gradient without a table
    refused(-1, bwd, None, relpos=rp, q_pos=one, lookup_pos=pos, bias_table=table)
    with pytest.raises(ValueError):
        bp.bp_embbag_attn_bwd(cfg, ok, w, slots, off, 1, q, q, lse, q, q.clone(), torch.zeros(5, 60), None, ws, stream=0)


def test_refusals_of_eviction():
    off, lens = torch.tensor([0, 4, 9]), torch.tensor([4, 5], dtype=torch.int32)
    f, i, l = (lambda n=9: torch.zeros(n)), (lambda n=9: torch.zeros(n, dtype=torch.int32)), (lambda n=9: torch.zeros(n, dtype=torch.int64))
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:]

    def call(budget=3, sinks=1, recent=1, kw=None, **over):
        a = dict(weight=f(), ids=l(), slots=i(), pos=i(), kept_ids=l(), kept_slots=i(), kept_pos=i(), kept_weight=f(), kept_lengths=i(2),
                 evict_ids=l(4), evict_slots=i(4), evict_offsets=l(3), workspace=ws)
        a.update(over)
        bp.bp_evict_by_weight(off, lens, 2, budget, sinks, recent, *a.values(), stream=0)

    for bad in (dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=2, recent=2), dict(ids=None), dict(kept_ids=None), dict(pos=None),
                dict(kept_pos=None), dict(evict_ids=None), dict(kept_lengths=lens)):
        refused(-1, call, **bad)
    same = i()
    refused(-1, call, slots=same, kept_slots=same)
    wide = i(17)
    refused(-1, call, pos=wide[:9], kept_pos=wide[8:])
    for bad in (dict(weight=f(8)), dict(kept_slots=i(8)), dict(evict_offsets=l(2)), dict(evict_ids=l(3)), dict(slots=l())):
        with pytest.raises(ValueError):
            call(**bad)
    refused(-6, bp.bp_evict_by_weight_workspace_bytes, 1 << 31, 2)
    refused(-6, bp.bp_evict_by_weight_workspace_bytes, 4, 1 << 24)
    refused(-1, bp.bp_evict_by_weight_workspace_bytes, -4, 2)


def test_workspaces_grow_with_the_call():
    """A workspace for the largest call serves every smaller one."""
    sizes, bags = [0, 1, 1023, 4096, 32768, 32769, 524288, 1 << 24], [0, 1, 63, 769, 1100, 2048, 2049, 2561, 1 << 20]
    rp = bp.make_relpos([1, 2, 4], True)
    queries = [bp.bp_evict_by_weight_workspace_bytes]
    for dtype in ("f32", "bf16"):
        cfg = bp.make_config(1000, 1000, 256, dtype)
        for at in (bp.make_attn(4, 4, 16, 0), bp.make_attn(8, 2, 32), bp.make_attn(16, 2, 64), bp.make_attn(3, 1, 40)):
            queries.append(lambda n, b, cfg=cfg, at=at: bp.bp_embbag_attn_fwd_workspace_bytes(cfg, at, n, b, True))
            queries.append(lambda n, b, cfg=cfg, at=at: bp.bp_embbag_attn_bwd_workspace_bytes(cfg, at, rp, n, b))
    for query in queries:
        need = np.array([[query(n, b) for b in bags] for n in sizes])
        assert (np.diff(need, axis=0) >= 0).all() and (np.diff(need, axis=1) >= 0).all()
    lengths = [1, 2, 7, 31, 64, 129, 512, 777, 1024, 2048, 4096]
    for batch, heads in ((1, 1), (1, 5), (3, 5), (2, 16), (8, 64)):
        need = np.array([[bp.bp_relpos_bias_bwd_workspace_bytes(rp, batch, heads, lq, lk) for lk in lengths] for lq in lengths])
        assert (np.diff(need, axis=0) >= 0).all() and (np.diff(need, axis=1) >= 0).all()
