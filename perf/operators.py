"""The operators of sequence models over cached rows, case by case: a learned bias by distance with its gradient, bags pooled
by attention with their gradients, and eviction by accumulated attention weight.

A case is one call of one operator:

  bias        bp_relpos_bias_fwd: the [heads][lq][lk] bias that a table of distance buckets gives
  bias_grad   bp_relpos_bias_bwd: the table's gradient from the gradient of that bias, broadcast over a batch
  attn        bp_embbag_attn_fwd: one query token a bag, keys and values in the bag's cached rows; the entries' weights add up
  attn_grad   bp_embbag_attn_bwd: gradients of the queries, of every entry's row and of the bias table
  evict       bp_evict_by_weight: lists over their budget lose the entries of the lowest accumulated weight

`own` false: the operators in elementary torch operations.  `own` true: the library's calls.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def _bias(name, kind, heads, lq, lk, q_start, buckets, far, two_sided, dtype, batch=1):
    return dict(name=name, kind=kind, heads=heads, lq=lq, lk=lk, q_start=q_start, buckets=buckets, far=far,
                two_sided=two_sided, dtype=dtype, batch=batch)


def _attn(name, kind, bags, len_min, len_max, q_heads, kv_heads, head_dim, dtype, capacity, shared=False, cap=0.0,
          buckets=0, far=128, two_sided=False, weights=False, room=False, inside=False, shape_seed=1):
    """shared: the values are the keys.  room: every bag has a stretch of len_max entries, of which it uses its length.
    inside: the query stands somewhere in its sequence, not behind it."""
    return dict(name=name, kind=kind, bags=bags, len_min=len_min, len_max=len_max, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, dtype=dtype, capacity=capacity, shared=shared, cap=cap, buckets=buckets, far=far,
                two_sided=two_sided, weights=weights, room=room, inside=inside, shape_seed=shape_seed)


def _evict(name, bags, len_min, len_max, budget, sinks, recent, shape_seed=1):
    return dict(name=name, kind="evict", bags=bags, len_min=len_min, len_max=len_max, budget=budget, sinks=sinks,
                recent=recent, shape_seed=shape_seed)


def listed():
    return [
        # ---- bias by distance
        # generating one token: the bias of a single query over everything before it; a launch and 128 KB
        _bias("bias_token", "bias", 8, 1, 4_096, 4_095, 32, 128, False, "f32"),
        # a model's bias for a whole sequence, both directions, an odd number of heads and of keys
        _bias("bias_grid", "bias", 15, 2_048, 1_999, 0, 32, 128, True, "bf16"),
        # training: the gradient of a causal bias that a batch of two shares, from a bf16 backward pass
        _bias("bias_grad", "bias_grad", 16, 2_048, 2_048, 0, 32, 128, False, "bf16", batch=2),
        # the same in fp32 at sizes that nothing divides, both directions
        _bias("bias_grad_odd", "bias_grad", 5, 777, 1_001, 100, 16, 300, True, "f32", batch=3),
        # ---- attention over cached rows
        # one user's token: 500 entries, 128 elements of bf16 a row, as the large bf16 configuration has them; latency
        _attn("attn_one", "attn", 1, 500, 500, 8, 2, 32, "bf16", 100_000, buckets=16, weights=True),
        # a batch that generates: 64 sequences of very different lengths in stretches with room to grow, the widest rows,
        # capped scores, bias by distance, weights accumulated for the eviction
        _attn("attn_serve", "attn", 64, 1, 8_192, 16, 4, 64, "bf16", 600_000, cap=30.0, buckets=32, weights=True, room=True),
        # two long contexts: the work is split along the sequence
        _attn("attn_long", "attn", 2, 120_001, 131_072, 16, 2, 128, "bf16", 300_000),
        # pooling short histories of fp32 embeddings (bags of up to 50, 64 elements: the multi-hot configuration), each
        # row its own key and value
        _attn("attn_pool", "attn", 20_000, 0, 50, 4, 4, 16, "f32", 400_000, shared=True),
        # training on histories: rows of keys and values, grouped heads, the query inside its sequence, so that what
        # comes after it is masked (and some bags see nothing)
        _attn("attn_grad", "attn_grad", 2_000, 1, 400, 8, 2, 64, "bf16", 500_000, cap=20.0, buckets=32, inside=True),
        # training the pooled histories
        _attn("attn_grad_pool", "attn_grad", 8_192, 0, 50, 4, 4, 16, "f32", 400_000, shared=True, buckets=16, two_sided=True,
              inside=True),
        # ---- eviction
        # after one more token in each of 32 lists: one entry leaves each
        _evict("evict_step", 32, 1_025, 1_025, 1_024, 4, 64),
        # after prompts: lists of any length come down to their budget
        _evict("evict_batch", 256, 100, 16_384, 8_000, 4, 256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["bias", "bias_grad", "attn", "attn", "attn_grad", "evict"])
    if kind in ("bias", "bias_grad"):
        heads = rng.randint(1, 32)
        batch = 1 if kind == "bias" else rng.randint(1, 4)
        lq = 1 if kind == "bias" and rng.random() < 0.25 else _log_int(rng, 1, 4_096)
        lk = _log_int(rng, 1, min(16_384, max(1, 100_000_000 // (heads * batch * lq))))
        far = _log_int(rng, 20, 2_000)
        return _bias("", kind, heads, lq, lk, rng.choice([0, max(0, lk - lq), rng.randint(0, 4_096)]),
                     rng.randint(2, 32), far, rng.random() < 0.5, rng.choice(["f32", "bf16"]), batch)
    seed = rng.randint(1, 1 << 30)
    if kind == "evict":
        bags = _log_int(rng, 1, 2_000)
        len_max = _log_int(rng, 2, min(300_000, 4_000_000 // bags))
        len_min = rng.randint(0, len_max)
        budget = rng.randint(1, len_max)
        sinks = rng.randint(0, min(8, budget))
        return _evict("", bags, len_min, len_max, budget, sinks, rng.randint(0, budget - sinks), seed)
    dtype = rng.choice(["f32", "bf16"])
    shared = rng.random() < 0.4
    most = (256 if dtype == "f32" else 512) // (1 if shared else 2)          # rows are up to 1,024 bytes
    head_dim = rng.choice([d for d in (16, 24, 32, 40, 48, 64, 80, 96, 128, 256) if d <= most])
    kv_heads = rng.randint(1, min(8, most // head_dim))
    group = rng.choice([1, 1, 2, 3, 4, 6, 8, 16])
    wide = kv_heads * head_dim * max(group, 2)
    bags = _log_int(rng, 1, 20_000)
    # (a bag of one entry has a gradient of zero for its query, of which only rounding is left to compare)
    least = 1 if kind == "attn" else 16
    len_max = _log_int(rng, least, min(131_072, max(least, 70_000_000 // (bags * wide))))
    len_min = rng.randint(0, len_max) if rng.random() < 0.7 else 0
    buckets = rng.choice([0, rng.randint(2, 32)])
    return _attn("", kind, bags, len_min, len_max, kv_heads * group, kv_heads, head_dim, dtype,
                 max(1_000, min(600_000, 2 * bags * len_max)), shared, rng.choice([0.0, 0.0, rng.uniform(5.0, 50.0)]), buckets,
                 _log_int(rng, 20, 2_000), rng.random() < 0.4, kind == "attn" and rng.random() < 0.5, rng.random() < 0.4,
                 rng.random() < 0.5, seed)


# ---------------------------------------------------------------------------------------------------------------------
# shapes and inputs
# ---------------------------------------------------------------------------------------------------------------------
def _borders(buckets, far):
    """Lower ends of the buckets 1 .. buckets-1: the first half one distance each, the others at equal ratios up to `far`, in
    whole numbers (the smallest n with (n/e)^k >= (far/e)^t)."""
    e = max(1, buckets // 2)
    k = buckets - e
    out = list(range(1, e + 1))
    far = max(far, e + 1)
    for t in range(1, k):
        n = int(e * (far / e) ** (t / k))
        while n > 1 and (n - 1) ** k * e ** t >= far ** t * e ** k:
            n -= 1
        while n ** k * e ** t < far ** t * e ** k:
            n += 1
        out.append(max(n, out[-1] + 1))
    return out[:buckets - 1]


def _lengths(case):
    rng = np.random.default_rng(case["shape_seed"])
    return rng.integers(case["len_min"], case["len_max"] + 1, case["bags"])


def _offsets(case, lens):
    room = np.full_like(lens, case["len_max"]) if case.get("room", True) else lens
    return np.concatenate([[0], np.cumsum(room)]).astype(np.int64)


def _row_dim(case):
    return case["kv_heads"] * case["head_dim"] * (1 if case["shared"] else 2)


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _inputs(case, seed):
    g = _gen(seed)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV)
    kind = case["kind"]
    s = {}
    if kind in ("bias", "bias_grad"):
        s["borders"] = _borders(case["buckets"], case["far"])
        rows = case["buckets"] * (2 if case["two_sided"] else 1)
        s["table"] = normal(rows, case["heads"])
        if kind == "bias_grad":
            s["grad"] = normal(case["batch"], case["heads"], case["lq"], case["lk"]).to(_dtype(case))
        return s
    lens = _lengths(case)
    off = _offsets(case, lens)
    n, bags = int(off[-1]), case["bags"]
    s["n"], s["lens_host"], s["off_host"] = n, lens, off
    s["off"] = torch.from_numpy(off).to(DEV)
    s["lens"] = torch.from_numpy(lens.astype(np.int32)).to(DEV)
    if kind == "evict":
        # what many steps of attention leave: a few entries with most of the weight, one in ten never attended to
        w = torch.exp(1.5 * normal(n))
        s["weight"] = torch.where(torch.rand(n, generator=g, device=DEV) < 0.1, torch.zeros_like(w), w)
        s["ids"] = torch.randint(0, 1 << 40, (n,), generator=g, device=DEV)
        s["slots"] = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
        s["pos"] = torch.cumsum(torch.randint(1, 3, (n,), generator=g, device=DEV), 0).to(torch.int32)
        return s
    dim, dt = _row_dim(case), _dtype(case)
    s["cache"] = normal(case["capacity"], dim).to(dt)
    if kind == "attn" and n <= case["capacity"]:
        s["slots"] = torch.randperm(case["capacity"], generator=g, device=DEV)[:n].to(torch.int32)
    else:       # rows that several bags look up, some of them often
        s["slots"] = (torch.rand(n, generator=g, device=DEV) ** 3 * case["capacity"]).to(torch.int32)
    s["q"] = 1.5 * normal(bags, case["q_heads"], case["head_dim"])
    if case["buckets"]:
        s["borders"] = _borders(case["buckets"], case["far"])
        s["table"] = normal(case["buckets"] * (2 if case["two_sided"] else 1), case["q_heads"])
        # positions grow along a bag, with gaps where entries left earlier
        start = s["off"][:-1].repeat_interleave(s["off"][1:] - s["off"][:-1], output_size=n)
        steps = torch.cumsum(1 + (torch.rand(n, generator=g, device=DEV) < 0.1).long(), 0)
        s["pos"] = (steps - (steps[start] if n else steps) + 1).to(torch.int32)
        last = torch.zeros(bags, dtype=torch.int64, device=DEV)
        if n:
            last = torch.where(s["lens"] > 0, s["pos"][(s["off"][:-1] + s["lens"] - 1).clamp(0, n - 1)].long(), last)
        if case["inside"]:
            s["q_pos"] = (torch.rand(bags, generator=g, device=DEV) * (last + 1)).to(torch.int32)
        else:
            s["q_pos"] = (last + 1).to(torch.int32)
    if case["weights"]:
        s["weight"] = torch.rand(n, generator=g, device=DEV)
    if kind == "attn_grad":
        s["grad_out"] = normal(bags, case["q_heads"], case["head_dim"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if kind == "attn_grad":
        # what the training program has from its forward pass
        s["out"], s["lse"] = _attn_plain(case, s)[:2]
    if not own:
        return s
    import paper_2202_12429_amd as bp
    new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=DEV)
    scratch = lambda b: torch.empty(b, dtype=torch.uint8, device=DEV)
    if kind in ("bias", "bias_grad"):
        s["rp"] = bp.make_relpos(s["borders"], case["two_sided"])
        if kind == "bias":
            s["dst"] = new(case["heads"], case["lq"], case["lk"], dtype=_dtype(case))
        else:
            s["dst"] = new(*s["table"].shape)
            s["ws"] = scratch(bp.bp_relpos_bias_bwd_workspace_bytes(s["rp"], case["batch"], case["heads"], case["lq"], case["lk"]))
        return s
    n, bags = s["n"], case["bags"]
    if kind == "evict":
        s["kept"] = [new(n, dtype=torch.int64), new(n, dtype=torch.int32), new(n, dtype=torch.int32), new(n),
                     new(bags, dtype=torch.int32)]
        most = sum(max(0, int(x) - case["budget"]) for x in np.diff(s["off_host"]))
        s["gone"] = [new(most, dtype=torch.int64), new(most, dtype=torch.int32), new(bags + 1, dtype=torch.int64)]
        s["ws"] = scratch(bp.bp_evict_by_weight_workspace_bytes(n, bags))
        return s
    s["cfg"] = bp.make_config(case["capacity"], case["capacity"], _row_dim(case), case["dtype"])
    s["at"] = bp.make_attn(case["q_heads"], case["kv_heads"], case["head_dim"], 0 if case["shared"] else None,
                           scale=1 / math.sqrt(case["head_dim"]), cap=case["cap"])
    s["rp"] = bp.make_relpos(s["borders"], case["two_sided"]) if case["buckets"] else None
    if kind == "attn":
        s["dst"] = [new(bags, case["q_heads"], case["head_dim"]), new(bags, case["q_heads"])]
        s["weight_out"] = new(n) if case["weights"] else None
        s["ws"] = scratch(bp.bp_embbag_attn_fwd_workspace_bytes(s["cfg"], s["at"], n, bags, case["weights"]))
    else:
        s["dst"] = [new(*s["q"].shape), new(n, _row_dim(case)), new(*s["table"].shape) if case["buckets"] else None]
        s["ws"] = scratch(bp.bp_embbag_attn_bwd_workspace_bytes(s["cfg"], s["at"], s["rp"], n, bags))
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"bias": _bias_plain, "bias_grad": _bias_grad_plain, "attn": _attn_plain, "attn_grad": _attn_grad_plain,
                "evict": _evict_plain}[kind](s["case"], s)
    import paper_2202_12429_amd as bp
    c = s["case"]
    if kind == "bias":
        bp.bp_relpos_bias_fwd(s["rp"], s["table"], c["q_start"], s["dst"])
        return [s["dst"]]
    if kind == "bias_grad":
        bp.bp_relpos_bias_bwd(s["rp"], s["grad"], c["q_start"], s["dst"], s["ws"])
        return [s["dst"]]
    if kind == "evict":
        bp.bp_evict_by_weight(s["off"], s["lens"], c["bags"], c["budget"], c["sinks"], c["recent"], s["weight"], s["ids"], s["slots"],
                              s["pos"], *s["kept"], *s["gone"], s["ws"])
        return s["kept"] + s["gone"]
    lens = s["lens"] if c["room"] else None
    if kind == "attn":
        bp.bp_embbag_attn_fwd(s["cfg"], s["at"], s["cache"], s["slots"], s["off"], c["bags"], s["q"], *s["dst"], s["ws"],
                              bag_lengths=lens, relpos=s["rp"], q_pos=s.get("q_pos"), lookup_pos=s.get("pos"),
                              bias_table=s.get("table"), weight_in=s.get("weight"), weight_out=s["weight_out"])
        return s["dst"] + ([s["weight_out"]] if c["weights"] else [])
    bp.bp_embbag_attn_bwd(s["cfg"], s["at"], s["cache"], s["slots"], s["off"], c["bags"], s["q"], s["out"], s["lse"], s["grad_out"],
                          *s["dst"], s["ws"], bag_lengths=lens, relpos=s["rp"], q_pos=s.get("q_pos"), lookup_pos=s.get("pos"),
                          bias_table=s.get("table"))
    return [t for t in s["dst"] if t is not None]


def work(case):
    """Inputs read once, outputs written once, masked places left out where a mask depends on places alone."""
    kind = case["kind"]
    if kind in ("bias", "bias_grad"):
        h, lq, lk = case["heads"], case["lq"], case["lk"]
        width = 4 if case["dtype"] == "f32" else 2
        table = 4 * h * case["buckets"] * (2 if case["two_sided"] else 1)
        if kind == "bias":
            return {"bytes": h * lq * lk * width + table, "flops": h * lq * lk}
        seen = lq * lk if case["two_sided"] else sum(min(lk, case["q_start"] + i + 1) for i in range(lq))
        return {"bytes": case["batch"] * h * seen * width + table, "flops": case["batch"] * h * seen}
    lens = _lengths(case)
    n = int(lens.sum())
    if kind == "evict":
        left = int(np.minimum(lens, case["budget"]).sum())
        return {"bytes": 20 * n + 20 * left + 12 * (n - left) + 16 * case["bags"], "flops": n}
    row = _row_dim(case) * (4 if case["dtype"] == "f32" else 2)
    hd = case["q_heads"] * case["head_dim"]
    per = row + 4 + (4 if case["buckets"] else 0) + (8 if case["weights"] else 0)
    if kind == "attn":
        return {"bytes": n * per + case["bags"] * (8 * hd + 4 * case["q_heads"] + 8), "flops": 4 * n * hd}
    return {"bytes": n * (per + 4 * _row_dim(case)) + case["bags"] * (16 * hd + 4 * case["q_heads"] + 8), "flops": 10 * n * hd}


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _total(t):
    """Sums over the last dimension in 64 bits, in stretches of 1,024."""
    if t.shape[-1] <= 1024:
        return t.sum(-1, dtype=torch.float64)
    parts = torch.nn.functional.pad(t, (0, -t.shape[-1] % 1024)).reshape(*t.shape[:-1], -1, 1024)
    return parts.sum(-1, dtype=torch.float64).sum(-1)


def _buckets_plain(delta, borders, two_sided):
    """delta = query position - key position.  Bucket numbers, and what is seen."""
    away = delta.abs()
    bucket = torch.zeros_like(away)
    for b in borders:
        bucket += away >= b
    if two_sided:
        return torch.where(delta < 0, bucket + len(borders) + 1, bucket), torch.ones_like(delta, dtype=torch.bool)
    return bucket, delta >= 0


def _grid_plain(case, s):
    i = torch.arange(case["lq"], device=DEV)[:, None] + case["q_start"]
    return _buckets_plain(i - torch.arange(case["lk"], device=DEV)[None], s["borders"], case["two_sided"])


def _bias_plain(case, s):
    bucket, seen = _grid_plain(case, s)
    bias = s["table"].t()[:, bucket]
    return [torch.where(seen[None], bias, torch.full_like(bias, -math.inf)).to(_dtype(case))]


def _bias_grad_plain(case, s):
    bucket, seen = _grid_plain(case, s)
    g = s["grad"].float()
    out = torch.zeros_like(s["table"])
    for b in range(out.shape[0]):
        out[b] = _total(torch.where((bucket == b) & seen, g, torch.zeros_like(g))).sum(2).sum(0).float()
    return [out]


def _padded(case, s):
    """Every bag padded to the longest: entry numbers [bags][most] and which of them are entries."""
    most = max(1, int(s["lens_host"].max()))
    k = torch.arange(most, device=DEV)[None]
    entry = k < s["lens"][:, None]
    at = torch.where(entry, s["off"][:-1, None] + k, torch.zeros_like(k))
    return at, entry


def _scores_plain(case, s):
    bags, hq, hk, d = case["bags"], case["q_heads"], case["kv_heads"], case["head_dim"]
    at, seen = _padded(case, s)
    if s["n"]:
        rows = s["cache"][s["slots"][at].long()].float()
    else:
        rows = torch.zeros(bags, 1, _row_dim(case), device=DEV)
    most = rows.shape[1]
    keys = rows[..., :hk * d].reshape(bags, most, hk, d).permute(0, 2, 1, 3).contiguous()
    vals = rows[..., -hk * d:].reshape(bags, most, hk, d).permute(0, 2, 1, 3).contiguous()
    q = s["q"].reshape(bags, hk, hq // hk, d)
    z = torch.matmul(q, keys.transpose(2, 3).contiguous()).reshape(bags, hq, most) / math.sqrt(d)
    bent = None
    if case["cap"]:
        bent = torch.tanh(z / case["cap"])
        z = case["cap"] * bent
    bucket = None
    if case["buckets"]:
        pos = s["pos"][at].long() if s["n"] else torch.zeros_like(at)
        bucket, visible = _buckets_plain(s["q_pos"].long()[:, None] - pos, s["borders"], case["two_sided"])
        z = z + s["table"][bucket].permute(0, 2, 1)
        seen = seen & visible
    z = torch.where(seen[:, None], z, torch.full_like(z, -math.inf))
    return at, seen, keys, vals, q, z, bent, bucket


def _attn_plain(case, s):
    bags, hq, d = case["bags"], case["q_heads"], case["head_dim"]
    at, seen, keys, vals, q, z, bent, bucket = _scores_plain(case, s)
    top = z.amax(2, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    e = torch.exp(z - top)
    total = _total(e)[..., None].float()
    lse = (torch.log(total) + top)[..., 0]
    p = e / torch.where(total > 0, total, torch.ones_like(total))
    out = torch.matmul(p.reshape(bags, case["kv_heads"], -1, p.shape[2]), vals).reshape(bags, hq, d)
    if not case["weights"]:
        return [out, lse]
    weight = torch.zeros_like(s["weight"])
    entry = _padded(case, s)[1]
    weight[at[entry]] = s["weight"][at[entry]] + p.sum(1)[entry]
    return [out, lse, weight]


def _attn_grad_plain(case, s):
    bags, hq, hk, d = case["bags"], case["q_heads"], case["kv_heads"], case["head_dim"]
    at, seen, keys, vals, q, z, bent, bucket = _scores_plain(case, s)
    lse = s["lse"]
    p = torch.exp(z - torch.where(torch.isfinite(lse), lse, torch.zeros_like(lse))[..., None])
    go = s["grad_out"].reshape(bags, hk, hq // hk, d)
    most = p.shape[2]
    dp = torch.matmul(go, vals.transpose(2, 3).contiguous()).reshape(bags, hq, most)
    dz = p * (dp - (s["grad_out"] * s["out"]).sum(2, keepdim=True))
    ds = (dz * (1 - bent * bent) if case["cap"] else dz) / math.sqrt(d)
    grouped = lambda t: t.reshape(bags, hk, hq // hk, most)
    grad_q = torch.matmul(grouped(ds), keys).reshape(bags, hq, d)
    grad_k = torch.matmul(grouped(ds).transpose(2, 3).contiguous(), q).permute(0, 2, 1, 3).reshape(bags, most, hk * d)
    grad_v = torch.matmul(grouped(p).transpose(2, 3).contiguous(), go).permute(0, 2, 1, 3).reshape(bags, most, hk * d)
    entry = _padded(case, s)[1]
    grad_rows = torch.zeros(s["n"], _row_dim(case), device=DEV)
    grad_rows[at[entry]] = (grad_k + grad_v if case["shared"] else torch.cat([grad_k, grad_v], 2))[entry]
    outs = [grad_q, grad_rows]
    if case["buckets"]:
        grad_table = torch.zeros_like(s["table"])
        for b in range(grad_table.shape[0]):
            grad_table[b] = _total(torch.where((bucket == b)[:, None], dz, torch.zeros_like(dz))).sum(0).float()
        outs.append(grad_table)
    return outs


def _evict_plain(case, s):
    bags, budget = case["bags"], case["budget"]
    at, entry = _padded(case, s)
    n, lens, most = s["n"], s["lens"].long(), at.shape[1]
    place = torch.arange(most, device=DEV)[None]
    may = entry & (place >= case["sinks"]) & (place < (lens - case["recent"])[:, None])
    weight = s["weight"][at] if n else torch.zeros(at.shape, device=DEV)
    order = torch.sort(torch.where(may, weight, torch.full_like(weight, math.inf)), dim=1, stable=True).indices
    rank = torch.empty_like(order)
    rank.scatter_(1, order, place.expand(bags, most).contiguous())
    over = (lens - budget).clamp(min=0)
    gone = (rank < over[:, None]) & may
    stay = entry & ~gone
    to = s["off"][:-1, None] + torch.cumsum(stay, 1) - 1
    kept = []
    for t in (s["ids"], s["slots"], s["pos"], s["weight"]):
        k = torch.zeros_like(t)
        k[to[stay]] = t[at[stay]]
        kept.append(k)
    ends = torch.cumsum(over, 0)
    evict_off = torch.cat([torch.zeros_like(ends[:1]), ends])
    room = sum(max(0, int(x) - budget) for x in np.diff(s["off_host"]))
    lists = []
    for t in (s["ids"], s["slots"]):
        k = torch.full((room,), -1, dtype=t.dtype, device=DEV)
        k[(evict_off[:-1, None] + torch.cumsum(gone, 1) - 1)[gone]] = t[at[gone]]
        lists.append(k)
    return kept + [(lens - over).to(torch.int32)] + lists + [evict_off]


# ---------------------------------------------------------------------------------------------------------------------
# the definitions, in 64 bits, bag by bag and bucket by bucket
# ---------------------------------------------------------------------------------------------------------------------
def _bucket_row(delta, borders, two_sided):
    """Buckets of an int64 array of query - key distances; -1: not seen."""
    side = np.searchsorted(np.asarray(borders, dtype=np.int64), np.abs(delta), side="right")
    return np.where(delta >= 0, side, side + len(borders) + 1 if two_sided else -1)


def _exact_bias(case, s):
    # the bias depends on j - i alone: one line of values, of which every query takes a stretch
    line = np.arange(case["q_start"] + case["lq"] - 1, case["q_start"] - case["lk"], -1)
    bucket = torch.from_numpy(_bucket_row(line, s["borders"], case["two_sided"])).to(DEV)
    table = torch.cat([s["table"].double(), torch.full_like(s["table"][:1].double(), -math.inf)])
    values = table[bucket]                                   # bucket -1: the last row
    out = torch.stack([values[case["lq"] - 1 - i:case["lq"] - 1 - i + case["lk"]] for i in range(case["lq"])])
    return [out.permute(2, 0, 1)]


def _exact_bias_grad(case, s):
    out = torch.zeros(s["table"].shape, dtype=torch.float64, device=DEV)
    place = np.arange(case["lk"])
    for i in range(case["lq"]):
        bucket = _bucket_row(case["q_start"] + i - place, s["borders"], case["two_sided"])
        pick = torch.from_numpy((bucket[:, None] == np.arange(out.shape[0])[None]).astype(np.float64)).to(DEV)
        out += torch.matmul(s["grad"][:, :, i].double().sum(0), pick).t()
    return [out]


def _exact_attn(case, s, backward):
    hq, hk, d, r = case["q_heads"], case["kv_heads"], case["head_dim"], case["q_heads"] // case["kv_heads"]
    dim = _row_dim(case)
    f64 = dict(dtype=torch.float64, device=DEV)
    out, lse = torch.zeros(case["bags"], hq, d, **f64), torch.full((case["bags"], hq), -math.inf, **f64)
    weight = torch.zeros(s["n"], **f64) if case["weights"] else None
    gq, gr = torch.zeros(case["bags"], hq, d, **f64), torch.zeros(s["n"], dim, **f64) if backward else None
    gt = torch.zeros(s["table"].shape, **f64) if backward and case["buckets"] else None
    slots = s["slots"].long()
    if case["buckets"]:
        pos, qpos = s["pos"].cpu().numpy().astype(np.int64), s["q_pos"].cpu().numpy().astype(np.int64)
        bucket = np.zeros(s["n"], dtype=np.int64)
        for b in range(case["bags"]):
            a, e = int(s["off_host"][b]), int(s["off_host"][b] + s["lens_host"][b])
            bucket[a:e] = _bucket_row(qpos[b] - pos[a:e], s["borders"], case["two_sided"])
        seen_all, bucket = bucket >= 0, torch.from_numpy(bucket).to(DEV)
        table = s["table"].double()
    for b in range(case["bags"]):
        a, e = int(s["off_host"][b]), int(s["off_host"][b] + s["lens_host"][b])
        if a == e:
            continue
        if weight is not None:
            weight[a:e] = s["weight"][a:e].double()
        pick = torch.arange(a, e, device=DEV)
        if case["buckets"] and not seen_all[a:e].all():
            if not seen_all[a:e].any():
                continue
            pick = pick[torch.from_numpy(seen_all[a:e]).to(DEV)]
        row = s["cache"][slots[pick]].double()
        k = row[:, :hk * d].reshape(-1, hk, d).transpose(0, 1)          # [hk, L, d]
        v = row[:, dim - hk * d:].reshape(-1, hk, d).transpose(0, 1)
        q = s["q"][b].double().reshape(hk, r, d)
        c = torch.matmul(q, k.transpose(1, 2)) * d ** -0.5
        bend = torch.ones_like(c)
        if case["cap"]:
            t = torch.tanh(c / case["cap"])
            c, bend = case["cap"] * t, 1 - t * t
        if case["buckets"]:
            c = c + table[bucket[pick]].t().reshape(hk, r, -1)
        l = torch.logsumexp(c, 2)
        p = torch.exp(c - l[..., None])
        o = torch.matmul(p, v)
        out[b], lse[b] = o.reshape(hq, d), l.reshape(hq)
        if weight is not None:
            weight[pick] += p.sum((0, 1))
        if backward:
            go = s["grad_out"][b].double().reshape(hk, r, d)
            dz = p * (torch.matmul(go, v.transpose(1, 2)) - (go * o).sum(2, keepdim=True))
            ds = dz * bend * d ** -0.5
            gq[b] = torch.matmul(ds, k).reshape(hq, d)
            dk = torch.matmul(ds.transpose(1, 2), q).transpose(0, 1).reshape(-1, hk * d)
            dv = torch.matmul(p.transpose(1, 2), go).transpose(0, 1).reshape(-1, hk * d)
            gr[pick, :hk * d] += dk
            gr[pick, dim - hk * d:] += dv
            if gt is not None:
                one = (bucket[pick][:, None] == torch.arange(gt.shape[0], device=DEV)[None]).double()
                gt += torch.matmul(one.t(), dz.reshape(hq, -1).t())
    if backward:
        return [gq, gr] + ([gt] if gt is not None else [])
    return [out, lse] + ([weight] if weight is not None else [])


def _exact_evict(case, s):
    budget = case["budget"]
    host = {k: s[k].cpu().numpy() for k in ("ids", "slots", "pos", "weight")}
    kept = {k: np.zeros_like(v) for k, v in host.items()}
    lens_out, lists, ends = [], {"ids": [], "slots": []}, [0]
    for a, length in zip(s["off_host"][:-1].tolist(), s["lens_host"].tolist()):
        over = max(0, length - budget)
        mine = np.arange(case["sinks"], max(case["sinks"], length - case["recent"]))
        out = np.sort(mine[np.lexsort((mine, host["weight"][a + mine]))[:over]])
        left = np.delete(np.arange(length), out)
        for k, v in host.items():
            kept[k][a:a + len(left)] = v[a + left]
        for k in lists:
            lists[k].append(host[k][a + out])
        lens_out.append(len(left))
        ends.append(ends[-1] + over)
    room = sum(max(0, int(x) - budget) for x in np.diff(s["off_host"]))
    tail = []
    for k in ("ids", "slots"):
        full = np.full(room, -1, dtype=host[k].dtype)
        full[:ends[-1]] = np.concatenate(lists[k]) if lists[k] else []
        tail.append(full)
    return [kept["ids"], kept["slots"], kept["pos"], kept["weight"].astype(np.float64), np.asarray(lens_out, dtype=np.int32)] + tail + [
        np.asarray(ends, dtype=np.int64)]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "bias":
        return _exact_bias(case, s)
    if case["kind"] == "bias_grad":
        return _exact_bias_grad(case, s)
    if case["kind"] == "evict":
        return _exact_evict(case, s)
    if case["kind"] == "attn_grad" and case["bags"] * case["len_max"] * _row_dim(case) > 3e8:
        return None
    return _exact_attn(case, s, case["kind"] == "attn_grad")
