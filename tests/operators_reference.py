"""The operators for sequences of cached rows in 64 bits, written from their formulas bag by bag, with bounds for what fp32
arithmetic may be off.  u is the unit of an fp32 rounding, 2^-24."""
import numpy as np

U = 2.0 ** -24


def bucket_rows(distance, borders, two_sided):
    """Table rows of an array of distances (query - key); -1 = not seen."""
    distance = np.asarray(distance, dtype=np.int64)
    b = np.zeros(distance.shape, dtype=np.int64)
    for x in borders:
        b += np.abs(distance) >= int(x)
    return np.where(distance >= 0, b, b + len(borders) + 1 if two_sided else -1)


def bias_grid(table, borders, two_sided, lq, lk, q_start):
    rows = bucket_rows(q_start + np.arange(lq)[:, None] - np.arange(lk)[None], borders, two_sided)
    out = np.where(rows[None] >= 0, np.moveaxis(np.asarray(table, dtype=np.float64)[rows], 2, 0), -np.inf)
    return out, rows


def bias_grad(grad, rows, table_rows):
    """Gradient of the table, and the sums of magnitudes that its error is measured by."""
    heads = grad.shape[1]
    out, size = np.zeros((table_rows, heads)), np.zeros((table_rows, heads))
    for r in range(table_rows):
        g = grad[:, :, rows == r].astype(np.float64)
        out[r], size[r] = g.sum((0, 2)), np.abs(g).sum((0, 2))
    return out, size


class Attention:
    """One batch: rows [n, dim] are the looked-up rows in fp64 (any value where an entry is not seen), seen[n] says which are."""

    def __init__(self, q, rows, seen, spans, hk, value_at, scale, cap, table=None, table_row=None):
        self.q, self.rows, self.seen, self.spans = q.astype(np.float64), rows, seen, spans
        self.hk, self.value_at, self.scale, self.cap, self.table, self.table_row = hk, value_at, scale, cap, table, table_row
        self.bags, self.hq, self.d = q.shape

    def bag(self, b):
        """Entries seen, their keys, values [hk, L, d], scores [hk, r, L], slopes of the cap, bounds of the scores' errors."""
        a, e = self.spans[b]
        pick = a + np.nonzero(self.seen[a:e])[0]
        w = self.hk * self.d
        k = self.rows[pick, :w].reshape(-1, self.hk, self.d).transpose(1, 0, 2)
        v = self.rows[pick, self.value_at:self.value_at + w].reshape(-1, self.hk, self.d).transpose(1, 0, 2)
        q = self.q[b].reshape(self.hk, -1, self.d)
        c = self.scale * (q @ k.transpose(0, 2, 1))
        off = (self.d + 4) * U * abs(self.scale) * (np.abs(q) @ np.abs(k).transpose(0, 2, 1))
        bend = np.ones_like(c)
        if self.cap:
            t = np.tanh(c / self.cap)
            c, bend = self.cap * t, 1 - t * t
            off = off + 8 * U * np.abs(c)
        if self.table is not None:
            c = c + self.table[self.table_row[pick]].astype(np.float64).T.reshape(self.hk, self.hq // self.hk, len(pick))
        return pick, k, v, q, c, bend, off + 4 * U * np.abs(c)

    def forward(self):
        """out, lse, weight sums, and the bounds of all three."""
        out, lse = np.zeros((self.bags, self.hq, self.d)), np.full((self.bags, self.hq), -np.inf)
        weight, t_w = np.zeros(len(self.seen)), np.zeros(len(self.seen))
        t_o, t_l = np.zeros_like(out), np.zeros_like(lse)
        for b in range(self.bags):
            pick, k, v, q, c, bend, off = self.bag(b)
            if not len(pick):
                continue
            top = c.max(2, keepdims=True)
            e = np.exp(c - top)
            total = e.sum(2, keepdims=True)
            p = e / total
            out[b] = (p @ v).reshape(self.hq, self.d)
            lse[b] = (top + np.log(total)).reshape(self.hq)
            weight[pick] = p.sum((0, 1))
            # a score off by x changes p by a factor of 1 +- 2x (its own and the sum's); exp and the sums add their roundings
            rel = 2 * off.max(2, keepdims=True) + (len(pick) + 32) * U + 4 * U * np.abs(c - top)
            t_o[b] = ((p * rel) @ np.abs(v)).reshape(self.hq, self.d) + 1e-37
            t_l[b] = (off.max(2) + 8 * U * (1 + np.abs(lse[b]).reshape(off.shape[:2])) + (len(pick) + 8) * U).reshape(self.hq)
            t_w[pick] = (p * (rel + self.hq * U)).sum((0, 1)) + 1e-37
        return (out, lse, weight), (t_o, t_l, t_w)

    def backward(self, out, lse, grad_out):
        """Gradients of q, of the rows and of the table from the given out and lse, and their bounds."""
        gq, t_q = np.zeros_like(self.q), np.zeros_like(self.q)
        gr, t_r = np.zeros(self.rows.shape), np.zeros(self.rows.shape)
        gt = t_t = None
        if self.table is not None:
            gt, t_t = np.zeros(self.table.shape), np.zeros(self.table.shape)
        w = self.hk * self.d
        flat = lambda x: x.transpose(1, 0, 2).reshape(-1, w)
        for b in range(self.bags):
            pick, k, v, q, c, bend, off = self.bag(b)
            if not len(pick):
                continue
            go, o = grad_out[b].astype(np.float64).reshape(q.shape), out[b].astype(np.float64).reshape(q.shape)
            l = lse[b].astype(np.float64).reshape(self.hk, -1, 1)
            p = np.exp(c - l)
            dp, d0 = go @ v.transpose(0, 2, 1), (go * o).sum(2, keepdims=True)
            dz = p * (dp - d0)
            ds = dz * bend * self.scale
            e_p = p * (off + 8 * U + 4 * U * np.abs(c - l))
            e_d = (self.d + 4) * U * (np.abs(go) @ np.abs(v).transpose(0, 2, 1) + np.abs(go * o).sum(2, keepdims=True))
            e_z = p * e_d + np.abs(dp - d0) * e_p + 4 * U * np.abs(dz)
            e_bend = 0 if not self.cap else 2 * (off / self.cap + 4 * U)          # 1 - t^2, with t off by as much as c / cap
            e_s = abs(self.scale) * (e_z * bend + np.abs(dz) * e_bend) + 4 * U * np.abs(ds)
            n = len(pick) + 8
            gq[b] = (ds @ k).reshape(self.hq, self.d)
            t_q[b] = ((e_s + n * U * np.abs(ds)) @ np.abs(k)).reshape(self.hq, self.d)
            r = q.shape[1] + 8
            gr[pick, :w] += flat(ds.transpose(0, 2, 1) @ q)
            t_r[pick, :w] += flat((e_s + r * U * np.abs(ds)).transpose(0, 2, 1) @ np.abs(q))
            gr[pick, self.value_at:self.value_at + w] += flat(p.transpose(0, 2, 1) @ go)
            t_r[pick, self.value_at:self.value_at + w] += flat((e_p + r * U * p).transpose(0, 2, 1) @ np.abs(go))
            if gt is not None:
                z, ez = dz.reshape(self.hq, -1), (e_z + n * U * np.abs(dz)).reshape(self.hq, -1)
                for i, at in enumerate(self.table_row[pick]):
                    gt[at] += z[:, i]
                    t_t[at] += ez[:, i]
        return (gq, gr, gt), (t_q, t_r, t_t)


def evict(spans, weight, budget, sinks, recent):
    """Per list: the places that stay and the places that leave, in order.  NaN counts as above every number, -0 as 0."""
    out = []
    for a, e in spans:
        n = e - a
        over = max(0, n - budget)
        may = np.arange(sinks, max(sinks, n - recent))
        w = weight[a:e][may].astype(np.float64) + 0.0
        may = may[np.lexsort((may, np.where(np.isnan(w), 0.0, w), np.isnan(w)))]
        leaves = np.zeros(n, dtype=bool)
        leaves[may[:over]] = True
        out.append((np.nonzero(~leaves)[0].tolist(), np.nonzero(leaves)[0].tolist()))
    return out
