"""The operators of include/tns_layer.h from their definitions, in 64 bits, with a bound of what the same formulas may be off by in 32 bits.

A `V` is a value and its bound.  Every operation hands on what its operands may be off by, to first order, and adds its own rounding: U, half a unit
in the last place of fp32, of its result; sums add U for every addition on the longest way through them (`depth`); exponentials and
logarithms what their comments say.  Results are twice the bound, for other orders of the same operations.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
TINY = 2.0 ** -126      # exponentials and reciprocals below it, no normal numbers, come out as 0: off by themselves, less than this


class V:
    def __init__(self, v, e=0.0):
        self.v = np.asarray(v, np.float64)
        self.e = np.zeros_like(self.v) + e

    def _rounded(self, v, e):
        return V(v, e + U * np.abs(v))

    def __add__(self, o):
        o = o if isinstance(o, V) else V(o)
        return self._rounded(self.v + o.v, self.e + o.e)

    def __neg__(self):
        return V(-self.v, self.e)

    def __sub__(self, o):
        return self + -(o if isinstance(o, V) else V(o))

    def __mul__(self, o):
        o = o if isinstance(o, V) else V(o)
        with np.errstate(invalid="ignore"):
            return self._rounded(self.v * o.v, np.abs(self.v) * o.e + np.abs(o.v) * self.e + self.e * o.e)

    __radd__, __rmul__ = __add__, __mul__

    def __getitem__(self, at):
        return V(self.v[at], self.e[at])

    def sum(self, axis, depth):
        return V(self.v.sum(axis), (self.e + depth * U * (np.abs(self.v) + self.e)).sum(axis))

    def wider(self, relative):
        return V(self.v, self.e + relative * np.abs(self.v))

    def inverse(self):
        with np.errstate(divide="ignore", invalid="ignore"):
            r = 1.0 / self.v
            return V(r, np.abs(r) * (self.e / np.abs(self.v) / np.maximum(1 - self.e / np.abs(self.v), 1e-300) + 2 * U))

    def rsqrt(self):
        r = self.v ** -0.5
        return V(r, np.maximum(self.v - self.e, 1e-300) ** -0.5 - r + 3 * U * r)

    def exp(self):
        """The exponent, rounded once more, is multiplied with log2 e, rounded: 2.5 U of it; the function itself 2 U."""
        r = np.exp(self.v)
        with np.errstate(invalid="ignore"):
            size = np.where(np.isfinite(self.v), np.abs(self.v), 0.0)
        return V(r, r * (np.expm1(np.minimum(self.e, 600)) + 4 * U + 2.5 * U * size) + TINY)

    def log(self):
        r = np.log(self.v)
        return V(r, -np.log1p(-np.minimum(self.e / self.v, 1 - 1e-9)) + 2 * U * np.abs(r) + 2 * U)


def where(c, a, b=0.0):
    b = b if isinstance(b, V) else V(b)
    return V(np.where(c, a.v, b.v), np.where(c, a.e, b.e))


def results(out):
    """name -> value, name_off -> its bound"""
    flat = {}
    for k, x in out.items():
        flat[k], flat[k + "_off"] = x.v, np.where(np.isinf(x.v), 0.0, 2 * x.e)
    return flat


def gap_of(t, before):
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.float32(t) - np.float32(before)
    return np.clip(np.where(np.isnan(d), np.float32(0), d), np.float32(0), np.finfo(np.float32).max)


def attend(rowptr, q, k, v, t=None, ts=None, edges=None, table=None, index=None, mask=None, scale=None, newest_first=False, dout=None):
    """out [S, heads, dim] and, given dout, dq, dk, dv, dtable."""
    S, heads, dim = q.shape
    kv_heads, rows = k.shape[1], int(rowptr[-1])
    group = heads // kv_heads
    scale = dim ** -0.5 if scale is None else scale
    out = V(np.zeros(q.shape))
    dq, dk, dv = V(np.zeros(q.shape)), V(np.zeros(k.shape)), V(np.zeros(v.shape))
    buckets = 1 if table is None else table.shape[0]
    bias = np.zeros((1, heads)) if table is None else table.astype(np.float64)
    dtable, size, count = V(np.zeros((buckets, heads))), np.zeros((buckets, heads)), np.zeros(buckets)
    for s in range(S):
        r = np.arange(int(rowptr[s]), int(rowptr[s + 1]))
        n = len(r)
        if not n:
            continue
        age = gap_of(t[s], ts[r]) if ts is not None else (np.arange(n) if newest_first else n - 1 - np.arange(n))
        bucket = np.zeros(n, np.int64) if buckets == 1 else (np.asarray(edges)[None, :] <= age[:, None]).sum(1)
        left = np.ones(n, bool) if mask is None else np.asarray(mask)[r] != 0
        at = r
        if index is not None:
            left = left & (index[r] >= 0) & (index[r] < k.shape[0])
            at = np.where(left, index[r], 0)
        for h in range(heads):
            of = left & ~np.isneginf(bias[bucket, h])
            rr, b = at[of], bucket[of]
            n = int(of.sum())
            if not n:
                continue
            # online maxima: every sixteen or so events a product with exp(old - new), 5 U at most, so 5 U an event and 100 for what is joined
            depth = 6 * min(n, 1100) + 100
            kk, vv, qq = k[rr, h // group].astype(np.float64), v[rr, h // group].astype(np.float64), q[s, h].astype(np.float64)
            terms = np.concatenate((scale * qq[None] * kk, bias[b, h][:, None]), 1)
            score = V(terms).sum(1, dim + 7)
            e = (score - score.v.max()).exp()
            total = e.sum(0, depth)
            p = e * total.inverse()
            o = (V(p.v[:, None], p.e[:, None]) * vv).sum(0, depth)
            out.v[s, h], out.e[s, h] = o.v, o.e
            if dout is None:
                continue
            d = dout[s, h].astype(np.float64)
            p = p.wider(8 * U)          # once more, from the largest score and one over the sum, rounded
            dp, delta = V(d[None] * vv).sum(1, dim + 3), (o * d).sum(0, dim + 3)
            ds = p * (dp - delta)
            col = lambda x: V(x.v[:, None], x.e[:, None])      # noqa: E731
            g = (col(ds) * kk * scale).sum(0, min(n, 1100) + 60)
            dq.v[s, h], dq.e[s, h] = g.v, g.e
            gk, gv = (col(ds) * (qq * scale)[None]).wider(8 * U), (col(p) * d[None]).wider(8 * U)
            for into, g in ((dk, gk), (dv, gv)):
                into.v[rr, h // group] += g.v
                into.e[rr, h // group] += g.e + group * U * np.abs(g.v)
            np.add.at(dtable.v, (b, h), ds.v)
            np.add.at(dtable.e, (b, h), ds.e)
            np.add.at(size, (b, h), np.abs(ds.v))
            np.add.at(count, b, 1)
    dtable.e += size * U * (np.minimum(count, 4096)[:, None] + 60)
    res = dict(out=out)
    if dout is not None:
        res.update(dq=dq, dk=dk[:rows] if index is None else dk, dv=dv[:rows] if index is None else dv, dtable=dtable)
    return results(res)


def _norm(x, eps, center):
    dim = x.v.shape[1]
    share, deep = V(1.0 / dim, U / dim), min(dim, 8) + 24      # additions: a lane's, the wave's six, the waves' sixteen
    if center:
        mean = x.sum(1, deep) * share
        x = x - V(mean.v[:, None], mean.e[:, None])
    r = ((x * x).sum(1, deep) * share + V(eps, U * eps)).rsqrt()
    r = V(r.v[:, None], r.e[:, None])
    return x * r, r


def _through(g, y, r, center):
    dim = g.v.shape[1]
    share, deep = V(1.0 / dim, U / dim), min(dim, 8) + 24
    along = (g * y).sum(1, deep) * share
    along = V(along.v[:, None], along.e[:, None])
    if center:
        mean = g.sum(1, deep) * share
        return (g - y * along - V(mean.v[:, None], mean.e[:, None])) * r
    return (g - y * along) * r


def block(x, branch, gate=None, scale=None, post=None, pre=None, eps=1e-6, center=False, dout=None, dnext=None):
    """out, next (with pre) and, given dout or dnext, dx, dbranch, dgate, dscale, dpost, dpre."""
    rows, dim = x.shape
    x, y = V(x), V(branch)
    r = None
    if post is not None:
        y, r = _norm(y, eps, center)
    one = np.ones(dim)
    factor = V(one if scale is None else scale) * (one if post is None else post.astype(np.float64))
    z, rest = V(np.ones((rows, dim))), V(np.zeros((rows, dim)))
    if gate is not None:
        u = gate.astype(np.float64)
        off = (1.5 * np.abs(u) + 6) * U
        z, rest = (V(1 / (1 + np.exp(-w)), off / (1 + np.exp(-w)) + TINY) for w in (u, -u))
    out = x + factor * z * y
    res = dict(out=out)
    if pre is not None:
        m, rm = _norm(out, eps, center)
        res["next"] = m * pre
    if dout is None and dnext is None:
        return results(res)
    g = V(np.zeros((rows, dim)) if dout is None else dout)
    if dnext is not None:
        d = V(dnext)
        res["dpre"] = (d * m).sum(0, rows + 20)
        g = g + _through(d * pre, m, rm, center)
    elif pre is not None:
        res["dpre"] = V(np.zeros(dim))
    res["dx"] = g
    g = g * z
    both = (g * y).sum(0, rows + 20)
    if scale is not None:
        res["dscale"] = both if post is None else both * post
    if post is not None:
        res["dpost"] = both if scale is None else both * scale
    g = g * factor
    if gate is not None:
        res["dgate"] = g * y * rest
    res["dbranch"] = g if post is None else _through(g, y, r, center)
    return results(res)


def distill(logits, ids, teacher, lse=None, weight=None, temperature=1.0, scale=1.0):
    """loss, rows [B], dlogits [B, V]."""
    B, n = logits.shape
    rate = 1.0 / temperature
    rows, grad = V(np.zeros(B)), V(np.zeros((B, n)))
    for b in range(B):
        w = 1.0 if weight is None else float(weight[b])
        if w == 0:
            continue
        named = (ids[b] >= 0) & (ids[b] < n)
        at = ids[b][named].astype(np.int64)
        with np.errstate(invalid="ignore"):
            t = teacher[b].astype(np.float64)[named]
        some = ~np.isneginf(t)
        if lse is None and not some.any():
            continue
        by = V(rate, 2 * U * rate)
        t = np.where(some, t, 0.0)
        if lse is None:                                           # (from the largest on: beside a far one the logarithm of the sum would be rounded away)
            t = t - t[some].max()
            tt = V(t, U * np.abs(t)) * by
            l = where(some, tt.exp()).sum(0, len(t) + 30).log()
        else:
            tt, l = V(t) * by, V(float(lse[b]))
        logp = tt - l
        p = where(some, logp.exp())
        mass = p.sum(0, len(t) + 30)
        x = V((logits[b].astype(np.float64) - logits[b].max()))
        x = V(x.v, U * np.abs(x.v)) * V(rate, 2 * U * rate)
        e = x.exp()
        deep = 80 + n // 4096
        total = e.sum(0, deep)
        log_total = total.log()
        logq = x[at] - log_total
        loss = where(p.v > 0, p * (logp - logq)).wider(4 * U).sum(0, 2 * len(t) + 60)
        loss.e += U * (np.abs(p.v * logp.v) + np.abs(p.v * logq.v)).sum() * 3
        inside = np.zeros(n, bool)
        inside[at] = True
        q = e * total.inverse()
        g = q * mass
        if lse is not None:
            rest = V(1.0) - mass
            if rest.v > 0:
                left = ~inside & ~np.isneginf(logits[b])
                g = q * (mass + rest)
                if left.any():
                    # by the others' own largest score: by that of all, a named one far above them would leave their sum no bits
                    raw = logits[b].astype(np.float64)
                    own, down = (np.where(left, raw - raw[left].max(), -np.inf), raw[left].max() - raw.max())
                    eo = (V(own, U * np.abs(np.where(left, own, 0.0))) * V(rate, 2 * U * rate)).exp()
                    others = where(left, eo).sum(0, deep)
                    log_others = others.log() + V(down, U * np.abs(down)) * V(rate, 2 * U * rate)
                    loss = loss + rest * (rest.log() - (log_others - log_total))
                    g = g - where(left, eo * (rest * others.inverse()))
                else:                                             # the student gives the others nothing
                    loss = V(np.inf)
        minus = V(np.zeros(n))
        np.add.at(minus.v, at, p.v)
        np.add.at(minus.e, at, p.e + len(at) * U * p.v)
        g = g - minus
        loss, g = loss * w, g * V(scale * rate * w, 4 * U * abs(scale * rate * w))
        rows.v[b], rows.e[b] = loss.v, loss.e
        grad.v[b], grad.e[b] = g.v, g.e
    return results(dict(rows=rows, loss=rows.sum(0, B + 20) * scale, dlogits=grad))
