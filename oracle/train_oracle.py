"""The operators of include/tns_train.h from their definitions, event after event, in 64 bits, with a bound of what the same
formulas may be off by in 32 bits beside every value.  The bounds are running first-order error analyses: U is half a unit in
the last place of fp32; an operation adds U of its result, exp and the reciprocal 2 U; exponents are rounded before they are
raised, which adds their size times 1.5 U (the product with log2 e) or 3.5 U (difference of times, decay, log2 e).  They are
doubled for other orders of the same operations (pieces of a list computed apart and joined).  Test infrastructure only."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
MASK = (1 << 64) - 1
GOLDEN, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


def sigmoid(u):
    return 1.0 / (1.0 + np.exp(-u))


def gap_of(t, before):
    """Rounded to fp32 as times are; NaN counts as 0, infinity as the largest fp32 value."""
    with np.errstate(invalid="ignore", over="ignore"):
        d = float(np.float32(t) - np.float32(before))
    return 0.0 if d != d else min(max(d, 0.0), float(np.finfo(np.float32).max))


def recurrence(rowptr, u, x, ts=None, decay=None, h0=None, t0=None, newest_first=False, dh=None, dlast=None):
    """States h [rows, dim], last [S, dim] and, where dh or dlast is given, du, dx, ddecay, dh0; each also under "<name>_off", its bound."""
    rowptr = np.asarray(rowptr, np.int64)
    S, dim = len(rowptr) - 1, u.shape[1]
    u, x = u.astype(np.float64), x.astype(np.float64)
    lam = np.zeros(dim) if decay is None else decay.astype(np.float64)
    out = {n: np.zeros((u.shape[0], dim)) for n in ("h", "h_off", "du", "du_off", "dx", "dx_off")}
    out.update({n: np.zeros((S, dim)) for n in ("last", "last_off", "dh0", "dh0_off")})
    ddecay, ddecay_size, ddecay_off = np.zeros(dim), np.zeros(dim), np.zeros(dim)
    rows_in_all = int(rowptr[-1])
    backward = dh is not None or dlast is not None
    for s in range(S):
        order = range(int(rowptr[s]), int(rowptr[s + 1]))
        order = list(order)[::-1] if newest_first else list(order)
        h = np.zeros(dim) if h0 is None else h0[s].astype(np.float64)
        off = np.zeros(dim)
        kept = []
        before = None if t0 is None else t0[s]
        for r in order:
            gap = 0.0
            if ts is not None:
                gap = gap_of(ts[r], ts[r] if before is None else before)
                before = ts[r]
            z, rest, e = sigmoid(u[r]), sigmoid(-u[r]), np.exp(-lam * gap)
            f = rest * e
            ez = (1.5 * np.abs(u[r]) + 6) * U
            ef = ez + (3.5 * np.minimum(lam * gap, 200.0) + 3) * U
            kept.append((r, gap, z, rest, f, h, off, ez, ef))
            off = f * off + (ef + 4 * U) * f * np.abs(h) + (ez + 4 * U) * z * np.abs(x[r])
            h = f * h + z * x[r]
            out["h"][r], out["h_off"][r] = h, 2 * off
        out["last"][s], out["last_off"][s] = h, 2 * off
        if not backward:
            continue
        g = np.zeros(dim) if dlast is None else dlast[s].astype(np.float64)
        off = np.zeros(dim)
        for r, gap, z, rest, f, h, h_off, ez, ef in reversed(kept):
            if dh is not None:
                off = off + U * (np.abs(g) + np.abs(dh[r]))
                g = g + dh[r]
            a, b = rest * x[r], f * h
            out["dx"][r], out["dx_off"][r] = z * g, 2 * (z * off + (ez + 2 * U) * np.abs(z * g))
            out["du"][r] = z * g * (a - b)
            out["du_off"][r] = 2 * (z * off * (np.abs(a) + np.abs(b)) + np.abs(z * g) * ((2 * ez + 6 * U) * np.abs(a) + (ez + ef + 6 * U) * np.abs(b) + f * h_off))
            with np.errstate(over="ignore", invalid="ignore"):
                term = np.nan_to_num(g * b * gap)
                ddecay -= term
                ddecay_size += np.abs(term)
                ddecay_off += np.nan_to_num((ef + 4 * U) * np.abs(term) + gap * f * (np.abs(g) * h_off + off * np.abs(h)))
            off = f * off + (ef + 4 * U) * np.abs(f * g)
            g = f * g
        out["dh0"][s], out["dh0_off"][s] = g, 2 * off
    out["ddecay"], out["ddecay_off"] = ddecay, 2 * (ddecay_off + rows_in_all * U * ddecay_size)
    return out


def scan(a, b):
    """h_i = a_i h_{i-1} + b_i along the first axis, in log2(rows) rounds."""
    by = 1
    while by < len(b):
        b = np.concatenate((b[:by], b[by:] + a[by:] * b[:-by]))
        a = np.concatenate((a[:by], a[by:] * a[:-by]))
        by *= 2
    return b


def recurrence_scanned(rowptr, u, x, ts=None, decay=None, h0=None, t0=None, newest_first=False, dh=None, dlast=None, change=None):
    """What recurrence() returns, for lists of many rows: all rows at once, by scans.  Times have to be finite and every list has to hold a row.
    change(f): what a test has a mistake in the factors do (f in the order of the walk)."""
    rowptr = np.asarray(rowptr, np.int64)
    S, n = len(rowptr) - 1, int(rowptr[-1])
    assert (rowptr[1:] > rowptr[:-1]).all()
    flip = (lambda v: v[::-1]) if newest_first else (lambda v: v)
    seq = flip(np.repeat(np.arange(S), np.diff(rowptr)))
    u, x = (flip(v.astype(np.float64)) for v in (u, x))
    first, last = (np.concatenate(([True], seq[1:] != seq[:-1]))[:, None], np.concatenate((seq[1:] != seq[:-1], [True]))[:, None])
    gap, lam = np.zeros((n, 1)), np.zeros(u.shape[1]) if decay is None else decay.astype(np.float64)
    if ts is not None:
        t = flip(ts.astype(np.float32))
        before = np.where(first[:, 0], t if t0 is None else t0.astype(np.float32)[seq], np.concatenate((t[:1], t[:-1])))
        gap = np.maximum(t - before, np.float32(0)).astype(np.float64)[:, None]
    at_first = np.zeros((n, u.shape[1])) if h0 is None else h0.astype(np.float64)[seq]
    z, rest = sigmoid(u), sigmoid(-u)
    f = rest * np.exp(-lam * gap)
    if change is not None:
        f = change(f)
    ez = (1.5 * np.abs(u) + 6) * U
    ef = ez + (3.5 * np.minimum(lam * gap, 200.0) + 3) * U
    inner = np.where(first, 0.0, f)
    shifted = lambda v: np.concatenate((v[:1], v[:-1]))      # noqa: E731
    h = scan(inner, z * x + np.where(first, f * at_first, 0.0))
    enters = np.where(first, at_first, shifted(h))
    off = scan(inner, (ef + 4 * U) * f * np.abs(enters) + (ez + 4 * U) * z * np.abs(x))
    enters_off = np.where(first, 0.0, shifted(off))
    out = dict(h=flip(h), h_off=flip(2 * off))
    ends, begins = np.flatnonzero(last[:, 0]), np.flatnonzero(first[:, 0])
    for name, v in (("last", h), ("last_off", 2 * off)):
        out[name] = np.zeros((S, u.shape[1]))
        out[name][seq[ends]] = v[ends]
    if dh is None and dlast is None:
        return out
    d = np.zeros(u.shape) if dh is None else flip(dh.astype(np.float64))
    end = np.zeros(u.shape) if dlast is None else np.where(last, dlast.astype(np.float64)[seq], 0.0)
    after = lambda v: np.concatenate((v[1:], v[:1]))         # noqa: E731
    back = np.where(last, 0.0, after(f))
    g = scan(back[::-1], (d + end)[::-1])[::-1]
    sent = np.where(last, end, after(f * g))                 # what comes to a row from behind it
    sent_off = np.where(last, 0.0, after((ef + 4 * U) * np.abs(f * g)))
    off = scan(back[::-1], (sent_off + (0 if dh is None else U * (np.abs(sent) + np.abs(d))))[::-1])[::-1]
    a, b = rest * x, f * enters
    out["dx"], out["dx_off"] = flip(z * g), flip(2 * (z * off + (ez + 2 * U) * np.abs(z * g)))
    out["du"] = flip(z * g * (a - b))
    out["du_off"] = flip(2 * (z * off * (np.abs(a) + np.abs(b)) + np.abs(z * g) * ((2 * ez + 6 * U) * np.abs(a) + (ez + ef + 6 * U) * np.abs(b) + f * enters_off)))
    term = g * b * gap
    out["ddecay"] = -term.sum(0)
    out["ddecay_off"] = 2 * (((ef + 4 * U) * np.abs(term) + gap * f * (np.abs(g) * enters_off + off * np.abs(enters))).sum(0) + n * U * np.abs(term).sum(0))
    for name, v in (("dh0", f * g), ("dh0_off", 2 * (f * off + (ef + 4 * U) * np.abs(f * g)))):
        out[name] = np.zeros((S, u.shape[1]))
        out[name][seq[begins]] = v[begins]
    return out


def step(ids, u, x, state, ts=None, decay=None, state_ts=None):
    """(out, out_off, state, state_off, state_ts) after one event for each id."""
    out, off = np.zeros(u.shape), np.zeros(u.shape)
    state, state_off = state.astype(np.float64), np.zeros(state.shape)
    state_ts = None if state_ts is None else state_ts.copy()
    for b, i in enumerate(ids):
        if not 0 <= i < state.shape[0]:
            continue
        one = recurrence([0, 1], u[b: b + 1], x[b: b + 1], None if ts is None else ts[b: b + 1], decay, state[i: i + 1], None if ts is None else state_ts[i: i + 1])
        out[b], off[b] = one["h"][0], one["h_off"][0]
        state[i], state_off[i] = one["h"][0], one["h_off"][0]
        if ts is not None:
            state_ts[i] = ts[b]
    return out, off, state, state_off, state_ts


def softplus(m):
    return np.log1p(np.exp(-np.abs(m))) + np.maximum(m, 0)


def pair_loss(anchor, pos, neg, ref=None, weight=None, beta=1.0, smoothing=0.0, scale=1.0):
    """loss, margin, danchor, dpos, dneg, each with its bound; what lies under a weight of 0 is not looked at."""
    a, p = anchor.astype(np.float64), pos.astype(np.float64)
    B, K, dim = neg.shape
    w = np.ones((B, K)) if weight is None else weight.astype(np.float64)
    some = w != 0
    n = np.where(some[:, :, None], neg, 0).astype(np.float64)
    a, p = (np.where(some.any(1)[:, None], v, 0) for v in (a, p))
    r = np.zeros((B, K)) if ref is None else np.where(some, ref, 0).astype(np.float64)
    beta, smoothing, scale = (float(np.float32(v)) for v in (beta, smoothing, scale))
    plus, minus = (a * p).sum(-1)[:, None], (a[:, None] * n).sum(-1)
    size = (np.abs(a) * np.abs(p)).sum(-1)[:, None] + (np.abs(a)[:, None] * np.abs(n)).sum(-1)
    margin = np.where(some, beta * (plus - minus - r), 0)
    margin_off = np.where(some, 2 * beta * ((dim + 4) * U * size + 4 * U * np.abs(r)), 0)
    terms = scale * w * ((1 - smoothing) * softplus(-margin) + smoothing * softplus(margin))
    terms = np.where(some, terms, 0)
    loss_off = (np.abs(scale * w) * margin_off).sum() + (16 + B * K) * U * np.abs(terms).sum()
    c = np.where(some, scale * w * beta * (smoothing - sigmoid(-margin)), 0)
    c_off = np.where(some, np.abs(scale * w * beta) * (margin_off / 4 + 16 * U), 0)
    diff = p[:, None] - n
    sums = (np.abs(c)[:, :, None] * (np.abs(p)[:, None] + np.abs(n))).sum(1)
    out = dict(loss=terms.sum(), loss_off=2 * loss_off, margin=margin, margin_off=margin_off,
               danchor=(c[:, :, None] * diff).sum(1), danchor_off=2 * ((c_off[:, :, None] * (np.abs(p)[:, None] + np.abs(n))).sum(1) + (K + 4) * U * sums),
               dpos=c.sum(1)[:, None] * a, dpos_off=2 * (c_off.sum(1)[:, None] + (K + 2) * U * np.abs(c).sum(1)[:, None]) * np.abs(a),
               dneg=-c[:, :, None] * a[:, None], dneg_off=2 * (c_off + 2 * U * np.abs(c))[:, :, None] * np.abs(a)[:, None])
    return {k: np.where(some[:, :, None], v, 0) if k.startswith("dneg") else v for k, v in out.items()}


# ---- AdamW, in fp32 operation by operation: what the library has to give bit for bit (the weights themselves: see weights_off) ------

def mix64(z):
    z = np.asarray(z, np.uint64)
    z = (z ^ (z >> np.uint64(30))) * np.uint64(MIX1)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(MIX2)
    return z ^ (z >> np.uint64(31))


def random16(seed, t, first, n):
    """The random bits of n weights of a tensor that begins at weight `first` of the numbering."""
    with np.errstate(over="ignore"):
        key = mix64(np.uint64((seed + GOLDEN * t) & MASK))
        i = np.arange(first, first + n, dtype=np.uint64)
        words = mix64(key + np.uint64(GOLDEN) * (i // np.uint64(4) + np.uint64(1)))
        return ((words >> (np.uint64(16) * (i % np.uint64(4)))) & np.uint64(0xFFFF)).astype(np.int64)


def e4m3_value(code):
    """OCP e4m3 (no infinities, 0x7f is NaN)."""
    code = np.asarray(code, np.int64)
    sign, e, f = np.where(code & 0x80, -1.0, 1.0), (code >> 3) & 15, code & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return (sign * np.where((code & 0x7F) == 0x7F, np.nan, v)).astype(np.float32)


def to_codes(v, signed, random):
    """(codes, scales) of the blocks of 256 of a tensor's values."""
    f = np.float32
    codes, scales = np.zeros(len(v), np.uint8), np.zeros(-(-len(v) // 256), f)
    for k in range(len(scales)):
        part, rnd = v[256 * k: 256 * k + 256], random[256 * k: 256 * k + 256]
        top = np.abs(part).max()
        if top < f(2.0 ** -100):
            continue
        scales[k] = top * f(1.0 / 448.0)
        y = part * (f(448.0) / top)
        if not signed:
            y = np.maximum(y, f(2.0 ** -6))
        bits = y.view(np.uint32).astype(np.int64)
        size = bits & 0x7FFFFFFF
        code = np.minimum(((size + rnd * 16) >> 20) - (120 << 3), 0x7E) | (((bits >> 24) & 0x80) if signed else 0)
        codes[256 * k: 256 * k + 256] = np.where(size < (121 << 23), 0, code)
    return codes, scales


def adamw(param, grad, state, t, first=0, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, seed=0, grad_scale=1.0):
    """One tensor's step.  state: dict(m, v) fp32, or codes with m_scale and v_scale.  Returns (param, weights_off, state)."""
    f = np.float32
    b1, b2 = betas
    eight = "m_scale" in state
    g = grad.astype(f) * f(grad_scale)
    if eight:
        spread = lambda s: np.repeat(s, 256)[: len(param)]      # noqa: E731
        m = e4m3_value(state["m"]) * spread(state["m_scale"])
        r = e4m3_value(state["v"]) * spread(state["v_scale"])
        v = r * r
    else:
        m, v = state["m"], state["v"]
    m = f(b1) * m + f(1 - b1) * g
    v = f(b2) * v + f(1 - b2) * (g * g)
    r = np.sqrt(v)
    change = (f(lr / (1 - b1 ** t)) * m).astype(np.float64) / (r * f(1 / np.sqrt(1 - b2 ** t)) + f(eps)).astype(np.float64)
    new = (param * (f(1) - f(lr) * f(weight_decay))).astype(np.float64) - change
    off = 2 * U * np.abs(new) + 8 * U * np.abs(change)      # a division by the reciprocal, one subtraction
    if not eight:
        return new, off, dict(m=m, v=v)
    random = random16(seed, t, first, len(param))
    (mc, ms), (vc, vs) = to_codes(m, True, random), to_codes(r, False, random)
    return new, off, dict(m=mc, v=vc, m_scale=ms, v_scale=vs)
